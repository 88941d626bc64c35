// RMS norms of queries and keys for each head and the rotation by their positions, one pass over the data.
//
//   x^ = x * r, r = (mean x^2 + eps)^-1/2 over a head's d values;  u = w x^  (u = x without a norm)
//   pairs (a, b) of the first `rot` values of u turn by theta = pos[axis] * freq:   a' = a cos - b sin,  b' = b cos + a sin
// Backward, from g' = dL/du': g = the pairs of g' turned by -theta;  dx = r (w g - x^ mean(w g x^)),  dw = sum g x^ over tokens and heads.
//
// Bound by memory: every value is read and written once.  A group of 4, 8 or 16 lanes holds a head (16 values a lane, as two pieces of
// 8 whose values are pairs of each other, so that a turn needs no other lane); a wave takes 64 / group heads of a token at a time.  The
// angles of a token are its own for all heads: a lane takes one pair, in double (a far position's angle has no bits left in fp32),
// and the wave's cosines and sines go through LDS once.  Weight gradients stay in registers from token to token; a block leaves
// one partial row, added up in a fixed order by a second kernel.
// 16384 tokens of 64 + 4 heads of 128: 112 us forward (5.1 TB/s, what a copy reaches), 171 us backward with the second kernel (5.0).
// One token: 2.7 us on the GPU, the latency of tables, angles and heads one after the other.
#include "head_rows.h"
#include "row_reduce.h"
#include "wave_ops.h"

#include <algorithm>
#include <type_traits>

namespace relibra {

constexpr int kQkMaxDim = 256, kQkMaxPairs = kQkMaxDim / 2, kQkThreads = 256, kQkWaves = kQkThreads / 64;
// Blocks a unit; backward as many as its registers let run at once, each leaves a row of sums: 16384 tokens of 64 + 4 heads with 3, 4, 6, 8 a unit
// 171, 185, 176, 178 us backward, 113.3, 115.5, 117.7, 113.0 forward.
constexpr int kQkBlocks = 256 * 8, kQkBwdBlocks = 256 * 3;

struct QkShape {
    int T, Hq, Hk, d, rot;
    int q_passes, passes, groups, per_group;                  // passes of a wave over a token's heads, dealt to `groups` waves
    float eps;
    uint32_t axis[kQkMaxPairs / 16];                          // two bits a pair
};
struct QkTables {
    const int32_t *pos;                                       // [axes][T]
    const float *freq;
    const bf16_t *w_q, *w_k;
};

// Where a lane's two pieces of 8 values lie in a head, and its eight pairs among them.
template <bool ADJ> struct QkLane {
    int at0, at1;
    bool in, turns;
    __device__ __forceinline__ QkLane(int pos, int d, int rot)
    {
        const int quarter = rot >> 4;                         // lanes that hold pairs
        in = pos < (d >> 4);
        turns = pos < quarter;
        const bool split = !ADJ && turns;
        at0 = split ? pos * 8 : pos * 16;
        at1 = split ? (pos + quarter) * 8 : pos * 16 + 8;
    }
    // (values of the two pieces) -> turned, by +theta or, with s = -1, by -theta
    static __device__ __forceinline__ void turn(float (&v0)[8], float (&v1)[8], const float2 *angles, float sign)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 at = angles[i];
            float &a = ADJ ? (i < 4 ? v0[2 * (i & 3)] : v1[2 * (i & 3)]) : v0[i];
            float &b = ADJ ? (i < 4 ? v0[2 * (i & 3) + 1] : v1[2 * (i & 3) + 1]) : v1[i];
            const float sn = sign * at.y, x = a * at.x - b * sn;
            b = b * at.x + a * sn;
            a = x;
        }
    }
};

// The cosines and sines of a token's pairs, through the wave's LDS.  Angles in whole turns: the position times the frequency in double,
// less its nearest integer; what is left has 24 good bits up to positions of 2^28.
__device__ __forceinline__ void qk_angles(const QkShape &sh, const QkTables &tab, int token, int lane, float2 *slot)
{
    for (int j = lane; j < sh.rot >> 1; j += 64) {
        const int axis = sh.axis[j >> 4] >> ((j & 15) * 2) & 3;
        const double turns = (double)tab.pos[(size_t)axis * sh.T + token] * (double)tab.freq[j] * 0.15915494309189535;
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        slot[j] = make_float2(c, s);
    }
}

// Weights as loaded to fp32, at every use: left to itself the compiler keeps them unpacked, 32 registers more.
__device__ __forceinline__ void unpack_weights(Raw8<bf16_t> r, float (&w)[8])
{
    asm volatile("" : "+v"(r.q.x), "+v"(r.q.y), "+v"(r.q.z), "+v"(r.q.w));
    unpack8(r, w);
}

template <int LANES, bool ADJ>
__global__ void __launch_bounds__(kQkThreads)
qk_fwd_kernel(QkShape sh, QkTables tab, const bf16_t *q, size_t q_ld, const bf16_t *k, size_t k_ld, bf16_t *q_out, size_t qo_ld, bf16_t *k_out, size_t ko_ld)
{
    constexpr int HEADS = 64 / LANES;
    __shared__ float2 angles[kQkWaves][kQkMaxPairs];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pos = lane & (LANES - 1);
    const QkLane<ADJ> me(pos, sh.d, sh.rot);
    const float inv_d = 1.0f / (float)sh.d;
    Raw8<bf16_t> wq[2], wk[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        wq[i] = tab.w_q && me.in ? fetch8(tab.w_q + (i ? me.at1 : me.at0)) : zero8<bf16_t>();
        wk[i] = tab.w_k && me.in ? fetch8(tab.w_k + (i ? me.at1 : me.at0)) : zero8<bf16_t>();
    }
    const long long items = (long long)sh.T * sh.groups;      // (below 2^31: groups are few tokens')
    for (long long item = (long long)blockIdx.x * kQkWaves + wave; item < items; item += (long long)gridDim.x * kQkWaves) {
        const int token = (int)(sh.groups == 1 ? (unsigned)item : (unsigned)item / (unsigned)sh.groups), group = (int)(item - (long long)token * sh.groups);
        if (sh.rot) {
            wave_lds_fence();                                 // the last token's are read
            qk_angles(sh, tab, token, lane, angles[wave]);
            wave_lds_fence();
        }
        auto pass = [&](auto is_q, int head) __attribute__((always_inline)) {
            constexpr bool Q = decltype(is_q)::value;
            const bool in = me.in && head < (Q ? sh.Hq : sh.Hk);
            const size_t col = (size_t)head * sh.d;
            const bf16_t *x = Q ? q + token * q_ld + col : k + token * k_ld + col;
            float v0[8], v1[8];
            unpack8(in ? fetch8(x + me.at0) : zero8<bf16_t>(), v0);
            unpack8(in ? fetch8(x + me.at1) : zero8<bf16_t>(), v1);
            if (Q ? tab.w_q != nullptr : tab.w_k != nullptr) {
                float sum = 0.0f, w0[8], w1[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += v0[i] * v0[i] + v1[i] * v1[i];
                const float r = 1.0f / sqrtf(group_sum<LANES>(sum) * inv_d + sh.eps);
                unpack_weights(Q ? wq[0] : wk[0], w0);
                unpack_weights(Q ? wq[1] : wk[1], w1);
#pragma unroll
                for (int i = 0; i < 8; ++i) v0[i] = v0[i] * r * w0[i], v1[i] = v1[i] * r * w1[i];
            }
            if (me.turns) me.turn(v0, v1, angles[wave] + pos * 8, 1.0f);
            if (in) {
                bf16_t *y = Q ? q_out + token * qo_ld + col : k_out + token * ko_ld + col;
                store8(y + me.at0, v0);
                store8(y + me.at1, v1);
            }
        };
        const int p0 = group * sh.per_group, p1 = min(p0 + sh.per_group, sh.passes), mine = lane / LANES;
#pragma unroll 1
        for (int p = p0; p < min(p1, sh.q_passes); ++p) pass(std::true_type{}, p * HEADS + mine);
#pragma unroll 1
        for (int p = max(p0, sh.q_passes); p < p1; ++p) pass(std::false_type{}, (p - sh.q_passes) * HEADS + mine);
    }
}

template <int LANES, bool ADJ>
__global__ void __launch_bounds__(kQkThreads)
qk_bwd_kernel(QkShape sh, QkTables tab, const bf16_t *q, size_t q_ld, const bf16_t *k, size_t k_ld, const bf16_t *dq_out, size_t dqo_ld, const bf16_t *dk_out,
              size_t dko_ld, bf16_t *dq, size_t dq_ld, bf16_t *dk, size_t dk_ld, float *__restrict__ part_q, float *__restrict__ part_k, int add)
{
    constexpr int HEADS = 64 / LANES;
    __shared__ float2 angles[kQkWaves][kQkMaxPairs];
    __shared__ __attribute__((aligned(16))) float join[kQkWaves][kQkMaxDim];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pos = lane & (LANES - 1);
    const QkLane<ADJ> me(pos, sh.d, sh.rot);
    const float inv_d = 1.0f / (float)sh.d;
    Raw8<bf16_t> wq[2], wk[2];
    float acc_q[16], acc_k[16];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        wq[i] = tab.w_q && me.in ? fetch8(tab.w_q + (i ? me.at1 : me.at0)) : zero8<bf16_t>();
        wk[i] = tab.w_k && me.in ? fetch8(tab.w_k + (i ? me.at1 : me.at0)) : zero8<bf16_t>();
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) acc_q[i] = acc_k[i] = 0.0f;
    const long long items = (long long)sh.T * sh.groups;
    for (long long item = (long long)blockIdx.x * kQkWaves + wave; item < items; item += (long long)gridDim.x * kQkWaves) {
        const int token = (int)(sh.groups == 1 ? (unsigned)item : (unsigned)item / (unsigned)sh.groups), group = (int)(item - (long long)token * sh.groups);
        if (sh.rot) {
            wave_lds_fence();
            qk_angles(sh, tab, token, lane, angles[wave]);
            wave_lds_fence();
        }
        auto pass = [&](auto is_q, int head) __attribute__((always_inline)) {
            constexpr bool Q = decltype(is_q)::value;
            const bool in = me.in && head < (Q ? sh.Hq : sh.Hk), norm = Q ? tab.w_q != nullptr : tab.w_k != nullptr;
            const size_t col = (size_t)head * sh.d;
            const bf16_t *up = Q ? dq_out + token * dqo_ld + col : dk_out + token * dko_ld + col;
            const bf16_t *x = Q ? q + token * q_ld + col : k + token * k_ld + col;
            const Raw8<bf16_t> x0 = in && norm ? fetch8(x + me.at0) : zero8<bf16_t>(), x1 = in && norm ? fetch8(x + me.at1) : zero8<bf16_t>();
            float g0[8], g1[8];
            unpack8(in ? fetch8(up + me.at0) : zero8<bf16_t>(), g0);
            unpack8(in ? fetch8(up + me.at1) : zero8<bf16_t>(), g1);
            if (me.turns) me.turn(g0, g1, angles[wave] + pos * 8, -1.0f);
            if (norm) {
                float v0[8], v1[8], w0[8], w1[8], sum = 0.0f, dot = 0.0f;
                unpack8(x0, v0);
                unpack8(x1, v1);
                unpack_weights(Q ? wq[0] : wk[0], w0);
                unpack_weights(Q ? wq[1] : wk[1], w1);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sum += v0[i] * v0[i] + v1[i] * v1[i];
                    dot += w0[i] * g0[i] * v0[i] + w1[i] * g1[i] * v1[i];
                }
                const float r = 1.0f / sqrtf(group_sum<LANES>(sum) * inv_d + sh.eps);
                const float md = group_sum<LANES>(dot) * r * inv_d, m = r > 0.0f ? md : 0.0f;      // (an infinite rms leaves zeros, whatever the products' sum)
                float(&acc)[16] = Q ? acc_q : acc_k;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float h0 = v0[i] * r, h1 = v1[i] * r;
                    acc[i] += g0[i] * h0;                     // (lanes without a head hold zeros)
                    acc[8 + i] += g1[i] * h1;
                    g0[i] = r * (w0[i] * g0[i] - h0 * m);
                    g1[i] = r * (w1[i] * g1[i] - h1 * m);
                }
            }
            if (in) {
                bf16_t *y = Q ? dq + token * dq_ld + col : dk + token * dk_ld + col;
                store8(y + me.at0, g0);
                store8(y + me.at1, g1);
            }
        };
        const int p0 = group * sh.per_group, p1 = min(p0 + sh.per_group, sh.passes), mine = lane / LANES;
#pragma unroll 1
        for (int p = p0; p < min(p1, sh.q_passes); ++p) pass(std::true_type{}, p * HEADS + mine);
#pragma unroll 1
        for (int p = max(p0, sh.q_passes); p < p1; ++p) pass(std::false_type{}, (p - sh.q_passes) * HEADS + mine);
    }
    // the wave's groups by swaps of lanes, the block's waves through LDS: one partial row a block, or (one block) the gradient itself
    auto leave = [&](float (&acc)[16], float *to) __attribute__((always_inline)) {
        if (!to) return;
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = place_sum<LANES>(acc[i]);
        __syncthreads();
        if (lane < LANES && me.in)
#pragma unroll
            for (int i = 0; i < 8; ++i) join[wave][me.at0 + i] = acc[i], join[wave][me.at1 + i] = acc[8 + i];
        __syncthreads();
        for (int i = threadIdx.x; i < sh.d; i += kQkThreads) {
            float sum = join[0][i];
            for (int w = 1; w < kQkWaves; ++w) sum += join[w][i];
            float *at = to + (size_t)blockIdx.x * sh.d + i;
            *at = add ? *at + sum : sum;
        }
    };
    leave(acc_q, part_q);
    leave(acc_k, part_k);
}

struct QkGrid {
    int lanes, blocks;
};
// A token's heads are one wave's where there are tokens for all waves; else its passes are dealt out to several.
inline QkGrid qk_grid(int T, int Hq, int Hk, int d, bool bwd, QkShape &sh)
{
    QkGrid g;
    g.lanes = d <= 64 ? 4 : d <= 128 ? 8 : 16;
    const int heads = 64 / g.lanes;
    sh.T = T, sh.Hq = Hq, sh.Hk = Hk, sh.d = d;
    sh.q_passes = (Hq + heads - 1) / heads;
    sh.passes = sh.q_passes + (Hk + heads - 1) / heads;
    const int blocks = bwd ? kQkBwdBlocks : kQkBlocks, slots = blocks * kQkWaves;
    sh.groups = std::max(1, std::min(sh.passes, slots / std::max(T, 1)));
    sh.per_group = (sh.passes + sh.groups - 1) / sh.groups;
    sh.groups = (sh.passes + sh.per_group - 1) / sh.per_group;
    const long long items = (long long)T * sh.groups;
    g.blocks = (int)std::max<long long>(1, std::min<long long>((items + kQkWaves - 1) / kQkWaves, blocks));
    return g;
}
inline bool qk_takes(int T, int Hq, int Hk, int d) { return d % 16 == 0 && d <= kQkMaxDim && T <= 1 << 30 && Hq <= 4096 && Hk <= 4096; }
size_t qk_ws_bytes(int T, int Hq, int Hk, int d)
{
    if (d < 16 || Hq < 1 || Hk < 0 || !qk_takes(T, Hq, Hk, d)) return 0;
    QkShape sh;
    return 2 * round256((size_t)qk_grid(T, Hq, Hk, d, true, sh).blocks * d * sizeof(float));
}

// What both calls check of the sizes and tables; fills in the axes.
inline int check_qk(const void *w_q, const void *w_k, const int32_t *pos, const float *freq, const uint8_t *axis, int n_axes, int T, int Hq, int Hk, int d,
                    int rot, float eps, int flags, int known, QkShape &sh)
{
    if (T < 0 || Hq < 1 || Hk < 0 || d < 16 || rot < 0 || rot > d || (flags & ~known)) return RELIBRA_EINVAL;
    if (!qk_takes(T, Hq, Hk, d) || rot % 16) return RELIBRA_EUNSUPPORTED;
    if ((w_q || w_k) && !(eps > 0.0f)) return RELIBRA_EINVAL;
    if (!rot && !w_q && !w_k) return RELIBRA_EINVAL;          // nothing to do
    if (w_k && !Hk) return RELIBRA_EINVAL;
    if (!aligned16(w_q) || !aligned16(w_k)) return RELIBRA_EINVAL;
    std::fill(sh.axis, sh.axis + kQkMaxPairs / 16, 0u);
    if (rot) {
        if (n_axes < 1 || n_axes > 4) return n_axes < 1 ? RELIBRA_EINVAL : RELIBRA_EUNSUPPORTED;
        if (T > 0 && (!pos || !freq)) return RELIBRA_EINVAL;
        if (axis)
            for (int j = 0; j < rot / 2; ++j) {
                if (axis[j] >= n_axes) return RELIBRA_ERANGE;
                sh.axis[j >> 4] |= (uint32_t)axis[j] << ((j & 15) * 2);
            }
    }
    sh.rot = rot, sh.eps = eps;
    return RELIBRA_OK;
}

// The tables' sizes, 0 where the call reads none.
inline size_t qk_pos_bytes(int T, int n_axes, int rot) { return rot ? (size_t)n_axes * T * sizeof(int32_t) : 0; }
inline size_t qk_freq_bytes(int rot) { return (size_t)rot / 2 * sizeof(float); }

template <class Fn> void qk_layout(int lanes, bool adjacent, const Fn &fn)
{
    auto with = [&](auto n) {
        if (adjacent) fn(n, std::true_type{});
        else fn(n, std::false_type{});
    };
    if (lanes == 4) with(std::integral_constant<int, 4>{});
    else if (lanes == 8) with(std::integral_constant<int, 8>{});
    else with(std::integral_constant<int, 16>{});
}

}  // namespace relibra

using namespace relibra;

extern "C" int relibra_qk_norm_rope_fwd(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *w_q, const void *w_k, const int32_t *pos,
                                        const float *freq, const uint8_t *axis, int n_axes, int T, int Hq, int Hk, int d, int rot, float eps, int flags,
                                        void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride, relibra_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    QkShape sh;
    const int rc = check_qk(w_q, w_k, pos, freq, axis, n_axes, T, Hq, Hk, d, rot, eps, flags, RELIBRA_ROPE_ADJACENT, sh);
    if (rc != RELIBRA_OK) return rc;
    if (T == 0) return RELIBRA_OK;
    const HeadRows in[2] = {{q, q_stride, Hq * d}, {k, k_stride, Hk * d}}, out[2] = {{q_out, q_out_stride, Hq * d}, {k_out, k_out_stride, Hk * d}};
    for (int i = 0; i < 2; ++i) {
        if (!in[i].usable() || !out[i].usable()) return RELIBRA_EINVAL;
        if (!in[i].same(out[i]) && in[i].overlaps(out[i], T)) return RELIBRA_EINVAL;
        if (in[1 - i].overlaps(out[i], T)) return RELIBRA_EINVAL;
    }
    if (out[0].overlaps(out[1], T)) return RELIBRA_EINVAL;
    if (!pieces_apart(T, {}, {out[0], out[1]}, {{w_q, d * sizeof(bf16_t)}, {w_k, d * sizeof(bf16_t)}, {pos, qk_pos_bytes(T, n_axes, rot)}, {freq, qk_freq_bytes(rot)}}, {}))
        return RELIBRA_EINVAL;
    const QkGrid g = qk_grid(T, Hq, Hk, d, false, sh);
    const QkTables tab{pos, freq, (const bf16_t *)w_q, (const bf16_t *)w_k};
    qk_layout(g.lanes, flags & RELIBRA_ROPE_ADJACENT, [&](auto n, auto adj) {
        RELIBRA_LAUNCH(RELIBRA_K_QK_FWD, stream, (qk_fwd_kernel<decltype(n)::value, decltype(adj)::value><<<g.blocks, kQkThreads, 0, stream>>>(
            sh, tab, (const bf16_t *)q, q_stride, (const bf16_t *)k, k_stride, (bf16_t *)q_out, q_out_stride, (bf16_t *)k_out, k_out_stride)));
    });
    RELIBRA_HIP_TRY(launch_check());
    return RELIBRA_OK;
}

extern "C" int relibra_qk_norm_rope_bwd(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *dq_out, int64_t dq_out_stride,
                                        const void *dk_out, int64_t dk_out_stride, const void *w_q, const void *w_k, const int32_t *pos, const float *freq,
                                        const uint8_t *axis, int n_axes, int T, int Hq, int Hk, int d, int rot, float eps, int flags, void *dq,
                                        int64_t dq_stride, void *dk, int64_t dk_stride, float *dw_q, float *dw_k, void *workspace, size_t workspace_bytes,
                                        relibra_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    QkShape sh;
    const int rc = check_qk(w_q, w_k, pos, freq, axis, n_axes, T, Hq, Hk, d, rot, eps, flags, RELIBRA_ROPE_ADJACENT | RELIBRA_QK_ACCUMULATE, sh);
    if (rc != RELIBRA_OK) return rc;
    if ((w_q && !dw_q) || (w_k && !dw_k) || !aligned16(dw_q) || !aligned16(dw_k) || !aligned16(workspace)) return RELIBRA_EINVAL;
    const HeadRows in[4] = {{dq_out, dq_out_stride, Hq * d}, {dk_out, dk_out_stride, Hk * d}, {w_q ? q : nullptr, q_stride, w_q ? Hq * d : 0},
                            {w_k ? k : nullptr, k_stride, w_k ? Hk * d : 0}};
    const HeadRows out[2] = {{dq, dq_stride, Hq * d}, {dk, dk_stride, Hk * d}};
    if (T > 0) {
        for (const HeadRows &r : in)
            if (!r.usable()) return RELIBRA_EINVAL;
        for (int i = 0; i < 2; ++i) {
            if (!out[i].usable()) return RELIBRA_EINVAL;
            for (int j = 0; j < 4; ++j)
                if (in[j].overlaps(out[i], T) && !(j % 2 == i && in[j].same(out[i]))) return RELIBRA_EINVAL;
        }
        if (out[0].overlaps(out[1], T)) return RELIBRA_EINVAL;
    }
    const bool norms = w_q || w_k;
    const size_t need = norms ? qk_ws_bytes(T, Hq, Hk, d) : 0;
    if (norms && (!workspace || workspace_bytes < need)) return RELIBRA_EWORKSPACE;
    // (one tensor for both weights' gradients would have two blocks add to the same values at once)
    if (!pieces_apart(T, {in[0], in[1], in[2], in[3]}, {out[0], out[1]},
                      {{w_q, d * sizeof(bf16_t)}, {w_k, d * sizeof(bf16_t)}, {pos, qk_pos_bytes(T, n_axes, rot)}, {freq, qk_freq_bytes(rot)}},
                      {{w_q ? dw_q : nullptr, d * sizeof(float)}, {w_k ? dw_k : nullptr, d * sizeof(float)}, {workspace, need}}))
        return RELIBRA_EINVAL;
    const QkGrid g = qk_grid(T, Hq, Hk, d, true, sh);
    const int P = T > 0 ? g.blocks : 0, add = flags & RELIBRA_QK_ACCUMULATE ? 1 : 0;
    const bool one = P == 1;
    float *part_q = !w_q ? nullptr : one ? dw_q : (float *)workspace;
    float *part_k = !w_k ? nullptr : one ? dw_k : (float *)((char *)workspace + need / 2);
    const QkTables tab{pos, freq, (const bf16_t *)w_q, (const bf16_t *)w_k};
    if (T > 0)
        qk_layout(g.lanes, flags & RELIBRA_ROPE_ADJACENT, [&](auto n, auto adj) {
            RELIBRA_LAUNCH(RELIBRA_K_QK_BWD, stream, (qk_bwd_kernel<decltype(n)::value, decltype(adj)::value><<<g.blocks, kQkThreads, 0, stream>>>(
                sh, tab, (const bf16_t *)q, q_stride, (const bf16_t *)k, k_stride, (const bf16_t *)dq_out, dq_out_stride, (const bf16_t *)dk_out, dk_out_stride,
                (bf16_t *)dq, dq_stride, (bf16_t *)dk, dk_stride, part_q, part_k, one && add)));
        });
    if (norms && !one)
        RELIBRA_LAUNCH(RELIBRA_K_QK_REDUCE, stream, row_reduce_kernel<<<dim3((d + 31) / 32, 2), kReduceStrips * 8, 0, stream>>>(
            part_q, part_k, w_q ? dw_q : nullptr, w_k ? dw_k : nullptr, P, d, add));
    RELIBRA_HIP_TRY(launch_check());
    return RELIBRA_OK;
}
