// RMS norms on either side of a block with the residual stream between them, one pass over the data.
//
//   z = y * r2 * w_post, r2 = (mean y^2 + eps)^-1/2   (or z = y without a norm behind the block)
//   x' = res_scale * x + gate * z                      n = x' * r1 * w_pre, r1 = (mean x'^2 + eps)^-1/2
// Backward, from dx' and dn, with xh = x' r1, yh = y r2:
//   D = dx' + r1 (w_pre dn - xh mean(w_pre dn xh));  dx = res_scale D;  dgate = D z (summed over the row for one gate a token)
//   dy = r2 (gate D w_post - yh mean(gate D w_post yh));  dw_pre = sum dn xh;  dw_post = sum gate D yh      (sums over the rows)
// The backward pass takes r1 and r2 from the rows it reads anyway; nothing is saved for it but x' and y.
//
// Bound by memory: every tensor is read or written once.  W waves share a row, a lane holds CH pieces of 8 values of
// every tensor, so that all of a row's loads are in flight together and stay in registers across the row's sums; the weights
// stay there from row to row.  Blocks walk the rows with a stride; weight gradients collect in registers, one partial
// row per block goes to the workspace, and a second kernel adds the partial rows in a fixed order.  16384 rows of 4096 in bf16, one gate
// a token: forward 98 us (537 MB at 5.5 TB/s), backward 153 us (805 MB at 5.3 TB/s); a plain copy moves 4.8 to 5.2 TB/s.  777 rows of 7168 in fp32 with
// a gate an element 47 us (122 MB at 2.6 TB/s; 40 + 5 in its kernels): a block a unit, so three rounds of rows and a fourth of nine rows, and a row's
// loads, sums and stores one behind the other, with no register left for the next row's.
// Requesting the next row's tensors while a row is finished gained nothing (backward 152 -> 161 and, in the kernel, 39 -> 39 us).
#include "wave_ops.h"

#include <algorithm>
#include <type_traits>

namespace relibra {

constexpr int kNormMaxWaves = 16, kComputeUnits = 256;
constexpr int kNormMaxWidth = kNormMaxWaves * 64 * 8;      // 16 waves of one piece a lane, or 8 of two

struct NormShape {
    int T, h, waves, rows_per_block;                          // waves of a row, rows in flight in a block
    float res_scale, eps;
};

// Sums of N values over the row's waves: wave results through LDS.  `turn` alternates between two sets of slots, so that one
// barrier a reduction suffices.
template <int N> __device__ __forceinline__ void row_sums(float (&v)[N], int waves, int first_wave, float (*slots)[3][kNormMaxWaves], int &turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = group_sum<64>(v[i]);
    if (waves == 1) return;
    float(*s)[kNormMaxWaves] = slots[turn];
    turn ^= 1;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[i][wave] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0.0f;
        for (int w = 0; w < waves; ++w) v[i] += s[i][first_wave + w];
    }
}

enum { GATE_NONE = 0, GATE_TOKEN = 1, GATE_ELEMENT = 2 };

template <class XT, int CH, int GATE>
__global__ void __launch_bounds__(CH == 1 ? 1024 : 512)
norm_fwd_kernel(NormShape sh, const XT *x, const bf16_t *y, const bf16_t *__restrict__ w_post, const bf16_t *__restrict__ w_pre,
                const void *__restrict__ gate, XT *x_out, bf16_t *n)          // (x_out may be x, n may be y: a lane reads its pieces of a row first)
{
    __shared__ float slots[2][3][kNormMaxWaves];
    int turn = 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, slot = wave / sh.waves, first_wave = slot * sh.waves;
    const int h = sh.h, pieces = h >> 3, lanes = sh.waves * 64, pos = (wave - first_wave) * 64 + lane;
    const float inv_h = 1.0f / (float)h;
    Raw8<bf16_t> w2[CH], w1[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = c * lanes + pos;
        w2[c] = w_post && at < pieces ? fetch8(w_post + at * 8) : zero8<bf16_t>();
        w1[c] = w_pre && at < pieces ? fetch8(w_pre + at * 8) : zero8<bf16_t>();
    }
    for (int row0 = blockIdx.x * sh.rows_per_block; row0 < sh.T; row0 += gridDim.x * sh.rows_per_block) {
        const bool live = row0 + slot < sh.T;
        const int row = min(row0 + slot, sh.T - 1);
        const size_t base = (size_t)row * h;
        Raw8<XT> xr[CH];
        Raw8<bf16_t> yr[CH], gr[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = c * lanes + pos;
            const bool in = at < pieces;
            xr[c] = in ? fetch8(x + base + at * 8) : zero8<XT>();
            yr[c] = in && y ? fetch8(y + base + at * 8) : zero8<bf16_t>();
            gr[c] = GATE == GATE_ELEMENT && in ? fetch8((const bf16_t *)gate + base + at * 8) : zero8<bf16_t>();
        }
        const float g_tok = GATE == GATE_TOKEN ? ((const float *)gate)[row] : 1.0f;
        float v[CH][8];
        if (y) {
            float r2 = 1.0f;
            if (w_post) {
                float s[1] = {0.0f};
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    float yv[8];
                    unpack8(yr[c], yv);
#pragma unroll
                    for (int j = 0; j < 8; ++j) s[0] += yv[j] * yv[j];
                }
                row_sums(s, sh.waves, first_wave, slots, turn);
                r2 = 1.0f / sqrtf(s[0] * inv_h + sh.eps);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float xv[8], yv[8], wv[8], gv[8];
                unpack8(xr[c], xv);
                unpack8(yr[c], yv);
                unpack8(w2[c], wv);
                unpack8(gr[c], gv);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float z = w_post ? yv[j] * r2 * wv[j] : yv[j];
                    v[c][j] = sh.res_scale * xv[j] + (GATE == GATE_ELEMENT ? gv[j] : g_tok) * z;
                }
                const int at = c * lanes + pos;
                if (live && at < pieces) store8(x_out + base + at * 8, v[c]);
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) unpack8(xr[c], v[c]);
        }
        if (w_pre) {
            float s[1] = {0.0f};
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) s[0] += v[c][j] * v[c][j];
            row_sums(s, sh.waves, first_wave, slots, turn);
            const float r1 = 1.0f / sqrtf(s[0] * inv_h + sh.eps);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float wv[8];
                unpack8(w1[c], wv);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] = v[c][j] * r1 * wv[j];
                const int at = c * lanes + pos;
                if (live && at < pieces) store8(n + base + at * 8, v[c]);
            }
        }
    }
}

template <class XT, int CH, int GATE>
__global__ void __launch_bounds__(CH == 1 ? 1024 : 512)
norm_bwd_kernel(NormShape sh, const XT *__restrict__ x_out, const XT *dx_out, const bf16_t *dn, const bf16_t *y,
                const bf16_t *__restrict__ w_post, const bf16_t *__restrict__ w_pre, const void *__restrict__ gate,
                XT *dx, bf16_t *dy, void *__restrict__ dgate, float *__restrict__ part_post, float *__restrict__ part_pre, int add)
{
    __shared__ float slots[2][3][kNormMaxWaves];
    int turn = 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, slot = wave / sh.waves, first_wave = slot * sh.waves;
    const int h = sh.h, pieces = h >> 3, lanes = sh.waves * 64, pos = (wave - first_wave) * 64 + lane;
    const float inv_h = 1.0f / (float)h;
    Raw8<bf16_t> w2[CH], w1[CH];
    float acc2[CH][8], acc1[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int at = c * lanes + pos;
        w2[c] = w_post && at < pieces ? fetch8(w_post + at * 8) : zero8<bf16_t>();
        w1[c] = w_pre && at < pieces ? fetch8(w_pre + at * 8) : zero8<bf16_t>();
#pragma unroll
        for (int j = 0; j < 8; ++j) acc2[c][j] = acc1[c][j] = 0.0f;
    }
    for (int row0 = blockIdx.x * sh.rows_per_block; row0 < sh.T; row0 += gridDim.x * sh.rows_per_block) {
        const bool live = row0 + slot < sh.T;
        const int row = min(row0 + slot, sh.T - 1);
        const size_t base = (size_t)row * h;
        Raw8<XT> xr[CH], dr[CH];
        Raw8<bf16_t> yr[CH], nr[CH], gr[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int at = c * lanes + pos;
            const bool in = at < pieces;
            xr[c] = in && w_pre ? fetch8(x_out + base + at * 8) : zero8<XT>();
            nr[c] = in && w_pre ? fetch8(dn + base + at * 8) : zero8<bf16_t>();
            yr[c] = in && y ? fetch8(y + base + at * 8) : zero8<bf16_t>();
            dr[c] = in && dx_out ? fetch8(dx_out + base + at * 8) : zero8<XT>();
            gr[c] = GATE == GATE_ELEMENT && in ? fetch8((const bf16_t *)gate + base + at * 8) : zero8<bf16_t>();
        }
        const float g_tok = GATE == GATE_TOKEN ? ((const float *)gate)[row] : 1.0f;
        float s[3] = {0.0f, 0.0f, 0.0f};                      // x'^2, w_pre dn x', y^2
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float xv[8], nv[8], yv[8], wv[8];
            unpack8(xr[c], xv);
            unpack8(nr[c], nv);
            unpack8(yr[c], yv);
            unpack8(w1[c], wv);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[0] += xv[j] * xv[j];
                s[1] += wv[j] * nv[j] * xv[j];
                s[2] += yv[j] * yv[j];
            }
        }
        row_sums(s, sh.waves, first_wave, slots, turn);
        const float r1 = 1.0f / sqrtf(s[0] * inv_h + sh.eps), m1 = s[1] * r1 * inv_h;
        const float r2 = w_post ? 1.0f / sqrtf(s[2] * inv_h + sh.eps) : 1.0f;
        float D[CH][8], q[2] = {0.0f, 0.0f};                  // sums of D z and of gate D z
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float xv[8], nv[8], yv[8], wv[8], vv[8], gv[8];
            unpack8(xr[c], xv);
            unpack8(nr[c], nv);
            unpack8(yr[c], yv);
            unpack8(w1[c], wv);
            unpack8(w2[c], vv);
            unpack8(gr[c], gv);
            unpack8(dr[c], D[c]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float xh = xv[j] * r1;
                D[c][j] += r1 * (wv[j] * nv[j] - xh * m1);
                if (live) acc1[c][j] += nv[j] * xh;
                const float z = w_post ? yv[j] * r2 * vv[j] : yv[j];
                q[0] += D[c][j] * z;
                if (GATE == GATE_ELEMENT) q[1] += D[c][j] * gv[j] * z;
            }
            const int at = c * lanes + pos;
            float out[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) out[j] = sh.res_scale * D[c][j];
            if (live && at < pieces) store8(dx + base + at * 8, out);
        }
        if (!y) continue;                                     // the same for all of the grid
        float m2 = 0.0f;
        if (w_post || GATE == GATE_TOKEN) {
            row_sums(q, sh.waves, first_wave, slots, turn);
            m2 = (GATE == GATE_ELEMENT ? q[1] : g_tok * q[0]) * inv_h;
            if (GATE == GATE_TOKEN && live && pos == 0) ((float *)dgate)[row] = q[0];
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float yv[8], vv[8], gv[8], out[8], dg[8];
            unpack8(yr[c], yv);
            unpack8(w2[c], vv);
            unpack8(gr[c], gv);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float dz = (GATE == GATE_ELEMENT ? gv[j] : g_tok) * D[c][j], yh = yv[j] * r2;
                dg[j] = D[c][j] * (w_post ? yh * vv[j] : yv[j]);
                out[j] = w_post ? r2 * (dz * vv[j] - yh * m2) : dz;
                if (live) acc2[c][j] += dz * yh;
            }
            const int at = c * lanes + pos;
            if (live && at < pieces) {
                store8(dy + base + at * 8, out);
                if (GATE == GATE_ELEMENT) store8((bf16_t *)dgate + base + at * 8, dg);
            }
        }
    }
    // the block's row groups, in ascending order: one partial row a block, or (one block, `add` with RELIBRA_NORM_ACCUMULATE) the gradient itself
    extern __shared__ __attribute__((aligned(16))) char smem[];
    float *join = reinterpret_cast<float *>(smem);            // [rows_per_block - 1][h]
    auto leave = [&](const float (&acc)[CH][8], float *to) __attribute__((always_inline)) {
        if (!to) return;
        __syncthreads();
        if (slot > 0)
#pragma unroll
            for (int c = 0; c < CH; ++c)
                if (c * lanes + pos < pieces) store8(join + (size_t)(slot - 1) * h + (c * lanes + pos) * 8, acc[c]);
        __syncthreads();
        if (slot == 0)
#pragma unroll
            for (int c = 0; c < CH; ++c)
                if (c * lanes + pos < pieces) {
                    float sum[8], v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[j] = acc[c][j];
                    for (int r = 1; r < sh.rows_per_block; ++r) {
                        load8(join + (size_t)(r - 1) * h + (c * lanes + pos) * 8, v);
#pragma unroll
                        for (int j = 0; j < 8; ++j) sum[j] += v[j];
                    }
                    if (add) {
                        load8(to + (c * lanes + pos) * 8, v);
#pragma unroll
                        for (int j = 0; j < 8; ++j) sum[j] += v[j];
                    }
                    store8(to + (size_t)blockIdx.x * h + (c * lanes + pos) * 8, sum);
                }
    };
    leave(acc2, part_post);
    leave(acc1, part_pre);
}

// dw (+)= the sum of P partial rows: 32 columns a block, 128 strips of rows, joined in ascending order.
constexpr int kReduceStrips = 128;
__global__ void __launch_bounds__(kReduceStrips * 8)
norm_reduce_kernel(const float *__restrict__ part0, const float *__restrict__ part1, float *__restrict__ dw0, float *__restrict__ dw1, int P, int h, int add)
{
    __shared__ float4 join[kReduceStrips][8];
    const float *part = blockIdx.y ? part1 : part0;
    float *dw = blockIdx.y ? dw1 : dw0;
    if (!dw) return;
    const int col = threadIdx.x & 7, strip = threadIdx.x >> 3, at = blockIdx.x * 32 + col * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (at < h)
#pragma unroll 4
        for (int p = strip; p < P; p += kReduceStrips) {
            const float4 v = *reinterpret_cast<const float4 *>(part + (size_t)p * h + at);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    join[strip][col] = s;
    __syncthreads();
    // 128 strips to 8, then one thread a column the rest
    if (strip < 8) {
        for (int i = strip + 8; i < kReduceStrips; i += 8) {
            const float4 v = join[i][col];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        join[strip][col] = s;
    }
    __syncthreads();
    if (strip == 0 && at < h) {
        for (int i = 1; i < 8; ++i) {
            const float4 v = join[i][col];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        float4 *to = reinterpret_cast<float4 *>(dw + at);
        if (add) {
            const float4 o = *to;
            s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
        }
        *to = s;
    }
}

struct NormGrid {
    int chunks, waves, rows_per_block, blocks;
};
// Forward: two pieces a lane, four waves a block, 16 waves a unit, half of them where a block then still has 16 rounds; few rows are
// latency and get twice the waves instead.  us, 16384 rows of 4096 in bf16 at 16 / 8 waves a unit 102 / 98, 4096 of 2048 12.2 / 13.4; 700 of
// 8192 in fp32 with one / two pieces 16.3 / 14.5.
// Backward: one piece a lane (two take 173 registers instead of 110: half the waves), eight waves a block, 16 a unit: 16384 rows of 4096 in one
// session 157 us, with 8 waves a unit 200, 32 167; with two pieces and four waves a block 176.  The row groups of a block are joined in LDS: with a
// partial row each the second kernel took longer than the first, 8000 rows of 512 56 -> 16 us, 4096 of 2048 48 -> 25.
// Up to four rounds of rows are one block's, without a second launch: us a call, 4 rows of 4096 12.9 (two launches 15.7), 4 of 8192 15.0 (15.8), 8 of
// 4096 18.0 (15.7).
constexpr int kOneBlockRounds = 4;
inline NormGrid norm_grid(int T, int h, bool bwd)
{
    NormGrid g;
    const int pieces = h / 8;
    g.chunks = bwd || pieces <= 64 || T < 256 ? 1 : 2;
    g.waves = (pieces + 64 * g.chunks - 1) / (64 * g.chunks);
    const int block_waves = bwd ? 8 : 4;
    g.rows_per_block = g.waves >= block_waves ? 1 : block_waves / g.waves;
    const int groups = (T + g.rows_per_block - 1) / g.rows_per_block;
    int want = kComputeUnits * std::max(1, 16 / (g.waves * g.rows_per_block));
    if (!bwd && groups >= 16 * want) want = std::max(kComputeUnits, want / 2);
    if (bwd && groups <= kOneBlockRounds) want = 1;
    g.blocks = std::max(1, std::min(groups, want));
    return g;
}
inline size_t norm_join_bytes(const NormGrid &g, int h) { return (size_t)(g.rows_per_block - 1) * h * sizeof(float); }
inline bool norm_takes(int T, int h) { return h % 8 == 0 && h <= kNormMaxWidth && T <= 1 << 30; }
size_t norm_ws_bytes(int T, int h)
{
    if (h < 8 || !norm_takes(T, h)) return 0;
    const NormGrid g = norm_grid(T, h, true);
    return 2 * round256((size_t)g.blocks * h * sizeof(float));
}

inline int check_norm(int T, int h, int flags, int known, float eps)
{
    if (T < 0 || h < 8 || (flags & ~known) || !(eps > 0.0f)) return RELIBRA_EINVAL;
    if (!norm_takes(T, h)) return RELIBRA_EUNSUPPORTED;
    if ((flags & RELIBRA_NORM_GATE_TOKEN) && (flags & RELIBRA_NORM_GATE_ELEMENT)) return RELIBRA_EINVAL;
    return RELIBRA_OK;
}
inline int gate_kind(int flags) { return flags & RELIBRA_NORM_GATE_TOKEN ? GATE_TOKEN : flags & RELIBRA_NORM_GATE_ELEMENT ? GATE_ELEMENT : GATE_NONE; }

template <bool TWO, class Fn> int norm_layout(int chunks, int gate, const Fn &fn)
{
    auto with_gate = [&](auto ch) {
        if (gate == GATE_TOKEN) return fn(ch, std::integral_constant<int, GATE_TOKEN>{});
        if (gate == GATE_ELEMENT) return fn(ch, std::integral_constant<int, GATE_ELEMENT>{});
        return fn(ch, std::integral_constant<int, GATE_NONE>{});
    };
    if constexpr (TWO)
        if (chunks == 2) return with_gate(std::integral_constant<int, 2>{});
    return with_gate(std::integral_constant<int, 1>{});
}

template <class XT>
int norm_fwd_impl(const XT *x, const bf16_t *y, const bf16_t *w_post, const bf16_t *w_pre, const void *gate, int gkind, const NormShape &sh, const NormGrid &g,
                  XT *x_out, bf16_t *n, hipStream_t stream)
{
    return norm_layout<true>(g.chunks, gkind, [&](auto ch, auto gk) {
        RELIBRA_LAUNCH(RELIBRA_K_NORM_FWD, stream, (norm_fwd_kernel<XT, decltype(ch)::value, decltype(gk)::value>
            <<<g.blocks, g.waves * g.rows_per_block * 64, 0, stream>>>(sh, x, y, w_post, w_pre, gate, x_out, n)));
        return RELIBRA_OK;
    });
}
template <class XT>
int norm_bwd_impl(const XT *x_out, const XT *dx_out, const bf16_t *dn, const bf16_t *y, const bf16_t *w_post, const bf16_t *w_pre, const void *gate, int gkind,
                  const NormShape &sh, const NormGrid &g, XT *dx, bf16_t *dy, void *dgate, float *part_post, float *part_pre, int add, hipStream_t stream)
{
    return norm_layout<false>(g.chunks, gkind, [&](auto ch, auto gk) {
        RELIBRA_LAUNCH(RELIBRA_K_NORM_BWD, stream, (norm_bwd_kernel<XT, decltype(ch)::value, decltype(gk)::value>
            <<<g.blocks, g.waves * g.rows_per_block * 64, norm_join_bytes(g, sh.h), stream>>>(sh, x_out, dx_out, dn, y, w_post, w_pre, gate, dx, dy, dgate, part_post, part_pre, add)));
        return RELIBRA_OK;
    });
}

}  // namespace relibra

using namespace relibra;

extern "C" int relibra_block_norm_fwd(const void *x, const void *y, const void *w_post, const void *w_pre, const void *gate, int T, int h,
                                      float res_scale, float eps, int flags, void *x_out, void *n, relibra_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    const int rc = check_norm(T, h, flags, RELIBRA_NORM_STREAM_FP32 | RELIBRA_NORM_GATE_TOKEN | RELIBRA_NORM_GATE_ELEMENT, eps);
    if (rc != RELIBRA_OK) return rc;
    const int gkind = gate_kind(flags);
    if (T == 0) return RELIBRA_OK;                            // (an empty tensor may be a null pointer)
    if (!y && (w_post || gkind != GATE_NONE || !w_pre)) return RELIBRA_EINVAL;
    if (!x || (y && !x_out) || (w_pre && !n) || (gkind != GATE_NONE && !gate)) return RELIBRA_EINVAL;
    if (!aligned16(x) || !aligned16(y) || !aligned16(w_post) || !aligned16(w_pre) || (gkind == GATE_ELEMENT && !aligned16(gate)) || !aligned16(x_out) || !aligned16(n)) return RELIBRA_EINVAL;
    const NormGrid g = norm_grid(T, h, false);
    const NormShape sh{T, h, g.waves, g.rows_per_block, res_scale, eps};
    if (flags & RELIBRA_NORM_STREAM_FP32)
        norm_fwd_impl((const float *)x, (const bf16_t *)y, (const bf16_t *)w_post, (const bf16_t *)w_pre, gate, gkind, sh, g, (float *)x_out, (bf16_t *)n, stream);
    else
        norm_fwd_impl((const bf16_t *)x, (const bf16_t *)y, (const bf16_t *)w_post, (const bf16_t *)w_pre, gate, gkind, sh, g, (bf16_t *)x_out, (bf16_t *)n, stream);
    RELIBRA_HIP_TRY(launch_check());
    return RELIBRA_OK;
}

extern "C" int relibra_block_norm_bwd(const void *x_out, const void *dx_out, const void *dn, const void *y, const void *w_post, const void *w_pre,
                                      const void *gate, int T, int h, float res_scale, float eps, int flags, void *dx, void *dy, void *dgate,
                                      float *dw_post, float *dw_pre, void *workspace, size_t workspace_bytes, relibra_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    const int rc = check_norm(T, h, flags, RELIBRA_NORM_STREAM_FP32 | RELIBRA_NORM_GATE_TOKEN | RELIBRA_NORM_GATE_ELEMENT | RELIBRA_NORM_ACCUMULATE, eps);
    if (rc != RELIBRA_OK) return rc;
    const int gkind = gate_kind(flags);
    if ((w_post && !dw_post) || (w_pre && !dw_pre)) return RELIBRA_EINVAL;
    if (T > 0) {
        if (!dx || (y && !dy) || (w_pre && (!x_out || !dn)) || (!w_pre && !dx_out) || (gkind != GATE_NONE && (!gate || !dgate))) return RELIBRA_EINVAL;
        if (!y && (w_post || gkind != GATE_NONE || !w_pre)) return RELIBRA_EINVAL;
    }
    for (const void *p : {x_out, dx_out, dn, y, w_post, w_pre, (const void *)dx, (const void *)dy, (const void *)dw_post, (const void *)dw_pre,
                          (const void *)workspace})
        if (!aligned16(p)) return RELIBRA_EINVAL;
    if (gkind == GATE_ELEMENT && (!aligned16(gate) || !aligned16(dgate))) return RELIBRA_EINVAL;
    const NormGrid g = norm_grid(T, h, true);
    const int P = T > 0 ? g.blocks : 0;
    if ((w_post || w_pre) && (!workspace || workspace_bytes < norm_ws_bytes(T, h))) return RELIBRA_EWORKSPACE;
    const bool one = P == 1;                                  // one block's sums are the gradients: no second launch
    float *part_post = !w_post ? nullptr : one ? dw_post : (float *)workspace;
    float *part_pre = !w_pre ? nullptr : one ? dw_pre : (float *)((char *)workspace + norm_ws_bytes(T, h) / 2);
    const int add = flags & RELIBRA_NORM_ACCUMULATE ? 1 : 0;
    if (T > 0) {
        const NormShape sh{T, h, g.waves, g.rows_per_block, y ? res_scale : 1.0f, eps};
        if (flags & RELIBRA_NORM_STREAM_FP32)
            norm_bwd_impl((const float *)x_out, (const float *)dx_out, (const bf16_t *)dn, (const bf16_t *)y, (const bf16_t *)w_post, (const bf16_t *)w_pre, gate, gkind,
                          sh, g, (float *)dx, (bf16_t *)dy, dgate, part_post, part_pre, one && add, stream);
        else
            norm_bwd_impl((const bf16_t *)x_out, (const bf16_t *)dx_out, (const bf16_t *)dn, (const bf16_t *)y, (const bf16_t *)w_post, (const bf16_t *)w_pre, gate, gkind,
                          sh, g, (bf16_t *)dx, (bf16_t *)dy, dgate, part_post, part_pre, one && add, stream);
    }
    if ((w_post || w_pre) && !one)
        RELIBRA_LAUNCH(RELIBRA_K_NORM_REDUCE, stream, norm_reduce_kernel<<<dim3((h + 31) / 32, 2), kReduceStrips * 8, 0, stream>>>(
            part_post, part_pre, w_post ? dw_post : nullptr, w_pre ? dw_pre : nullptr, P, h, add));
    RELIBRA_HIP_TRY(launch_check());
    return RELIBRA_OK;
}
