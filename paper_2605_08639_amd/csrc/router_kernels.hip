// Router gates of replayed expert ids, the load-balance loss over per-expert counts, and the logits' gradient.
//
// A token's E logits z give log scores u = z (softmax) or u = log sigmoid(z), probabilities p = softmax(u), and gates on
// the replayed ids: exp(u) over the sum of the token's k selected (normalised), or p (softmax) or sigmoid(z) as they are, times
// `scale`.  With f_e = counts_e / (k n) over the n valid tokens of a micro-batch and P_e = mean p_e, the loss is coef E sum_e f_e P_e.
//
// sigmoid(z) = exp(min(z, 0)) / (1 + exp(-|z|)), so both scores are w = exp(v - m) * r with v = z, r = 1 or v = min(z, 0),
// r = 1 / (1 + exp(-|z|)), and m the largest v of the set that is summed over: the row for p, the selected alone for normalised gates
// (their ratio survives however far below the row's maximum they lie).  A set of -infinities only has the sum 0 and yields zeros.
//
// Layout: LT lanes share a token (2, 8, 16, 32 or 64: the least with 8 LT >= E), each holds 8 consecutive experts of every CH-th
// run, so a wave has 64 / LT tokens in flight, rows are read in 16-byte pieces, and a lane's experts stay its own
// over all tokens: sum_t p_te accumulates in registers, and only the finished sums of a block are stored.
#include "wave_ops.h"

#include <algorithm>
#include <type_traits>

namespace relibra {

constexpr int kRouterMaxExperts = 4096;

struct RouterShape {
    int T, k, E, flags;
    float scale;
};

// exp(x) for x <= 0, -infinity and NaN: 2^t with t = x log2(e) rounded once, and what that rounding left out put back to first
// order.  (For x = -infinity that rest is a NaN, which the median takes out; 2^t is 0 then.)  Six instructions instead of
// expf's fourteen; off by 2 units in the last place and |x| 2^-26.  Reciprocals are the hardware's, off by one.  Together, over the norm of each result
// (of torch operations in fp32, sums over tokens in double): gates 3e-8 to 7e-8 (3e-8 to 6e-8), prob_mean 2e-8 to 8e-8 (2.5e-8), fp32 logits' gradient 1.1e-7
// (9e-8); single values up to 4.5e-7 (3.4e-7).
__device__ __forceinline__ float exp_down(float x)
{
    const float t = x * 1.44269504f;
    const float rest = __builtin_amdgcn_fmed3f(fmaf(x, 1.44269504f, -t), -1.0f, 1.0f);
    const float e = __builtin_amdgcn_exp2f(t);
    return fmaf(e, rest * 0.693147181f, e);
}
// Largest of three, NaN left out (fmaxf spends an instruction on each operand to quiet signalling ones).
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// The score of z in the form exp(v) * r, and sigmoid(-z).
struct Score {
    float v, r, down;
};
template <bool SIGMOID> __device__ __forceinline__ Score score_of(float z)
{
    if constexpr (SIGMOID) {
        const float e = exp_down(-fabsf(z)), r = __builtin_amdgcn_rcpf(1.0f + e);
        return Score{z < 0.0f ? z : z >= 0.0f ? 0.0f : z, r, z < 0.0f ? r : e * r};      // (v: NaN stays)
    }
    return Score{z, 1.0f, 1.0f};
}
template <bool SIGMOID> __device__ __forceinline__ float top_of(float z) { return SIGMOID ? fminf(z, 0.0f) : z; }

// exp(v - m) with m finite or the -infinity of an empty set (then v = -infinity too, and the result is 0)
__device__ __forceinline__ float exp_below(float v, float m) { return exp_down(v - (m == -INFINITY ? 0.0f : m)); }

// One token's row as it comes from memory: lane `sub` of LT holds experts (c * LT + sub) * 8 + j; beyond E: -infinity.  Rows
// start anywhere (E need not be a multiple of 8): whole pieces are 16-byte loads all the same, a row's last piece may be shorter.
template <class ZT> __device__ __forceinline__ Raw8<ZT> raw_of(const float (&v)[8])
{
    if constexpr (sizeof(ZT) == 2) return Raw8<ZT>{make_uint4(pack2bf(v[0], v[1]), pack2bf(v[2], v[3]), pack2bf(v[4], v[5]), pack2bf(v[6], v[7]))};
    else return Raw8<ZT>{make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7])};
}
template <class ZT, int LT, int CH>
__device__ __forceinline__ void fetch_row(const ZT *row, int E, int sub, Raw8<ZT> (&raw)[CH])
{
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e0 = (c * LT + sub) * 8;
        if (E % 8 == 0) {                                    // the same for the whole launch: no lane has a piece of its own kind
            raw[c] = fetch8_any(row + min(e0, E - 8));
            if (e0 >= E) raw[c] = raw_of<ZT>({-INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY});
        } else if (e0 + 8 <= E) raw[c] = fetch8_any(row + e0);
        else {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = e0 + j < E ? to_f32(row[e0 + j]) : -INFINITY;
            raw[c] = raw_of<ZT>(v);
        }
    }
}

// The token's selections, dealt to its lanes: selection i * LT + sub, at most NS each: one where the lanes are as many as the
// selections, which is most routers; else up to 8 (k <= E <= 8 LT).  Raw logits through the wave's LDS row.
template <int NS> struct Selection {
    int id[NS];                                              // -1: none, or an id outside [0, E)
    float z[NS];
};

// p = w / sum over the row; the row's largest v and the sum's reciprocal (0 for a row of -infinities) come back too.
template <bool SIGMOID, int LT, int CH>
__device__ __forceinline__ void row_probabilities(const float (&z)[CH][8], float (&p)[CH][8], float &top, float &inv, float (&down)[CH][8])
{
    top = -INFINITY;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 8; j += 2) top = max3(top, top_of<SIGMOID>(z[c][j]), top_of<SIGMOID>(z[c][j + 1]));
    top = group_max<LT>(top);
    float total = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const Score s = score_of<SIGMOID>(z[c][j]);
            p[c][j] = exp_below(s.v, top) * s.r;
            down[c][j] = s.down;
            total += p[c][j];
        }
    total = group_sum<LT>(total);
    inv = total == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(total);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) p[c][j] *= inv;
}

template <int LT, int NS> __device__ __forceinline__ void fetch_ids(const int32_t *ids, int k, int sub, int n_sel, int (&id)[NS])
{
#pragma unroll
    for (int i = 0; i < NS; ++i)
        if (i < n_sel && i * LT + sub < k) id[i] = ids[i * LT + sub];
}
// Puts the row into the wave's LDS and picks the lane's selections from it.  `bad`: an id outside [0, E) in a live token.
template <int LT, int CH, int NS>
__device__ __forceinline__ void pick_selections(const float (&z)[CH][8], float *row, const int (&ids)[NS], int k, int E, int sub, int n_sel, bool live,
                                                Selection<NS> &sel, bool &bad)
{
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        sel.id[i] = -1;
        if (i < n_sel && i * LT + sub < k) {
            if ((unsigned)ids[i] < (unsigned)E) sel.id[i] = ids[i];
            else bad |= live;
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) store8(row + (c * LT + sub) * 8, z[c]);
    wave_lds_fence();
#pragma unroll
    for (int i = 0; i < NS; ++i) sel.z[i] = i < n_sel && sel.id[i] >= 0 ? row[sel.id[i]] : -INFINITY;
    wave_lds_fence();                                        // the row may be overwritten
}

// The part of each selection of this lane: its share of the token's selected (normalised), or its score as it is.
template <bool SIGMOID, int LT, int NS>
__device__ __forceinline__ void selected_parts(const Selection<NS> &sel, int n_sel, bool normalize, float row_top, float row_inv,
                                               float (&part)[NS])
{
    float top = SIGMOID ? 0.0f : row_top, inv = SIGMOID ? 1.0f : row_inv;
    if (normalize) {
        top = -INFINITY;
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (i < n_sel && sel.id[i] >= 0) top = max3(top, top, top_of<SIGMOID>(sel.z[i]));
        top = group_max<LT>(top);
    }
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
        part[i] = 0.0f;
        if (i < n_sel && sel.id[i] >= 0) {
            const Score s = score_of<SIGMOID>(sel.z[i]);
            part[i] = exp_below(s.v, top) * s.r;
            total += part[i];
        }
    }
    if (normalize) {
        total = group_sum<LT>(total);
        inv = total == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(total);
    }
#pragma unroll
    for (int i = 0; i < NS; ++i) part[i] *= inv;
}

// What a block leaves for the micro-batch's sums: per expert sum of p and count, and its number of valid tokens.
struct RouterPartials {
    float *prob;                                             // [n_mb, blocks, E]
    int32_t *count;                                          // [n_mb, blocks, E]
    int32_t *tokens;                                         // [n_mb, blocks]
};
struct RouterSums {
    int32_t *counts, *n_valid;
    float *prob_mean, *loss;
};

// coef E sum_e f_e P_e from dot = sum_e counts_e sum_t p_te
__device__ __forceinline__ float balance_loss(double dot, float coef, int E, int k, double n)
{
    return n > 0.0 ? (float)((double)coef * E * dot / ((double)k * n * n)) : 0.0f;
}

// The block's sum for all of its threads: waves by shuffles, then the waves' sums in ascending order.
__device__ __forceinline__ double block_sum(double v, double *red, int threads)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double total = 0.0;
    for (int w = 0; w < threads / 64; ++w) total += red[w];
    __syncthreads();
    return total;
}

// Whether the next round's loads go out a round ahead: not where the row alone fills the registers.
template <int CH> constexpr bool router_ahead() { return CH <= 2; }

template <int CH> constexpr int router_waves() { return CH == 8 ? 2 : 4; }

// grid (blocks, n_mb); a block takes `per_block` tokens of its micro-batch, with SOLO all of them: it finishes the sums itself.  Bound by
// the vector units and the latency of a round, not by memory: a round is a chain of LDS round trips and exponentials, so the
// next round's row, ids and mask are requested before the present one is worked on, and a selection has a lane of its
// own.  524288 tokens, 128 experts, 8 selected, bf16, 32 micro-batches: 50 us in this kernel (168 MB at 3.4 TB/s), 56 a call; without the loads ahead, with a loop over the
// selections and expf 93.
template <class ZT, bool SIGMOID, int LT, int CH, int NS, bool SOLO>
__global__ void __launch_bounds__(router_waves<CH>() * 64)
router_fwd_kernel(const ZT *__restrict__ logits, const int32_t *__restrict__ ids, const uint8_t *__restrict__ valid, RouterShape sh, int per_block,
                  float *__restrict__ gates, RouterPartials part_out, RouterSums sums, float coef, int32_t *err_flag)
{
    constexpr int NW = router_waves<CH>(), TPW = 64 / LT, ROW = LT * 8 * CH;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    float *stage = reinterpret_cast<float *>(smem);          // [NW][TPW][ROW]
    int32_t *bins = reinterpret_cast<int32_t *>(stage + NW * TPW * ROW);      // [E], then the count of valid tokens
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sub = lane % LT, group = lane / LT;
    const int mb = blockIdx.y, E = sh.E, k = sh.k;
    const int n_sel = (k + LT - 1) / LT;
    const bool normalize = sh.flags & RELIBRA_ROUTER_NORMALIZE;
    const int t_end = min(sh.T, (int)(blockIdx.x + 1) * per_block);
    Raw8<ZT> raw[CH];
    int next_id[NS];
    uint8_t next_valid = 1;
    auto fetch = [&](int t0) __attribute__((always_inline)) {
        const size_t tok = (size_t)mb * sh.T + min(t0 + wave * TPW + group, sh.T - 1);
        fetch_row<ZT, LT, CH>(logits + tok * E, E, sub, raw);
        fetch_ids<LT, NS>(ids + tok * k, k, sub, n_sel, next_id);
        if (valid) next_valid = valid[tok];
    };
    if (router_ahead<CH>() && sh.T > 0) fetch(blockIdx.x * per_block);
    for (int i = tid; i <= E; i += NW * 64) bins[i] = 0;
    __syncthreads();
    float *row = stage + (wave * TPW + group) * ROW;
    float acc[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[c][j] = 0.0f;
    bool bad = false;
    int n_live = 0;
    for (int t0 = blockIdx.x * per_block; t0 < t_end; t0 += NW * TPW) {
        if (!router_ahead<CH>()) fetch(t0);
        const int t = t0 + wave * TPW + group;
        const size_t tok = (size_t)mb * sh.T + min(t, sh.T - 1);
        const bool live = t < t_end && next_valid;
        float z[CH][8], p[CH][8], top, inv, part[NS];
#pragma unroll
        for (int c = 0; c < CH; ++c) unpack8(raw[c], z[c]);
        int id[NS];
#pragma unroll
        for (int i = 0; i < NS; ++i) id[i] = next_id[i];
        if (router_ahead<CH>() && t0 + NW * TPW < t_end) fetch(t0 + NW * TPW);
        Selection<NS> sel;
        pick_selections<LT, CH, NS>(z, row, id, k, E, sub, n_sel, live, sel, bad);
        float down[CH][8];
        row_probabilities<SIGMOID, LT, CH>(z, p, top, inv, down);
        selected_parts<SIGMOID, LT, NS>(sel, n_sel, normalize, top, inv, part);
        if (live) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[c][j] += p[c][j];
            n_live += sub == 0;
        }
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (i < n_sel && i * LT + sub < k) {
                if (live && sel.id[i] >= 0) atomicAdd(&bins[sel.id[i]], 1);
                if (t < t_end) gates[tok * k + i * LT + sub] = live ? sh.scale * part[i] : 0.0f;
            }
    }
    if (n_live) atomicAdd(&bins[E], n_live);
    if (bad) atomicOr(err_flag, RELIBRA_ERR_ID_RANGE);
    __syncthreads();                                         // every wave is done with its rows
    // the wave's token groups, then the waves, in a fixed order
#pragma unroll
    for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int off = LT; off < 64; off <<= 1) acc[c][j] += __shfl_xor(acc[c][j], off);
        if (group == 0) store8(stage + wave * ROW + (c * LT + sub) * 8, acc[c]);
    }
    __syncthreads();
    const size_t at = (size_t)mb * gridDim.x + blockIdx.x;
    const int n = bins[E];
    double dot = 0.0;
    for (int e = tid; e < E; e += NW * 64) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) s += stage[w * ROW + e];
        if (SOLO) {
            sums.prob_mean[at * E + e] = n > 0 ? s * (float)(1.0 / n) : 0.0f;
            sums.counts[at * E + e] = bins[e];
            dot += (double)s * bins[e];
        } else {
            part_out.prob[at * E + e] = s;
            part_out.count[at * E + e] = bins[e];
        }
    }
    if (SOLO) {
        __syncthreads();                                     // the sums have been read
        dot = block_sum(dot, reinterpret_cast<double *>(smem), NW * 64);
        if (tid == 0) {
            sums.n_valid[mb] = n;
            sums.loss[mb] = balance_loss(dot, coef, E, k, n);
        }
    } else if (tid == 0) part_out.tokens[at] = n;
}

// Many blocks' sums to kFoldRows: grid (64 experts, fold, n_mb), a fold's rows dealt to four waves, which join in ascending order.  (One
// block alone took 235 us for the sums of 8192 tokens of 1000 experts; with the fold both launches take 11.)
constexpr int kFoldRows = 16;
__global__ void __launch_bounds__(256)
router_fold_kernel(RouterPartials part, int blocks, int per_fold, int E, float *__restrict__ prob, int32_t *__restrict__ count)
{
    __shared__ float s_prob[4][64];
    __shared__ int32_t s_count[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x * 64 + lane, fold = blockIdx.y, mb = blockIdx.z;
    const size_t base = (size_t)mb * blocks;
    const int end = min(blocks, (fold + 1) * per_fold);
    float p = 0.0f;
    int32_t c = 0;
    if (e < E)
#pragma unroll 8
        for (int b = fold * per_fold + wave; b < end; b += 4) {
            p += part.prob[(base + b) * E + e];
            c += part.count[(base + b) * E + e];
        }
    s_prob[wave][lane] = p;
    s_count[wave][lane] = c;
    __syncthreads();
    if (wave == 0 && e < E) {
        const size_t at = ((size_t)mb * kFoldRows + fold) * E + e;
        prob[at] = ((p + s_prob[1][lane]) + s_prob[2][lane]) + s_prob[3][lane];
        count[at] = c + s_count[1][lane] + s_count[2][lane] + s_count[3][lane];
    }
}

// One block per micro-batch adds up `rows` rows of sums in ascending order and finishes the loss.
constexpr int kFinishThreads = 1024;
__global__ void __launch_bounds__(kFinishThreads)
router_finish_kernel(RouterPartials part, int blocks, int rows, int k, int E, int lanes_e, float coef, RouterSums out)
{
    __shared__ double red[kFinishThreads / 64];
    __shared__ float s_prob[kFinishThreads];
    __shared__ int32_t s_count[kFinishThreads];
    const int tid = threadIdx.x, mb = blockIdx.x;
    const size_t base = (size_t)mb * rows;
    double tokens = 0.0;
    for (int b = tid; b < blocks; b += kFinishThreads) tokens += part.tokens[(size_t)mb * blocks + b];
    double n = 0.0;
    float inv_n = 0.0f;
    const int el = tid % lanes_e, strip = tid / lanes_e, strips = kFinishThreads / lanes_e;
    double dot = 0.0;
    for (int e0 = 0; e0 < E; e0 += lanes_e) {
        const int e = e0 + el;
        float p = 0.0f;
        int32_t c = 0;
        if (e < E)
#pragma unroll 8
            for (int b = strip; b < rows; b += strips) {
                p += part.prob[(base + b) * E + e];
                c += part.count[(base + b) * E + e];
            }
        s_prob[tid] = p;
        s_count[tid] = c;
        if (e0 == 0) {                                        // (behind the first experts' loads: both are on their way together)
            n = block_sum(tokens, red, kFinishThreads);
            inv_n = n > 0.0 ? (float)(1.0 / n) : 0.0f;
        }
        __syncthreads();
        if (strip == 0 && e < E) {
            for (int s = 1; s < strips; ++s) {
                p += s_prob[s * lanes_e + el];
                c += s_count[s * lanes_e + el];
            }
            out.prob_mean[(size_t)mb * E + e] = p * inv_n;
            out.counts[(size_t)mb * E + e] = c;
            dot += (double)p * c;
        }
        __syncthreads();
    }
    dot = block_sum(dot, red, kFinishThreads);
    if (tid == 0) {
        out.n_valid[mb] = (int)n;
        out.loss[mb] = balance_loss(dot, coef, E, k, n);
    }
}

// dL/dz of the gates (upstream dgates) and of the balance loss (upstream dloss).  With c_e = dloss coef E counts_e / (k n^2):
//   du_e = p_e (d_e - sum d p),  d = c, plus scale dgates on the selected where the gates are softmax probabilities as they are;
//   normalised gates: du_{id_s} += part_s (scale dg_s - sum part scale dg);  sigmoid scores as they are: du_{id_s} += part_s scale dg_s;
//   dz = du (softmax), du sigmoid(-z) (sigmoid).
// What falls on the selected experts goes through the token's LDS row, one selection after the other: the same expert twice adds
// up in the order of the selections.  Probabilities are worked out again rather than saved: the row is read anyway.  524288 tokens, 128 experts, 8
// selected, bf16: 76 us, 303 MB at 4.0 TB/s; 32768 tokens of 256 sigmoid scores in fp32 22 us, 69 MB at 3.1 TB/s.
template <class ZT, bool SIGMOID, int LT, int CH, int NS>
__global__ void __launch_bounds__(router_waves<CH>() * 64)
router_bwd_kernel(const ZT *__restrict__ logits, const int32_t *__restrict__ ids, const uint8_t *__restrict__ valid, const float *__restrict__ dgates,
                  const int32_t *__restrict__ counts, const int32_t *__restrict__ n_valid, const float *__restrict__ dloss, RouterShape sh, float coef,
                  int per_block, ZT *__restrict__ dlogits, int32_t *err_flag)
{
    constexpr int NW = router_waves<CH>(), TPW = 64 / LT, ROW = LT * 8 * CH;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sub = lane % LT, group = lane / LT;
    const int mb = blockIdx.y, E = sh.E, k = sh.k;
    const int n_sel = (k + LT - 1) / LT;
    const bool normalize = sh.flags & RELIBRA_ROUTER_NORMALIZE;
    float *row = reinterpret_cast<float *>(smem) + (wave * TPW + group) * ROW;
    const int t_end = min(sh.T, (int)(blockIdx.x + 1) * per_block);
    Raw8<ZT> raw[CH];
    int next_id[NS];
    float next_dg[NS];
    uint8_t next_valid = 1;
    auto fetch = [&](int t0) __attribute__((always_inline)) {
        const size_t tok = (size_t)mb * sh.T + min(t0 + wave * TPW + group, sh.T - 1);
        fetch_row<ZT, LT, CH>(logits + tok * E, E, sub, raw);
        fetch_ids<LT, NS>(ids + tok * k, k, sub, n_sel, next_id);
#pragma unroll
        for (int i = 0; i < NS; ++i) next_dg[i] = dgates && i < n_sel && i * LT + sub < k ? dgates[tok * k + i * LT + sub] : 0.0f;
        if (valid) next_valid = valid[tok];
    };
    if (router_ahead<CH>()) fetch(blockIdx.x * per_block);
    float cost[CH][8];
    {
        const int n = dloss ? n_valid[mb] : 0;
        const float per_count = n > 0 ? (float)((double)dloss[mb] * coef * E / ((double)k * n * n)) : 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int e = (c * LT + sub) * 8 + j;
                cost[c][j] = n > 0 && e < E ? per_count * (float)counts[(size_t)mb * E + e] : 0.0f;
            }
    }
    bool bad = false;
    for (int t0 = blockIdx.x * per_block; t0 < t_end; t0 += NW * TPW) {
        if (!router_ahead<CH>()) fetch(t0);
        const int t = t0 + wave * TPW + group;
        const size_t tok = (size_t)mb * sh.T + min(t, sh.T - 1);
        const bool live = t < t_end && next_valid;
        float z[CH][8], p[CH][8], top, inv, part[NS], add[CH][8], dg[NS];
#pragma unroll
        for (int c = 0; c < CH; ++c) unpack8(raw[c], z[c]);
        int id[NS];
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            id[i] = next_id[i];
            dg[i] = sh.scale * next_dg[i];
        }
        if (router_ahead<CH>() && t0 + NW * TPW < t_end) fetch(t0 + NW * TPW);
        Selection<NS> sel;
        pick_selections<LT, CH, NS>(z, row, id, k, E, sub, n_sel, live, sel, bad);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) add[c][j] = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) store8(row + (c * LT + sub) * 8, add[c]);
        float down[CH][8];
        row_probabilities<SIGMOID, LT, CH>(z, p, top, inv, down);
        selected_parts<SIGMOID, LT, NS>(sel, n_sel, normalize, top, inv, part);
        float mean = 0.0f;
        if (normalize) {
#pragma unroll
            for (int i = 0; i < NS; ++i) mean += part[i] * dg[i];
            mean = group_sum<LT>(mean);
        }
        wave_lds_fence();
#pragma unroll
        for (int i = 0; i < NS; ++i)
            if (i < n_sel) {
                const float v = !normalize && !SIGMOID ? dg[i] : part[i] * (dg[i] - mean);
                const int last = min(LT, k - i * LT);
                for (int q = 0; q < last; ++q)
                    if (sub == q && sel.id[i] >= 0) unsafeAtomicAdd(row + sel.id[i], v);
            }
        wave_lds_fence();
#pragma unroll
        for (int c = 0; c < CH; ++c) load8(row + (c * LT + sub) * 8, add[c]);
        wave_lds_fence();
        // softmax gates as they are: the upstream gradient joins c; otherwise it is a du of its own
        const bool joins = !normalize && !SIGMOID;
        float dot = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) dot += p[c][j] * (joins ? cost[c][j] + add[c][j] : cost[c][j]);
        dot = group_sum<LT>(dot);
        if (t < t_end) {
            ZT *out = dlogits + tok * E;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int e0 = (c * LT + sub) * 8;
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float du = p[c][j] * ((joins ? cost[c][j] + add[c][j] : cost[c][j]) - dot) + (joins ? 0.0f : add[c][j]);
                    if (SIGMOID) du *= down[c][j];
                    v[j] = live ? du : 0.0f;
                }
                if (e0 + 8 <= E) store8_any(out + e0, v);
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (e0 + j < E) from_f32(out + e0 + j, v[j]);
            }
        }
    }
    if (bad) atomicOr(err_flag, RELIBRA_ERR_ID_RANGE);
}

// Blocks per micro-batch: enough that the chip is full over all micro-batches, and no fewer tokens than a block has in flight.
// A micro-batch of few tokens is one block's, which finishes its sums without a second launch.
constexpr int kRouterBlocks = 2048, kSoloRounds = 4;
struct RouterGrid {
    int lanes, chunks, waves, blocks, per_block;
    bool solo;
};
inline RouterGrid router_grid(int n_mb, int T, int E, bool fwd)
{
    RouterGrid g;
    g.lanes = E <= 16 ? 2 : E <= 64 ? 8 : E <= 128 ? 16 : E <= 256 ? 32 : 64;
    g.chunks = 1;
    while (8 * 64 * g.chunks < E) g.chunks *= 2;
    g.waves = g.chunks == 8 ? 2 : 4;
    const int round = g.waves * (64 / g.lanes);              // tokens in flight in a block
    const int rounds = (T + round - 1) / round;
    g.solo = fwd && rounds <= kSoloRounds;
    const int want = g.solo ? 1 : (kRouterBlocks + n_mb - 1) / n_mb;
    // forward: every block leaves E sums that are read again, so up to 4 rounds a block while the blocks fill the units
    const int least = fwd ? (int)std::min(4LL, std::max(1LL, (long long)n_mb * rounds / 256)) : 1;
    const int each = std::max(least, (rounds + want - 1) / want);
    g.per_block = each * round;
    g.blocks = std::max(1, (T + g.per_block - 1) / g.per_block);
    return g;
}
// Rows of sums are folded first where a thread of the one block would read more than 32 of them.
inline bool router_folds(const RouterGrid &g, int E) { return !g.solo && (size_t)g.blocks * E > 32 * kFinishThreads; }
struct RouterWs {
    size_t prob, count, tokens, fold_prob, fold_count, bytes;
};
inline RouterWs router_ws(int n_mb, const RouterGrid &g, int E)
{
    const size_t cells = (size_t)n_mb * g.blocks, folded = router_folds(g, E) ? (size_t)n_mb * kFoldRows * E : 0;
    RouterWs w;
    w.prob = 0;
    w.count = w.prob + round256(cells * E * sizeof(float));
    w.tokens = w.count + round256(cells * E * sizeof(int32_t));
    w.fold_prob = w.tokens + round256(cells * sizeof(int32_t));
    w.fold_count = w.fold_prob + round256(folded * sizeof(float));
    w.bytes = w.fold_count + round256(folded * sizeof(int32_t));
    return w;
}
inline bool router_takes(int n_mb, int T, int k, int E)
{
    return E <= kRouterMaxExperts && k <= 64 && n_mb <= 65535 && (long long)n_mb * T <= 1 << 30 && (long long)T * k <= INT32_MAX;
}
size_t router_ws_bytes(int n_mb, int T, int k, int E)
{
    return k <= E && router_takes(n_mb, T, k, E) ? router_ws(n_mb, router_grid(n_mb, T, E, true), E).bytes : 0;
}

inline int check_router(int n_mb, int T, int k, int E, int flags, const void *logits, const void *ids)
{
    const int known = RELIBRA_ROUTER_SIGMOID | RELIBRA_ROUTER_NORMALIZE | RELIBRA_ROUTER_FP32;
    if (n_mb < 0 || T < 0 || E < 1 || k < 1 || k > E || (flags & ~known)) return RELIBRA_EINVAL;
    if (!router_takes(n_mb, T, k, E)) return RELIBRA_EUNSUPPORTED;
    if ((size_t)n_mb * T > 0 && (!logits || !ids || !aligned16(logits))) return RELIBRA_EINVAL;
    return RELIBRA_OK;
}

// Calls fn(LT, CH, NS) as constants.
template <class Fn> int router_layout(const RouterGrid &g, int k, const Fn &fn)
{
    auto with = [&](auto lt, auto ch) {
        if constexpr (decltype(lt)::value < 64)
            if (k > decltype(lt)::value) return fn(lt, ch, std::integral_constant<int, 8>{});
        return fn(lt, ch, std::integral_constant<int, 1>{});
    };
#define RELIBRA_ROUTER_CASE(l, c) \
    if (g.lanes == l && g.chunks == c) return with(std::integral_constant<int, l>{}, std::integral_constant<int, c>{})
    RELIBRA_ROUTER_CASE(2, 1);
    RELIBRA_ROUTER_CASE(8, 1);
    RELIBRA_ROUTER_CASE(16, 1);
    RELIBRA_ROUTER_CASE(32, 1);
    RELIBRA_ROUTER_CASE(64, 1);
    RELIBRA_ROUTER_CASE(64, 2);
    RELIBRA_ROUTER_CASE(64, 4);
    RELIBRA_ROUTER_CASE(64, 8);
#undef RELIBRA_ROUTER_CASE
    return RELIBRA_EUNSUPPORTED;
}

template <class ZT, bool SIGMOID>
int router_fwd_impl(const ZT *logits, const int32_t *ids, const uint8_t *valid, int n_mb, const RouterShape &sh, const RouterGrid &g,
                    float *gates, const RouterPartials &part, const RouterSums &sums, float coef, int32_t *err_flag, hipStream_t stream)
{
    return router_layout(g, sh.k, [&](auto lt, auto ch, auto ns) {
        constexpr int LT = decltype(lt)::value, CH = decltype(ch)::value, NS = decltype(ns)::value;
        const size_t lds = (size_t)g.waves * 512 * CH * sizeof(float) + (sh.E + 1) * sizeof(int32_t);
        if (g.solo) RELIBRA_LAUNCH(RELIBRA_K_ROUTER_FWD, stream, (router_fwd_kernel<ZT, SIGMOID, LT, CH, NS, true><<<dim3(1, n_mb), g.waves * 64, lds, stream>>>(
            logits, ids, valid, sh, g.per_block, gates, part, sums, coef, err_flag)));
        else RELIBRA_LAUNCH(RELIBRA_K_ROUTER_FWD, stream, (router_fwd_kernel<ZT, SIGMOID, LT, CH, NS, false><<<dim3(g.blocks, n_mb), g.waves * 64, lds, stream>>>(
            logits, ids, valid, sh, g.per_block, gates, part, sums, coef, err_flag)));
        return RELIBRA_OK;
    });
}

template <class ZT, bool SIGMOID>
int router_bwd_impl(const ZT *logits, const int32_t *ids, const uint8_t *valid, const float *dgates, const int32_t *counts, const int32_t *n_valid,
                    const float *dloss, int n_mb, const RouterShape &sh, float coef, const RouterGrid &g, ZT *dlogits, int32_t *err_flag, hipStream_t stream)
{
    return router_layout(g, sh.k, [&](auto lt, auto ch, auto ns) {
        constexpr int LT = decltype(lt)::value, CH = decltype(ch)::value, NS = decltype(ns)::value;
        const size_t lds = (size_t)g.waves * 512 * CH * sizeof(float);
        RELIBRA_LAUNCH(RELIBRA_K_ROUTER_BWD, stream, (router_bwd_kernel<ZT, SIGMOID, LT, CH, NS><<<dim3(g.blocks, n_mb), g.waves * 64, lds, stream>>>(
            logits, ids, valid, dgates, counts, n_valid, dloss, sh, coef, g.per_block, dlogits, err_flag)));
        return RELIBRA_OK;
    });
}

}  // namespace relibra

using namespace relibra;

extern "C" int relibra_router_fwd(const void *logits, const int32_t *ids, const uint8_t *valid, int n_mb, int T, int k, int E, int flags,
                                  float scale, float balance_coef, float *gates, int32_t *counts, int32_t *n_valid, float *prob_mean, float *loss,
                                  void *workspace, size_t workspace_bytes, int32_t *err_flag, relibra_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    const int rc = check_router(n_mb, T, k, E, flags, logits, ids);
    if (rc != RELIBRA_OK) return rc;
    if (n_mb == 0) return RELIBRA_OK;
    if (!counts || !n_valid || !prob_mean || !loss || !err_flag || (T > 0 && !gates)) return RELIBRA_EINVAL;
    const RouterGrid g = router_grid(n_mb, T, E, true);
    const RouterWs at = router_ws(n_mb, g, E);
    if (!workspace || workspace_bytes < at.bytes) return RELIBRA_EWORKSPACE;
    if (!aligned16(workspace)) return RELIBRA_EINVAL;
    char *ws = (char *)workspace;
    RouterPartials part{(float *)(ws + at.prob), (int32_t *)(ws + at.count), (int32_t *)(ws + at.tokens)};
    const RouterShape sh{T, k, E, flags, scale};
    const RouterSums sums{counts, n_valid, prob_mean, loss};
    int rl;
    if (flags & RELIBRA_ROUTER_FP32)
        rl = flags & RELIBRA_ROUTER_SIGMOID ? router_fwd_impl<float, true>((const float *)logits, ids, valid, n_mb, sh, g, gates, part, sums, balance_coef, err_flag, stream)
                                            : router_fwd_impl<float, false>((const float *)logits, ids, valid, n_mb, sh, g, gates, part, sums, balance_coef, err_flag, stream);
    else
        rl = flags & RELIBRA_ROUTER_SIGMOID ? router_fwd_impl<bf16_t, true>((const bf16_t *)logits, ids, valid, n_mb, sh, g, gates, part, sums, balance_coef, err_flag, stream)
                                            : router_fwd_impl<bf16_t, false>((const bf16_t *)logits, ids, valid, n_mb, sh, g, gates, part, sums, balance_coef, err_flag, stream);
    if (rl != RELIBRA_OK) return rl;
    if (!g.solo) {
        int lanes_e = 1;
        while (lanes_e < kFinishThreads && lanes_e < E) lanes_e *= 2;
        int rows = g.blocks;
        if (router_folds(g, E)) {
            float *prob = (float *)(ws + at.fold_prob);
            int32_t *count = (int32_t *)(ws + at.fold_count);
            const int per_fold = (g.blocks + kFoldRows - 1) / kFoldRows;
            RELIBRA_LAUNCH(RELIBRA_K_ROUTER_FINISH, stream, router_fold_kernel<<<dim3((E + 63) / 64, kFoldRows, n_mb), 256, 0, stream>>>(part, g.blocks, per_fold, E, prob, count));
            part.prob = prob;
            part.count = count;
            rows = kFoldRows;
        }
        RELIBRA_LAUNCH(RELIBRA_K_ROUTER_FINISH, stream, router_finish_kernel<<<n_mb, kFinishThreads, 0, stream>>>(part, g.blocks, rows, k, E, lanes_e, balance_coef, sums));
    }
    RELIBRA_HIP_TRY(launch_check());
    return RELIBRA_OK;
}

extern "C" int relibra_router_bwd(const void *logits, const int32_t *ids, const uint8_t *valid, const float *dgates, const int32_t *counts,
                                  const int32_t *n_valid, const float *dloss, int n_mb, int T, int k, int E, int flags, float scale,
                                  float balance_coef, void *dlogits, int32_t *err_flag, relibra_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    const int rc = check_router(n_mb, T, k, E, flags, logits, ids);
    if (rc != RELIBRA_OK) return rc;
    if (n_mb == 0 || T == 0) return RELIBRA_OK;
    if (!dlogits || !aligned16(dlogits) || !err_flag || (dloss && (!counts || !n_valid))) return RELIBRA_EINVAL;
    const RouterGrid g = router_grid(n_mb, T, E, false);
    const RouterShape sh{T, k, E, flags, scale};
    int rl;
    if (flags & RELIBRA_ROUTER_FP32)
        rl = flags & RELIBRA_ROUTER_SIGMOID
                 ? router_bwd_impl<float, true>((const float *)logits, ids, valid, dgates, counts, n_valid, dloss, n_mb, sh, balance_coef, g, (float *)dlogits, err_flag, stream)
                 : router_bwd_impl<float, false>((const float *)logits, ids, valid, dgates, counts, n_valid, dloss, n_mb, sh, balance_coef, g, (float *)dlogits, err_flag, stream);
    else
        rl = flags & RELIBRA_ROUTER_SIGMOID
                 ? router_bwd_impl<bf16_t, true>((const bf16_t *)logits, ids, valid, dgates, counts, n_valid, dloss, n_mb, sh, balance_coef, g, (bf16_t *)dlogits, err_flag, stream)
                 : router_bwd_impl<bf16_t, false>((const bf16_t *)logits, ids, valid, dgates, counts, n_valid, dloss, n_mb, sh, balance_coef, g, (bf16_t *)dlogits, err_flag, stream);
    if (rl != RELIBRA_OK) return rl;
    RELIBRA_HIP_TRY(launch_check());
    return RELIBRA_OK;
}
