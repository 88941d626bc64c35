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
// Layout: LT lanes share a token (the power of two with 8 LT >= E, at most 64), each holds 8 consecutive experts of every CH-th
// run, so a wave has 64 / LT tokens in flight, rows are read in 16-byte pieces, and a lane's experts stay its own
// over all tokens: sum_t p_te accumulates in registers, and only the finished sums of a block are stored.
#include "wave_ops.h"

#include <type_traits>

namespace relibra {

constexpr int kRouterMaxExperts = 4096;
constexpr int kRouterMaxSel = 8;                 // selections a lane handles: k <= 64 and k <= E <= 8 LT CH

struct RouterShape {
    int T, k, E, flags;
    float scale;
};

// Log score of z in the form exp(v) * r.
struct Score {
    float v, r;
};
template <bool SIGMOID> __device__ __forceinline__ Score score_of(float z)
{
    if constexpr (SIGMOID) return Score{z < 0.0f ? z : z >= 0.0f ? 0.0f : z, 1.0f / (1.0f + expf(-fabsf(z)))};      // NaN stays
    else return Score{z, 1.0f};
}

// exp(v - m) with m finite or the -infinity of an empty set (then v = -infinity too, and the result is 0)
__device__ __forceinline__ float exp_below(float v, float m) { return expf(v - (m == -INFINITY ? 0.0f : m)); }

// One token's row in registers: lane `sub` of LT holds experts (c * LT + sub) * 8 + j; beyond E: -infinity.
template <class ZT, int LT, int CH>
__device__ __forceinline__ void load_row(const ZT *row, int E, int sub, bool vec, float (&z)[CH][8])
{
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e0 = (c * LT + sub) * 8;
        if (vec) {                                           // E % 8 == 0: a piece is whole or absent
            if (e0 < E) load8(row + e0, z[c]);
            else
#pragma unroll
                for (int j = 0; j < 8; ++j) z[c][j] = -INFINITY;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) z[c][j] = e0 + j < E ? to_f32(row[e0 + j]) : -INFINITY;
        }
    }
}

// The token's selections, dealt to its lanes: selection i * LT + sub.  Raw logits through the wave's LDS row.
struct Selection {
    int id[kRouterMaxSel];                                   // -1: none, or an id outside [0, E)
    float z[kRouterMaxSel];
};

// p = w / sum over the row; the row's largest v and the sum's reciprocal (0 for a row of -infinities) come back too.
template <bool SIGMOID, int LT, int CH>
__device__ __forceinline__ void row_probabilities(const float (&z)[CH][8], float (&p)[CH][8], float &top, float &inv)
{
    top = -INFINITY;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, SIGMOID ? fminf(z[c][j], 0.0f) : z[c][j]);
    top = group_max<LT>(top);
    float total = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const Score s = score_of<SIGMOID>(z[c][j]);
            p[c][j] = exp_below(s.v, top) * s.r;
            total += p[c][j];
        }
    total = group_sum<LT>(total);
    inv = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) p[c][j] *= inv;
}

// Puts the row into the wave's LDS and picks the lane's selections from it.  `bad`: an id outside [0, E) in a live token.
template <int LT, int CH>
__device__ __forceinline__ void pick_selections(const float (&z)[CH][8], float *row, const int32_t *ids, int k, int E, int sub, int n_sel, bool live,
                                                Selection &sel, bool &bad)
{
#pragma unroll
    for (int i = 0; i < kRouterMaxSel; ++i) {
        sel.id[i] = -1;
        if (i < n_sel && i * LT + sub < k) {
            const int id = ids[i * LT + sub];
            if ((unsigned)id < (unsigned)E) sel.id[i] = id;
            else bad |= live;
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) store8(row + (c * LT + sub) * 8, z[c]);
    wave_lds_fence();
#pragma unroll
    for (int i = 0; i < kRouterMaxSel; ++i) sel.z[i] = i < n_sel && sel.id[i] >= 0 ? row[sel.id[i]] : -INFINITY;
    wave_lds_fence();                                     // the row may be overwritten
}

// The part of each selection of this lane: its share of the token's selected (normalised), or its score as it is.
template <bool SIGMOID, int LT>
__device__ __forceinline__ void selected_parts(const Selection &sel, int n_sel, bool normalize, float row_top, float row_inv,
                                               float (&part)[kRouterMaxSel])
{
    float top = SIGMOID ? 0.0f : row_top, inv = SIGMOID ? 1.0f : row_inv;
    if (normalize) {
        top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kRouterMaxSel; ++i)
            if (i < n_sel && sel.id[i] >= 0) top = fmaxf(top, SIGMOID ? fminf(sel.z[i], 0.0f) : sel.z[i]);
        top = group_max<LT>(top);
    }
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < kRouterMaxSel; ++i) {
        part[i] = 0.0f;
        if (i < n_sel && sel.id[i] >= 0) {
            const Score s = score_of<SIGMOID>(sel.z[i]);
            part[i] = exp_below(s.v, top) * s.r;
            total += part[i];
        }
    }
    if (normalize) {
        total = group_sum<LT>(total);
        inv = total == 0.0f ? 0.0f : 1.0f / total;
    }
#pragma unroll
    for (int i = 0; i < kRouterMaxSel; ++i) part[i] *= inv;
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

__device__ __forceinline__ double block_sum(double v, double *red, int threads)
{
    const int tid = threadIdx.x;
    red[tid] = v;
    __syncthreads();
    for (int n = threads / 2; n > 0; n >>= 1) {
        if (tid < n) red[tid] += red[tid + n];
        __syncthreads();
    }
    const double total = red[0];
    __syncthreads();
    return total;
}

template <int CH> constexpr int router_waves() { return CH == 8 ? 2 : 4; }

// grid (blocks, n_mb); a block takes `per_block` tokens of its micro-batch.
template <class ZT, bool SIGMOID, int LT, int CH>
__global__ void __launch_bounds__(router_waves<CH>() * 64)
router_fwd_kernel(const ZT *__restrict__ logits, const int32_t *__restrict__ ids, const uint8_t *__restrict__ valid, RouterShape sh, int per_block,
                  int vec, float *__restrict__ gates, RouterPartials part_out, int32_t *err_flag)
{
    constexpr int NW = router_waves<CH>(), TPW = 64 / LT, ROW = LT * 8 * CH;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    float *stage = reinterpret_cast<float *>(smem);          // [NW][TPW][ROW]
    int32_t *bins = reinterpret_cast<int32_t *>(stage + NW * TPW * ROW);      // [E], then the count of valid tokens
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sub = lane % LT, group = lane / LT;
    const int mb = blockIdx.y, E = sh.E, k = sh.k;
    const int n_sel = (k + LT - 1) / LT;
    const bool normalize = sh.flags & RELIBRA_ROUTER_NORMALIZE;
    for (int i = tid; i <= E; i += NW * 64) bins[i] = 0;
    __syncthreads();
    float *row = stage + (wave * TPW + group) * ROW;
    float acc[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[c][j] = 0.0f;
    bool bad = false;
    const int t_end = min(sh.T, (int)(blockIdx.x + 1) * per_block);
    for (int t0 = blockIdx.x * per_block; t0 < t_end; t0 += NW * TPW) {
        const int t = t0 + wave * TPW + group;
        const size_t tok = (size_t)mb * sh.T + min(t, sh.T - 1);
        const bool live = t < t_end && (!valid || valid[tok]);
        float z[CH][8], p[CH][8], top, inv, part[kRouterMaxSel];
        load_row<ZT, LT, CH>(logits + tok * E, E, sub, vec, z);
        Selection sel;
        pick_selections<LT, CH>(z, row, ids + tok * k, k, E, sub, n_sel, live, sel, bad);
        row_probabilities<SIGMOID, LT, CH>(z, p, top, inv);
        selected_parts<SIGMOID, LT>(sel, n_sel, normalize, top, inv, part);
        if (live) {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[c][j] += p[c][j];
            if (sub == 0) atomicAdd(&bins[E], 1);
        }
#pragma unroll
        for (int i = 0; i < kRouterMaxSel; ++i)
            if (i < n_sel && i * LT + sub < k) {
                if (live && sel.id[i] >= 0) atomicAdd(&bins[sel.id[i]], 1);
                if (t < t_end) gates[tok * k + i * LT + sub] = live ? sh.scale * part[i] : 0.0f;
            }
    }
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
    for (int e = tid; e < E; e += NW * 64) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) s += stage[w * ROW + e];
        part_out.prob[at * E + e] = s;
        part_out.count[at * E + e] = bins[e];
    }
    if (tid == 0) part_out.tokens[at] = bins[E];
}

// One block per micro-batch adds up the blocks' sums in ascending order and finishes the loss.
__global__ void __launch_bounds__(256)
router_finish_kernel(RouterPartials part, int blocks, int k, int E, int lanes_e, float coef, RouterSums out)
{
    __shared__ double red[256];
    __shared__ float s_prob[256];
    __shared__ int32_t s_count[256];
    const int tid = threadIdx.x, mb = blockIdx.x;
    const size_t base = (size_t)mb * blocks;
    double tokens = 0.0;
    for (int b = tid; b < blocks; b += 256) tokens += part.tokens[base + b];
    const double n = block_sum(tokens, red, 256);
    const float inv_n = n > 0.0 ? (float)(1.0 / n) : 0.0f;
    const int el = tid % lanes_e, strip = tid / lanes_e, strips = 256 / lanes_e;
    double dot = 0.0;
    for (int e0 = 0; e0 < E; e0 += lanes_e) {
        const int e = e0 + el;
        float p = 0.0f;
        int32_t c = 0;
        if (e < E)
            for (int b = strip; b < blocks; b += strips) {
                p += part.prob[(base + b) * E + e];
                c += part.count[(base + b) * E + e];
            }
        s_prob[tid] = p;
        s_count[tid] = c;
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
    dot = block_sum(dot, red, 256);
    if (tid == 0) {
        out.n_valid[mb] = (int)n;
        out.loss[mb] = n > 0.0 ? (float)((double)coef * E * dot / ((double)k * n * n)) : 0.0f;
    }
}

// dL/dz of the gates (upstream dgates) and of the balance loss (upstream dloss).  With c_e = dloss coef E counts_e / (k n^2):
//   du_e = p_e (d_e - sum d p),  d = c, plus scale dgates on the selected where the gates are softmax probabilities as they are;
//   normalised gates: du_{id_s} += part_s (scale dg_s - sum part scale dg);  sigmoid scores as they are: du_{id_s} += part_s scale dg_s;
//   dz = du (softmax), du sigmoid(-z) (sigmoid).
// What falls on the selected experts goes through the token's LDS row, one selection after the other: the same expert twice adds
// up in the order of the selections.
template <class ZT, bool SIGMOID, int LT, int CH>
__global__ void __launch_bounds__(router_waves<CH>() * 64)
router_bwd_kernel(const ZT *__restrict__ logits, const int32_t *__restrict__ ids, const uint8_t *__restrict__ valid, const float *__restrict__ dgates,
                  const int32_t *__restrict__ counts, const int32_t *__restrict__ n_valid, const float *__restrict__ dloss, RouterShape sh, float coef,
                  int per_block, int vec, ZT *__restrict__ dlogits, int32_t *err_flag)
{
    constexpr int NW = router_waves<CH>(), TPW = 64 / LT, ROW = LT * 8 * CH;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sub = lane % LT, group = lane / LT;
    const int mb = blockIdx.y, E = sh.E, k = sh.k;
    const int n_sel = (k + LT - 1) / LT;
    const bool normalize = sh.flags & RELIBRA_ROUTER_NORMALIZE;
    float *row = reinterpret_cast<float *>(smem) + (wave * TPW + group) * ROW;
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
    const int t_end = min(sh.T, (int)(blockIdx.x + 1) * per_block);
    for (int t0 = blockIdx.x * per_block; t0 < t_end; t0 += NW * TPW) {
        const int t = t0 + wave * TPW + group;
        const size_t tok = (size_t)mb * sh.T + min(t, sh.T - 1);
        const bool live = t < t_end && (!valid || valid[tok]);
        float z[CH][8], p[CH][8], top, inv, part[kRouterMaxSel], add[CH][8];
        load_row<ZT, LT, CH>(logits + tok * E, E, sub, vec, z);
        float dg[kRouterMaxSel];
#pragma unroll
        for (int i = 0; i < kRouterMaxSel; ++i) dg[i] = dgates && i < n_sel && i * LT + sub < k ? sh.scale * dgates[tok * k + i * LT + sub] : 0.0f;
        Selection sel;
        pick_selections<LT, CH>(z, row, ids + tok * k, k, E, sub, n_sel, live, sel, bad);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) add[c][j] = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) store8(row + (c * LT + sub) * 8, add[c]);
        row_probabilities<SIGMOID, LT, CH>(z, p, top, inv);
        selected_parts<SIGMOID, LT>(sel, n_sel, normalize, top, inv, part);
        float mean = 0.0f;
        if (normalize) {
#pragma unroll
            for (int i = 0; i < kRouterMaxSel; ++i) mean += part[i] * dg[i];
            mean = group_sum<LT>(mean);
        }
        wave_lds_fence();
#pragma unroll
        for (int i = 0; i < kRouterMaxSel; ++i)
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
                    if (SIGMOID) {
                        const float e = expf(-fabsf(z[c][j]));
                        du *= (z[c][j] < 0.0f ? 1.0f : e) / (1.0f + e);
                    }
                    v[j] = live ? du : 0.0f;
                }
                if (vec) {
                    if (e0 < E) store8(out + e0, v);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (e0 + j < E) from_f32(out + e0 + j, v[j]);
                }
            }
        }
    }
    if (bad) atomicOr(err_flag, RELIBRA_ERR_ID_RANGE);
}

// Blocks per micro-batch: enough that the chip is full over all micro-batches, and no fewer than a wave's worth of tokens each.
constexpr int kRouterBlocks = 1024;
struct RouterGrid {
    int lanes, chunks, waves, blocks, per_block;
};
inline RouterGrid router_grid(int n_mb, int T, int E)
{
    RouterGrid g;
    g.lanes = 1;
    while (g.lanes < 64 && 8 * g.lanes < E) g.lanes *= 2;
    g.chunks = 1;
    while (8 * 64 * g.chunks < E) g.chunks *= 2;
    g.waves = g.chunks == 8 ? 2 : 4;
    const int round = g.waves * (64 / g.lanes);              // tokens in flight in a block
    const int rounds = (T + round - 1) / round;
    const int want = (kRouterBlocks + n_mb - 1) / n_mb;
    const int each = rounds > want ? (rounds + want - 1) / want : 1;
    g.per_block = each * round;
    g.blocks = (T + g.per_block - 1) / g.per_block;
    if (g.blocks < 1) g.blocks = 1;
    return g;
}
size_t router_ws_bytes(int n_mb, int T, int E)
{
    const RouterGrid g = router_grid(n_mb, T, E);
    const size_t cells = (size_t)n_mb * g.blocks;
    return round256(cells * E * sizeof(float)) + round256(cells * E * sizeof(int32_t)) + round256(cells * sizeof(int32_t));
}

inline int check_router(int n_mb, int T, int k, int E, int flags, const void *logits, const void *ids)
{
    const int known = RELIBRA_ROUTER_SIGMOID | RELIBRA_ROUTER_NORMALIZE | RELIBRA_ROUTER_FP32;
    if (n_mb < 0 || T < 0 || E < 1 || k < 1 || k > E || (flags & ~known)) return RELIBRA_EINVAL;
    if (E > kRouterMaxExperts || k > 64 || n_mb > 65535 || (long long)n_mb * T > 1 << 30) return RELIBRA_EUNSUPPORTED;
    if ((size_t)n_mb * T > 0 && (!logits || !ids || !aligned16(logits))) return RELIBRA_EINVAL;
    return RELIBRA_OK;
}

// Calls fn(ZT, SIGMOID, LT, CH) as constants.
template <class ZT, bool SIGMOID, class Fn> int router_layout(const RouterGrid &g, const Fn &fn)
{
#define RELIBRA_ROUTER_CASE(l, c) \
    if (g.lanes == l && g.chunks == c) return fn(std::integral_constant<int, l>{}, std::integral_constant<int, c>{})
    RELIBRA_ROUTER_CASE(1, 1);
    RELIBRA_ROUTER_CASE(2, 1);
    RELIBRA_ROUTER_CASE(4, 1);
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
                    float *gates, const RouterPartials &part, int32_t *err_flag, hipStream_t stream)
{
    const int vec = sh.E % 8 == 0;
    return router_layout<ZT, SIGMOID>(g, [&](auto lt, auto ch) {
        constexpr int LT = decltype(lt)::value, CH = decltype(ch)::value;
        const size_t lds = (size_t)g.waves * 512 * CH * sizeof(float) + (sh.E + 1) * sizeof(int32_t);
        RELIBRA_LAUNCH(RELIBRA_K_ROUTER_FWD, stream, (router_fwd_kernel<ZT, SIGMOID, LT, CH><<<dim3(g.blocks, n_mb), g.waves * 64, lds, stream>>>(
            logits, ids, valid, sh, g.per_block, vec, gates, part, err_flag)));
        return RELIBRA_OK;
    });
}

template <class ZT, bool SIGMOID>
int router_bwd_impl(const ZT *logits, const int32_t *ids, const uint8_t *valid, const float *dgates, const int32_t *counts, const int32_t *n_valid,
                    const float *dloss, int n_mb, const RouterShape &sh, float coef, const RouterGrid &g, ZT *dlogits, int32_t *err_flag, hipStream_t stream)
{
    const int vec = sh.E % 8 == 0;
    return router_layout<ZT, SIGMOID>(g, [&](auto lt, auto ch) {
        constexpr int LT = decltype(lt)::value, CH = decltype(ch)::value;
        const size_t lds = (size_t)g.waves * 512 * CH * sizeof(float);
        RELIBRA_LAUNCH(RELIBRA_K_ROUTER_BWD, stream, (router_bwd_kernel<ZT, SIGMOID, LT, CH><<<dim3(g.blocks, n_mb), g.waves * 64, lds, stream>>>(
            logits, ids, valid, dgates, counts, n_valid, dloss, sh, coef, g.per_block, vec, dlogits, err_flag)));
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
    const RouterGrid g = router_grid(n_mb, T, E);
    if (!workspace || workspace_bytes < router_ws_bytes(n_mb, T, E)) return RELIBRA_EWORKSPACE;
    if (!aligned16(workspace)) return RELIBRA_EINVAL;
    const size_t cells = (size_t)n_mb * g.blocks;
    char *ws = (char *)workspace;
    RouterPartials part;
    part.prob = (float *)ws;
    part.count = (int32_t *)(ws += round256(cells * E * sizeof(float)));
    part.tokens = (int32_t *)(ws + round256(cells * E * sizeof(int32_t)));
    const RouterShape sh{T, k, E, flags, scale};
    int rl;
    if (flags & RELIBRA_ROUTER_FP32)
        rl = flags & RELIBRA_ROUTER_SIGMOID ? router_fwd_impl<float, true>((const float *)logits, ids, valid, n_mb, sh, g, gates, part, err_flag, stream)
                                            : router_fwd_impl<float, false>((const float *)logits, ids, valid, n_mb, sh, g, gates, part, err_flag, stream);
    else
        rl = flags & RELIBRA_ROUTER_SIGMOID ? router_fwd_impl<bf16_t, true>((const bf16_t *)logits, ids, valid, n_mb, sh, g, gates, part, err_flag, stream)
                                            : router_fwd_impl<bf16_t, false>((const bf16_t *)logits, ids, valid, n_mb, sh, g, gates, part, err_flag, stream);
    if (rl != RELIBRA_OK) return rl;
    int lanes_e = 1;
    while (lanes_e < 256 && lanes_e < E) lanes_e *= 2;
    RELIBRA_LAUNCH(RELIBRA_K_ROUTER_FINISH, stream, router_finish_kernel<<<n_mb, 256, 0, stream>>>(
        part, g.blocks, k, E, lanes_e, balance_coef, RouterSums{counts, n_valid, prob_mean, loss}));
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
    const RouterGrid g = router_grid(n_mb, T, E);
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
