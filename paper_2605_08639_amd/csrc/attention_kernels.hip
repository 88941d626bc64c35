// Causal attention of packed sequences with grouped heads, and its gradients.
//
//   z_ij = scale q_i . k_j for the keys j <= i of row i's sequence;  lse_i = ln sum_j exp z_ij;  p_ij = exp(z_ij - lse_i);  o_i = sum_j p_ij v_j
//   D_i = do_i . o_i;  ds_ij = p_ij (do_i . v_j - D_i);  dq_i = scale sum_j ds_ij k_j;  dk_j = scale sum_i ds_ij q_i;  dv_j = sum_i p_ij do_i
//
// The G query heads of a key head are rows of one matrix: packed row r of a sequence is token r / G, head r % G of the group.  A block takes
// 128 packed rows (forward, dq; 32 a wave) or 64 keys (dk, dv; 32 for two waves) of one key head, and walks the other side in tiles of 64 through LDS, two
// tiles in turn, filled by direct loads.  Products are MFMA 32x32x16 with the block's own side on the lanes: a lane then holds one row's
// (one key's) scores in its registers, so that softmax statistics and rescaling are a lane's own work, and the exponentials, rounded
// to bf16, are the next product's operand as they lie: MFMA does not care for the order of the contracted index as long as both sides
// agree, so the other side is read (by transposing LDS reads) in the order that the registers have.  Everything else is fp32.  Gradients
// are computed from the scores again in two kernels, seven products where five would do with atomics: fixed order, the same bits every call.
//
// Roundings: p and ds to bf16 for their products, whose operands have one type (2^-8 of a term at most; the terms' errors are independent and cost the
// sum about what its own rounding does), and D has the error that `out` was rounded with; unless keys are few, see attn_dq_kernel.  dq and dk are 0.0021 to
// 0.0024 off (root mean square over that of the result) for values of a normal distribution, where the last rounding alone costs 0.0017.
//
// Long calls are bound by the matrix units at the clock that the chip's power leaves them, 1.6 to 1.9 GHz of 2.4: one sequence of 16384 tokens, 32
// heads of 4 key heads of 128, forward 2000 us, 1100 TFLOP/s; a loop of the bare products reaches 1900, with one LDS read a product 1710, with the
// softmax's vector work as well 1460, and the library's product of 8192 x 8192 matrices 1390.  Short sequences are bound by blocks' beginnings and ends (a
// micro-batch of 24 sequences, 16384 tokens in all, 64 heads: 450 us, 870 TFLOP/s), small calls by launches and the latency of one block's chain.
#include "gemm_tile.h"
#include "head_rows.h"
#include "wave_ops.h"

#include <algorithm>
#include <type_traits>

namespace relibra {

constexpr int kAttnThreads = 256, kAttnWaves = 4;
// Packed rows of a block and keys of a step.  Blocks of 256 rows and 8 waves: the long sequence 1.3 % faster, the packed micro-batch 3.5 % slower.
constexpr int kRowTile = 128, kKeyTile = 64;
// Gradients of keys: keys of a block and packed rows of a step.  128 keys and 8 waves: the long sequence's launch 1128 -> 1097 us with two tiles in
// LDS, but 2 to 3 % slower in all with three and one barrier a step, and a packed micro-batch has too few long tiles for it.
constexpr int kKeyRows = 64, kRowStep = 64;
constexpr int kAttnMaxDim = 128, kAttnMaxSeq = 8192, kAttnMaxGroup = 64;
constexpr int kSelfSeq = 64;                                 // sequences of calls whose blocks find their units themselves: a lane each
constexpr int kAttnMaxRows = 1 << 26;                        // packed rows of a key head
constexpr int kAttnSlots = 512;                              // blocks that run at once: two a unit
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct AttnShape {
    int T, Hq, Hk, G, d;
    unsigned magic;                                           // for token_of
    float scale;
};
// r / G: for r <= 2^26 + 2^20 and G <= 64 the upper half of r * ceil(2^32 / G): its excess over r / G, below r (G - 1) / (2^32 G) < 1 / G, never reaches
// the next integer.
inline unsigned token_magic(int G) { return G == 1 ? 0u : (unsigned)(((1ull << 32) + G - 1) / G); }
__device__ __forceinline__ int token_of(int r, unsigned magic) { return magic ? (int)__umulhi((unsigned)r, magic) : r; }
// A tensor of heads: element (token, head * d + c) at p[token * ld + head * d + c].
struct HeadsIn {
    const bf16_t *p;
    long long ld;
};
struct HeadsOut {
    bf16_t *p;
    long long ld;
};
// One block's work: rows (or keys) tile * 128 (64) .. of the sequence that starts at row0, over steps from .. to - 1 of the keys (of the packed rows), 64
// each; into slot `slot` of the partial sums, or all there are (-1).  tile < 0: rows row0 .. row0 + len - 1 are padding.
struct alignas(16) AttnUnit {
    int row0, len, tile, from, to, slot, chunks, pad;
    __device__ __forceinline__ void make_uniform()            // (the same in every lane: scalars from here on)
    {
        for (int *x : {&row0, &len, &tile, &from, &to, &slot, &chunks}) *x = __builtin_amdgcn_readfirstlane(*x);
    }
};
struct alignas(16) AttnList {
    int count, joins, pad[6];
};

// At the start of a rare branch: keeps the compiler from turning it into selects that every step pays for.
__device__ __forceinline__ void rare() { asm volatile(""); }

// Nothing moves across: the order of a step's instructions is written out, fragment reads some products ahead of their use and vector
// instructions in the shadow of the products before them (left to itself the compiler reads a fragment, waits for it and multiplies).
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// ---------------------------------------------------------------- LDS tiles: [R][W] of 16-bit values, W = 64 or 128
template <int ND, int R = kKeyTile> struct AttnTile {
    static constexpr int W = ND <= 2 ? 64 : 128;             // ND blocks of 32 columns are used
    static constexpr int ROW = W * 2, SPR = W / 8;            // bytes and 16-byte pieces of a row
    static constexpr int RPB = 64 / SPR;                      // rows of a 1 KiB load
    static constexpr int BYTES = R * ROW, LOADS = BYTES / 1024 / kAttnWaves;
    // Piece c of row r lies at piece c ^ swz(r).  16 consecutive rows at one piece fall into distinct 16-byte bank groups (row reads), and so
    // do 4 consecutive rows at 4 pieces (transposing reads).
    static __device__ __forceinline__ int swz(int r) { return W == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3); }
    // Fragment reads from an LDS address plus the lane's part of it; what is left is an exclusive or and an offset, both constants (a piece's
    // number is bits 4 to 7 of an address, tiles start at multiples of 1 KiB).
    // rows r0 + lane % 32, columns kk * 16 + lane / 32 * 8 .. + 7
    static __device__ __forceinline__ uint32_t row_lane(int lane)
    {
        const int r = lane & 31;
        return r * ROW + (((lane >> 5) ^ swz(r)) << 4);
    }
    static __device__ __forceinline__ bf16x8_t rows(uint32_t at, int r0, int kk)
    {
        return *reinterpret_cast<const __attribute__((address_space(3))) bf16x8_t *>((at ^ (kk << 5)) + r0 * ROW);
    }
    // columns c0 + lane % 32 of rows k0 + 4 (lane / 32) + {0..3, 8..11}: the order in which a lane holds 16 rows of an accumulator
    static __device__ __forceinline__ uint32_t col_lane(int lane)
    {
        const int b = lane >> 4, i = lane & 15, c = (b & 1) * 16 + (i & 3) * 4, k = (b >> 1) * 4 + (i >> 2);
        return k * ROW + (((c >> 3) ^ swz(k)) << 4) + (c >> 2 & 1) * 8;
    }
    static __device__ __forceinline__ bf16x8_t cols(uint32_t at, int c0, int k0)
    {
        typedef __attribute__((address_space(3))) s16x4_t *lds_ptr;
        const s16x4_t l = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)((at ^ (c0 << 1)) + k0 * ROW));
        const s16x4_t h = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)((at ^ (c0 << 1) ^ 32) + (k0 + 8) * ROW));   // (8 rows on: 2 in the swizzle)
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(l, h, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
// A lane's LDS address, opaque to the compiler: kept as one register instead of one for every constant it is combined with.
__device__ __forceinline__ uint32_t lds_at(const char *tile, uint32_t lane_part)
{
    uint32_t at = (uint32_t)(uintptr_t)RELIBRA_LDS(tile) + lane_part;
    asm volatile("" : "+v"(at));
    return at;
}

__device__ __forceinline__ f32x16_t mfma16(bf16x8_t a, bf16x8_t b, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ f32x16_t zero16()
{
    f32x16_t z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    return z;
}

// Registers 8 j .. 8 j + 7 of an accumulator as bf16: the operand of the 16 contracted values they are (rounded once, half a step).
__device__ __forceinline__ bf16x8_t pack_half(const f32x16_t &v, int j)
{
    typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(bf16x8_t, u32x4_t{pack2bf(v[8 * j], v[8 * j + 1]), pack2bf(v[8 * j + 2], v[8 * j + 3]), pack2bf(v[8 * j + 4], v[8 * j + 5]),
                                                pack2bf(v[8 * j + 6], v[8 * j + 7])});
}

// What pack_half's rounding left of them, as bf16: 16 bits together.
__device__ __forceinline__ bf16x8_t pack_rest(const f32x16_t &v, int j)
{
    const bf16x8_t packed = pack_half(v, j);
    f32x16_t rest;
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = v[8 * j + i] - (float)packed[i];
    return pack_half(rest, 0);
}

// A lane's own row as a product's operand: values kk * 16 + lane / 32 * 8 .. + 7 of `row`, zeros from d on (d > 32 (ND - 1)).
template <int ND> __device__ __forceinline__ void load_row(bf16x8_t (&f)[2 * ND], const bf16_t *row, int d, int lane)
{
#pragma unroll
    for (int kk = 0; kk < 2 * ND; ++kk) {
        const int c = kk * 16 + (lane >> 5) * 8;
        const uint4 v = kk < 2 * ND - 2 || c < d ? *reinterpret_cast<const uint4 *>(row + c) : make_uint4(0, 0, 0, 0);
        f[kk] = __builtin_bit_cast(bf16x8_t, v);
    }
}

// An accumulator [d][row on the lanes] to the lanes' rows: the halves of a wave trade 8-byte pieces, so that a lane stores 16 bytes.
template <int ND> __device__ __forceinline__ void store_row(const f32x16_t (&acc)[ND], float by, bf16_t *row, int d, int lane, bool live)
{
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const f32x16_t &v = acc[n];
            uint32_t a0 = pack2bf(v[8 * p] * by, v[8 * p + 1] * by), a1 = pack2bf(v[8 * p + 2] * by, v[8 * p + 3] * by);
            uint32_t b0 = pack2bf(v[8 * p + 4] * by, v[8 * p + 5] * by), b1 = pack2bf(v[8 * p + 6] * by, v[8 * p + 7] * by);
            const auto s0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), s1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
            const int c = n * 32 + p * 16 + (lane >> 5) * 8;
            if (live && (n < ND - 1 || c < d)) *reinterpret_cast<uint4 *>(row + c) = make_uint4(s0[0], s1[0], s0[1], s1[1]);
        }
}

__device__ __forceinline__ float halves_max(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float halves_sum(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}

// This wave's loads have landed, and everyone's: the tile is there, and nobody reads the one before it any more.
__device__ __forceinline__ void tile_barrier()
{
    wait_vm_lgkm0<0>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Loads of tiles of 64 consecutive tokens of one head (keys, values), one after the other.  Rows behind the sequence are its last row again and
// pieces behind d the last piece: nothing outside of the sequence is read, and what lands there is masked or never stored.
template <int ND> struct TokenTiles {
    typedef AttnTile<ND> Tile;
    const bf16_t *at;                                         // (uniform) where this wave's next load starts
    long long ld, step;                                       // elements to the next row, to the wave's next load
    int left, sub, col, row;                                  // rows from the next tile on; the lane's row in a load, its column, its row in the first tile
    uint32_t lane_off;
    __device__ __forceinline__ TokenTiles(const HeadsIn &x, const AttnUnit &u, int head, int d, int wave, int lane) : ld(x.ld), left(u.len - u.from * kKeyTile)
    {
        at = x.p + (long long)(u.row0 + u.from * kKeyTile + wave * Tile::RPB) * ld + (long long)head * d;
        step = (long long)(kAttnWaves * Tile::RPB) * ld;
        sub = lane / Tile::SPR;
        row = wave * Tile::RPB + sub;                         // the swizzle is the same in all of a wave's loads
        col = min((lane % Tile::SPR) ^ Tile::swz(row), d / 8 - 1) * 8;
        lane_off = (uint32_t)(sub * ld + col) * 2u;
    }
    __device__ __forceinline__ void load_next(char *lds, int wave)
    {
        lds += wave * 1024;
        if (left >= kKeyTile) {
#pragma unroll
            for (int i = 0; i < Tile::LOADS; ++i) {
                load_lds16_sv(at, lane_off, lds + i * kAttnWaves * 1024);
                at += step;
            }
        } else {
            rare();
#pragma unroll
            for (int i = 0; i < Tile::LOADS; ++i) {
                const int over = max(row + i * kAttnWaves * Tile::RPB - (left - 1), 0);      // rows behind the last one
                const bf16_t *lane_at = at + (long long)(sub - over) * ld + col;
                load_lds16(lane_at, lds + i * kAttnWaves * 1024);
                at += step;
            }
        }
        left -= kKeyTile;
    }
};

// ---------------------------------------------------------------- schedule
// Lists the blocks' work, heaviest first: one block for the rows, one for the keys.  Sequences are counted (their tiles, and those of the padding behind
// them), every thread finds the sequence of its share of the tiles by bisection, and a counting sort by work puts them in order (within a
// bin in any order: results do not depend on it).  A table that does not ascend within [0, T], or lengths beyond their places: nothing is listed.
// A tile with more than `chunk` steps is several blocks', whose partial sums a second kernel joins.  Rows: a fair share of all steps a block, so that one long
// tile does not outlast the rest, 8 at least (4, 8, 16: 9 sequences in 4999 tokens of 12 heads 37.5, 35.5, 36.9 us; one of 2048 of 8 heads 37.1, 36.8, 35.9,
// backward 79.0, 79.4, 83.4).  Keys: two chunks to each of the blocks that run at once, of 16 steps at least (8, 16, 32: that backward 89.1, 79.4, 79.8 us), or
// one of 4 (4, 8: 5 sequences in 901 tokens of 10 heads backward 33.2, 35.1 us).
// 7 to 11 us of latencies in a row for any table: a launch where rows are shared or sequences are many; else it makes only the keys' list, beside dq.
constexpr int kSchedThreads = 1024, kSchedBins = 1024, kMinRowChunk = 8, kMinKeyChunk = 4, kFullKeyChunk = 16;
// Whether rows are shared at all, from T and Hq alone: where the longest possible tile has so many steps more than the rest of the chip needs meanwhile
// that it pays for the list, partial sums and (forward; the keys have it anyway) the join's launch.  One sequence, not shared / shared, us: 16384 tokens of
// 1 head 254 / 106, 4096 of 8 heads 72 / 65, 8192 of 8 169 / 168, 2048 of 8 37 / 36, 1024 of 32 24 / 33; 8 sequences in 8192 of 4 heads 54 / 47, in 4096 of 8
// 31 / 34, of 12 33 / 44.  Backward one of 2048 of 8 heads 86 / 72, of 16 115 / 115, of 32 168 / 172; 5 in 901 of 10 29 / 35.
constexpr int kShareTiles = 640, kFwdShareSteps = 32, kBwdShareSteps = 24;

template <int THREADS> __device__ __forceinline__ int scan_block(int v, int *sums, int &total)      // inclusive; two barriers
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    v = wave_scan(v);
    if (lane == 63) sums[wave] = v;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) v += sums[w];
        total += sums[w];
    }
    __syncthreads();
    return v;
}

__host__ __device__ inline int tiles_of(long long n, int tile) { return (int)((n + tile - 1) / tile); }

// Steps of 64 keys of tile t: up to the token of its last row.
__device__ __forceinline__ int row_steps(int t, int G, int len, unsigned magic) { return tiles_of(token_of(min(t * kRowTile + kRowTile, len * G) - 1, magic) + 1, kKeyTile); }

struct SchedOut {
    AttnList *head;
    AttnUnit *units, *joins;
    int share;                                                // whether long tiles may be several blocks'
};

template <int THREADS, int SEQ> struct SchedLds {
    unsigned long long steps;
    int before[SEQ + 1], starts[SEQ + 1], lens[SEQ];          // tiles of the sequences before; the tables
    int bins[kSchedBins], sums[THREADS / 64], n_slots, n_joins;
};

// One block of THREADS, at most SEQ sequences.
template <int THREADS, int SEQ>
__device__ __forceinline__ void schedule(bool KEYS, const int32_t *__restrict__ seq_start, const int32_t *__restrict__ seq_len, int n_seq, int T, int G, unsigned magic, int Hk,
                                         const SchedOut &to, int32_t *err_flag, SchedLds<THREADS, SEQ> &lds)
{
    auto &[steps, before, starts, lens, bins, sums, n_slots, n_joins] = lds;
    constexpr int PER = kSchedBins / THREADS;
    const int tid = threadIdx.x;
    if (tid == 0) steps = 0, n_slots = 0, n_joins = 0, before[0] = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) bins[tid * PER + i] = 0;
    __syncthreads();
    bool bad = false;
    int carry = 0;
    for (int s0 = 0; s0 < n_seq; s0 += THREADS) {
        const int s = s0 + tid;
        int tiles = 0;
        if (s < n_seq) {
            const int a = seq_start[s], b = seq_start[s + 1], len = seq_len ? seq_len[s] : b - a;
            starts[s] = a, lens[s] = len;
            if (s == n_seq - 1) starts[n_seq] = b;
            if (a < 0 || b < a || b > T || len < 0 || len > b - a) bad = true;
            else {
                const int own = KEYS ? tiles_of(len, kKeyRows) : tiles_of((long long)len * G, kRowTile);
                tiles = own + tiles_of(b - a - len, kRowTile);
                // keys: the sum of ceil(len G / 64) - G t over the tiles t;  rows: no less than that of (128 t + 127) / (64 G) + 1
                const long long n = own;
                const long long key_steps = n * tiles_of((long long)len * G, kRowStep) - (long long)G * n * (n - 1) / 2, row_steps = (long long)((double)(n * (n + 1)) / G) + 1 + n;
                if (own) atomicAdd(&steps, (unsigned long long)(KEYS ? key_steps : row_steps));
            }
        }
        int total;
        const int incl = scan_block<THREADS>(tiles, sums, total);
        if (s < n_seq) before[s + 1] = carry + incl;
        carry += total;
    }
    if (__syncthreads_or(bad)) {
        if (tid == 0) {
            to.head->count = 0, to.head->joins = 0;
            atomicOr(err_flag, RELIBRA_ERR_SEQ_TABLE);
        }
        return;
    }
    const unsigned long long share = (steps * Hk + kAttnSlots - 1) / kAttnSlots;
    const int longest = KEYS ? tiles_of((long long)T * G, kRowStep) : tiles_of(T, kKeyTile);
    int chunk = longest;
    if (to.share) {
        const unsigned long long want = !KEYS ? max(share, (unsigned long long)kMinRowChunk)
                                        : share < kFullKeyChunk ? max(share, (unsigned long long)kMinKeyChunk) : max((share + 1) / 2, (unsigned long long)kFullKeyChunk);
        chunk = (int)min(want, (unsigned long long)longest);
    }
    const int most = chunk;                                   // the largest work of a unit
    int shift = 0;
    while ((most >> shift) >= kSchedBins) ++shift;
    const int flat = before[n_seq];
    int total = 0;
    // Twice over the tiles: counts of units, then their places.  (One body for both, small as it is: what the kernel waits for is its code's first arrival.)
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
        for (int f = tid; f < flat; f += THREADS) {
            int lo = 0, hi = n_seq;                           // the last sequence with before[s] <= f
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (before[mid] <= f) lo = mid;
                else hi = mid;
            }
            const int a = starts[lo], len = lens[lo], t = f - before[lo], own = KEYS ? tiles_of(len, kKeyRows) : tiles_of((long long)len * G, kRowTile);
            AttnUnit u{a, len, t, 0, 0, -1, 1, 0};
            int first = 0, end = 0, chunks = 1, per = 0;
            if (t >= own) {
                u.row0 = a + len + (t - own) * kRowTile;
                u.len = min(kRowTile, starts[lo + 1] - u.row0);
                u.tile = -1;
            } else {
                first = KEYS ? G * t : 0;
                end = KEYS ? tiles_of((long long)len * G, kRowStep) : row_steps(t, G, len, magic);
                per = end - first;
                if (per > chunk) {
                    chunks = (unsigned)(per + chunk - 1) / (unsigned)chunk;
                    per = (unsigned)(per + chunks - 1) / (unsigned)chunks;
                }
            }
            if (!pass) {
                atomicAdd(&bins[per >> shift], chunks);
                continue;
            }
            if (chunks > 1) {
                u.chunks = chunks;
                u.slot = atomicAdd(&n_slots, chunks);
                to.joins[atomicAdd(&n_joins, 1)] = u;
            }
            int at = atomicAdd(&bins[per >> shift], chunks);
#pragma unroll 1
            for (int c = 0; c < chunks; ++c, ++at) {
                // keys: from the last rows on, so that chunks of one number begin at the same rows
                u.from = KEYS ? max(end - (c + 1) * per, first) : c * per;
                u.to = KEYS ? end - c * per : min(u.from + per, end);
                to.units[at] = u;
                if (chunks > 1) ++u.slot;
            }
        }
        __syncthreads();
        if (!pass) {
            int *mine = bins + kSchedBins - 1 - tid * PER, sum = 0;            // heaviest first
#pragma unroll
            for (int i = 0; i < PER; ++i) sum += mine[-i];
            int at = scan_block<THREADS>(sum, sums, total) - sum;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int n = mine[-i];
                mine[-i] = at;
                at += n;
            }
            __syncthreads();
        }
    }
    if (tid == 0) to.head->count = total, to.head->joins = n_joins;
}

__global__ void __launch_bounds__(kSchedThreads)
attn_sched_kernel(const int32_t *__restrict__ seq_start, const int32_t *__restrict__ seq_len, int n_seq, int T, int G, unsigned magic, int Hk, SchedOut row_out, SchedOut key_out,
                  int32_t *err_flag)
{
    __shared__ SchedLds<kSchedThreads, kAttnMaxSeq> lds;
    const bool keys = blockIdx.x == 1;
    schedule(keys, seq_start, seq_len, n_seq, T, G, magic, Hk, keys ? key_out : row_out, err_flag, lds);
}

// Where a block finds its unit: in the list, or, where no tile is shared and sequences are few, from the tables itself, a sequence a lane, the longest
// tiles of each sequence first.  No scheduling launch (one prompt of 33 tokens, 32 heads: 14.2 -> 10.4 us; 1024 tokens of 64 heads 34.7 -> 29.1), and the
// blocks of a sequence, which read the same keys, run together (60 sequences in 16384 tokens of 32 heads with keys of their own 182 -> 174 us, backward 610 ->
// 589); without an order among sequences the last rounds of blocks are less even (24 in 8192 of 128 heads 326 -> 329).
struct UnitSource {
    const AttnList *list;                                     // NULL: from the tables
    const AttnUnit *units;
    const int32_t *seq_start, *seq_len;
    int n_seq, T;
    int32_t *err_flag;
    template <bool KEYS> __device__ __forceinline__ bool find(int at, int G, unsigned magic, AttnUnit &u) const
    {
        if (list) {
            if (at >= list->count) return false;
            u = units[at];
            return true;
        }
        const int lane = threadIdx.x & 63, s = min(lane, n_seq - 1);
        const int a = seq_start[s], b = seq_start[s + 1], len = seq_len ? seq_len[s] : b - a;
        if (__any(a < 0 || b < a || b > T || len < 0 || len > b - a)) {
            if (at == 0 && threadIdx.x == 0) atomicOr(err_flag, RELIBRA_ERR_SEQ_TABLE);
            return false;
        }
        const int own = KEYS ? tiles_of(len, kKeyRows) : tiles_of((long long)len * G, kRowTile), tiles = lane < n_seq ? own + tiles_of(b - a - len, kRowTile) : 0;
        const int upto = wave_scan(tiles);
        const unsigned long long behind = __ballot(upto > at);
        if (!behind) return false;
        const int mine = __builtin_ctzll(behind);
        auto of = [&](int v) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(v, mine); };
        const int t = at - of(upto - tiles), row0 = of(a), end = of(b), n = of(len), n_own = of(own);
        u.slot = -1, u.chunks = 1, u.from = 0, u.to = 0, u.row0 = row0, u.len = n;
        if (t >= n_own) u.row0 = row0 + n + (t - n_own) * kRowTile, u.len = min(kRowTile, end - u.row0), u.tile = -1;
        else if (KEYS) u.tile = t, u.from = G * t, u.to = tiles_of((long long)n * G, kRowStep);
        else u.tile = n_own - 1 - t, u.to = row_steps(u.tile, G, n, magic);       // the longest first here, too
        return true;
    }
};

// Partial sums of a unit: registers as they lie, 16 bytes a lane, so that stores are whole lines; and in the forward pass two values a row, behind them.
template <int ND> struct Part {
    static constexpr size_t FLOATS = (size_t)kAttnWaves * ND * 16 * 64;
    static __device__ __forceinline__ float *at(float *parts, int slot, int wave, int n, int quad, int lane)
    {
        return parts + (size_t)slot * FLOATS + (((wave * ND + n) * 4 + quad) * 64 + lane) * 4;
    }
    static __device__ __forceinline__ void put(float *parts, int slot, int wave, int lane, const f32x16_t (&acc)[ND])
    {
#pragma unroll
        for (int n = 0; n < ND; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4 *>(at(parts, slot, wave, n, g, lane)) = make_float4(acc[n][4 * g], acc[n][4 * g + 1], acc[n][4 * g + 2], acc[n][4 * g + 3]);
    }
    // acc += by * the part's columns 32 n ..
    static __device__ __forceinline__ void add(float *parts, int slot, int wave, int lane, int n, float by, f32x16_t &acc)
    {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float4 v = *reinterpret_cast<const float4 *>(at(parts, slot, wave, n, g, lane));
            acc[4 * g] += by * v.x, acc[4 * g + 1] += by * v.y, acc[4 * g + 2] += by * v.z, acc[4 * g + 3] += by * v.w;
        }
    }
};

// ---------------------------------------------------------------- forward
// One pass over the keys with a running maximum and sum.  A step of a wave is 32 products of 32x32x16 (d = 128), 32 exponentials a lane and 48 LDS reads, 32 of
// them transposing ones of 8 bytes a lane; the order below keeps the first two side by side (ragged batch 46.9 -> 38.5 us; long calls spend the 14 % of cycles on
// a lower clock: 2100 -> 2083).
template <int ND>
__global__ void __launch_bounds__(kAttnThreads, 2)
attn_fwd_kernel(AttnShape sh, HeadsIn q, HeadsIn k, HeadsIn v, UnitSource source, HeadsOut out, float *__restrict__ lse,
                float *__restrict__ parts, float2 *__restrict__ sums)
{
    typedef AttnTile<ND> Tile;
    __shared__ __attribute__((aligned(1024))) char lds[4 * Tile::BYTES];      // keys and values, two tiles each
    const int at = blockIdx.x / sh.Hk, hk = blockIdx.x - at * sh.Hk;
    AttnUnit u;
    if (!source.find<false>(at, sh.G, sh.magic, u)) return;
    u.make_uniform();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), G = sh.G, d = sh.d;
    if (u.tile < 0) {                                         // padding: zeros
        const int pieces = G * d / 8;
        for (int i = threadIdx.x; i < u.len * pieces; i += kAttnThreads)
            *reinterpret_cast<uint4 *>(out.p + (u.row0 + i / pieces) * out.ld + (long long)hk * G * d + i % pieces * 8) = make_uint4(0, 0, 0, 0);
        for (int i = threadIdx.x; i < u.len * G; i += kAttnThreads) lse[(long long)(u.row0 + i / G) * sh.Hq + hk * G + i % G] = 0.0f;
        return;
    }
    const int rows = u.len * G, first = u.tile * kRowTile + wave * 32;         // (this wave's first packed row)
    const int r = min(first + (lane & 31), rows - 1), tok = token_of(r, sh.magic), head = hk * G + r - tok * G;
    const int wave_lo = token_of(min(first, rows - 1), sh.magic), wave_hi = token_of(min(first + 31, rows - 1), sh.magic);

    const uint32_t row_lane = Tile::row_lane(lane), col_lane = Tile::col_lane(lane);
    TokenTiles<ND> kt(k, u, hk, d, wave, lane), vt(v, u, hk, d, wave, lane);
    kt.load_next(lds + (u.from & 1) * Tile::BYTES, wave);
    bf16x8_t qf[2 * ND];
    load_row<ND>(qf, q.p + (long long)(u.row0 + tok) * q.ld + head * d, d, lane);
    vt.load_next(lds + (2 + (u.from & 1)) * Tile::BYTES, wave);

    const float c = sh.scale * kLog2e;
    float m = -INFINITY, l = 0.0f;
    f32x16_t o[ND], s[2];
#pragma unroll
    for (int n = 0; n < ND; ++n) o[n] = zero16();
    // A step's scores are computed beside the exponentials of the step before: matrix and vector instructions of one wave, independent of each other.
    // Keys are therefore one step ahead of values.
    auto step_in = [&](int t) __attribute__((always_inline)) {       // keys of step t + 1 and values of step t are there; the next ones go out
        tile_barrier();
        if (t + 2 < u.to) kt.load_next(lds + (t & 1) * Tile::BYTES, wave);
        if (t + 1 < u.to) vt.load_next(lds + (2 + (~t & 1)) * Tile::BYTES, wave);
    };
    // scores of step t, and beside(kk) vector work for each of the 2 ND pairs of products
    auto scores = [&](int t, f32x16_t (&to)[2], auto beside) __attribute__((always_inline)) {
        const uint32_t key_rows = lds_at(lds + (t & 1) * Tile::BYTES, row_lane);
        constexpr int N = 2 * ND, AHEAD = 2;
        bf16x8_t f[N][2];
        auto fetch = [&](int kk) __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < 2; ++b) f[kk][b] = Tile::rows(key_rows, b * 32, kk);
        };
        to[0] = to[1] = zero16();
#pragma unroll
        for (int kk = 0; kk < AHEAD; ++kk) fetch(kk);
#pragma unroll
        for (int kk = 0; kk < N; ++kk) {
            if (kk + AHEAD < N) fetch(kk + AHEAD);
            in_order();
#pragma unroll
            for (int b = 0; b < 2; ++b) to[b] = mfma16(f[kk][b], qf[kk], to[b]);
            beside(kk);
            in_order();
        }
    };
    auto mask = [&](int t, f32x16_t (&x)[2]) __attribute__((always_inline)) {
        if (t * kKeyTile + kKeyTile - 1 > wave_lo) {          // keys behind a row's token
            rare();
            const int seen = tok - t * kKeyTile - (lane >> 5) * 4;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (b * 32 + (i >> 2) * 8 + (i & 3) > seen) x[b][i] = -INFINITY;
        }
    };
    // The reference value of the exponentials follows the maximum only where it has risen by more than 2^8: the sums then stay below
    // 2^8 times their count, and most steps need no rescaling.
    auto follow = [&](float top) __attribute__((always_inline)) {
        if (__any((top - m) * c > 8.0f)) {
            rare();
            const float m_new = fmaxf(m, top), by = __builtin_amdgcn_exp2f((m - m_new) * c);
            m = m_new;
            l *= by;
#pragma unroll
            for (int n = 0; n < ND; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[n][i] *= by;
        }
    };
    // exponentials number from .. to - 1 of a lane's 32, their sum, and every eight of them as an operand
    float sum[4];
    auto exponentials = [&](f32x16_t (&x)[2], bf16x8_t (&p)[4], float mc, int from, int to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = from; i < to; ++i) {
            float &e = reinterpret_cast<float(&)[32]>(x)[i];
            e = __builtin_amdgcn_exp2f(fmaf(e, c, -mc));
            sum[i & 3] += e;
            if ((i & 7) == 7) {
                p[i >> 3] = pack_half(x[i >> 4], i >> 3 & 1);
                asm volatile("" : "+v"(p[i >> 3]));           // (here, not put off until the next products)
            }
        }
        asm volatile("" : "+v"(sum[0]), "+v"(sum[1]), "+v"(sum[2]), "+v"(sum[3]));
    };
    auto weigh = [&](int t, const bf16x8_t (&p)[4], auto beside) __attribute__((always_inline)) {
        const uint32_t val_cols = lds_at(lds + (2 + (t & 1)) * Tile::BYTES, col_lane);
        constexpr int N = 4 * ND, AHEAD = 3;
        bf16x8_t f[N];
        auto fetch = [&](int i) __attribute__((always_inline)) { f[i] = Tile::cols(val_cols, i % ND * 32, i / ND * 16); };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) fetch(i);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (i + AHEAD < N) fetch(i + AHEAD);
            in_order();
            o[i % ND] = mfma16(f[i], p[i / ND], o[i % ND]);
            beside(i);
            in_order();
        }
    };
    auto nothing = [](int) {};

    auto step = [&](int t, f32x16_t (&now)[2], f32x16_t (&next)[2]) __attribute__((always_inline)) {
        step_in(t);
        bf16x8_t p[4];
        const float mc = m * c;
        sum[0] = l, sum[1] = sum[2] = sum[3] = 0.0f;
        scores(t + 1, next, [&](int kk) __attribute__((always_inline)) { exponentials(now, p, mc, kk * 16 / ND, (kk + 1) * 16 / ND); });
        l = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        mask(t + 1, next);
        float top = next[0][0];
        weigh(t, p, [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int e = i * 8 / ND; e < (i + 1) * 8 / ND; ++e) top = fmaxf(top, next[e >> 4][e & 15]);
        });
        follow(halves_max(top));
    };
    tile_barrier();                                           // the first keys and values
    if (u.from + 1 < u.to) kt.load_next(lds + (~u.from & 1) * Tile::BYTES, wave);
    const int own = min(wave_hi / kKeyTile, u.to - 1);        // this wave's last step; the block's other waves may have more
    int t = u.from;
    if (t <= own) {
        scores(t, s, nothing);
        mask(t, s);
        float top = s[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) top = fmaxf(top, s[i >> 4][i & 15]);
        follow(halves_max(top));
        f32x16_t other[2];
        for (; t + 1 < own; t += 2) {
            step(t, s, other);
            step(t + 1, other, s);
        }
        if (t < own) {
            step(t, s, other);
            s[0] = other[0], s[1] = other[1];
        }
        step_in(own);
        bf16x8_t p[4];
        sum[0] = l, sum[1] = sum[2] = sum[3] = 0.0f;
        exponentials(s, p, m * c, 0, 32);
        l = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        weigh(own, p, nothing);
        t = own + 1;
    }
    for (; t < u.to; ++t) step_in(t);
    l = halves_sum(l);
    if (u.slot >= 0) {
        Part<ND>::put(parts, u.slot * sh.Hk + hk, wave, lane, o);
        if (lane < 32) sums[(u.slot * sh.Hk + hk) * kRowTile + wave * 32 + lane] = make_float2(m * c, l);
        return;
    }
    const bool live = first + (lane & 31) < rows;
    store_row<ND>(o, 1.0f / l, out.p + (long long)(u.row0 + tok) * out.ld + head * d, d, lane, live);
    if (live && lane < 32) lse[(long long)(u.row0 + tok) * sh.Hq + head] = (m * c + __builtin_amdgcn_logf(l)) * kLn2;
}

// Joins the rows whose keys several blocks shared: their sums at one reference value, in ascending order.  A part without keys has the sum 0 at -infinity.
// 32 columns a block and four parts' loads together: reading one part after the other took longer than the attention (11 us for 4999 rows of 12 heads).
template <int ND>
__global__ void __launch_bounds__(kAttnThreads)
attn_join_out_kernel(AttnShape sh, const AttnList *__restrict__ list, const AttnUnit *__restrict__ joins, float *__restrict__ parts, const float2 *__restrict__ sums, HeadsOut out,
                     float *__restrict__ lse)
{
    const int n = blockIdx.x % ND, tile = blockIdx.x / ND, at = tile / sh.Hk, hk = tile - at * sh.Hk;
    if (at >= list->joins) return;
    const AttnUnit u = joins[at];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rows = u.len * sh.G, first = u.tile * kRowTile + wave * 32;
    const int r = min(first + (lane & 31), rows - 1), tok = token_of(r, sh.magic), head = hk * sh.G + r - tok * sh.G;
    const float2 *mine = sums + (u.slot * sh.Hk + hk) * kRowTile + wave * 32 + (lane & 31);
    float top = -INFINITY, l = 0.0f;
#pragma unroll 4
    for (int c = 0; c < u.chunks; ++c) top = fmaxf(top, mine[c * sh.Hk * kRowTile].x);
    f32x16_t o[1] = {zero16()};
#pragma unroll 4
    for (int c = 0; c < u.chunks; ++c) {
        const float2 part = mine[c * sh.Hk * kRowTile];
        const float by = __builtin_amdgcn_exp2f(part.x - top);
        l += by * part.y;
        Part<ND>::add(parts, (u.slot + c) * sh.Hk + hk, wave, lane, n, by, o[0]);
    }
    const bool live = first + (lane & 31) < rows;
    store_row<1>(o, 1.0f / l, out.p + (long long)(u.row0 + tok) * out.ld + head * sh.d + n * 32, sh.d - n * 32, lane, live);
    if (n == 0 && live && lane < 32) lse[(long long)(u.row0 + tok) * sh.Hq + head] = (top + __builtin_amdgcn_logf(l)) * kLn2;
}

// s = rows of x0 times the lanes' f0, dp = rows of x1 times f1 plus what `start` has (-D: a subtraction a value less); fragments are read two products ahead.
template <int ND>
__device__ __forceinline__ void score_pair(uint32_t x0, uint32_t x1, const bf16x8_t (&f0)[2 * ND], const bf16x8_t (&f1)[2 * ND], const f32x16_t &start, f32x16_t &s, f32x16_t &dp)
{
    typedef AttnTile<ND> Tile;                                // (rows lie alike in tiles of any height)
    constexpr int N = 2 * ND, AHEAD = 2;
    bf16x8_t a[N][2];
    auto fetch = [&](int kk) __attribute__((always_inline)) { a[kk][0] = Tile::rows(x0, 0, kk), a[kk][1] = Tile::rows(x1, 0, kk); };
    s = zero16();
#pragma unroll
    for (int kk = 0; kk < AHEAD; ++kk) fetch(kk);
#pragma unroll
    for (int kk = 0; kk < N; ++kk) {
        if (kk + AHEAD < N) fetch(kk + AHEAD);
        in_order();
        s = mfma16(a[kk][0], f0[kk], s);
        dp = mfma16(a[kk][1], f1[kk], kk ? dp : start);
        in_order();
    }
}

// ---------------------------------------------------------------- backward: queries
// dq of 128 packed rows, and for the other kernel each row's lse in powers of two and -D.  Three products a step; scores are not kept, p comes from lse.
// One sequence of 8192 tokens, 32 heads with keys of their own: 700 us, 1180 TFLOP/s of its three products.
// Where few keys make up `out`, its rounding puts an error into D that is as large as ds, and ds' own roundings are too few to average out.  Tiles that see two
// steps' keys therefore put D right first by the sum of ds, which is zero with the right one, and multiply what ds' rounding left, too; the other kernel
// does that for the same rows.  For values of a normal distribution it takes dq and dk from 0.0035 to 0.0021 off in sequences of a few tokens, 0.0029 to 0.0022
// in those of 180, 0.0026 to 0.0024 in one of 8192; the packed micro-batch 1503 -> 1522 us, the long sequence 1728 -> 1742.
constexpr int kExactSteps = 2;                               // both steps' tiles are in LDS at once: nothing is loaded twice
template <int ND>
__global__ void __launch_bounds__(kAttnThreads, 2)
attn_dq_kernel(AttnShape sh, HeadsIn q, HeadsIn k, HeadsIn v, HeadsIn out, HeadsIn dout, const float *__restrict__ lse, UnitSource source,
               int with_keys, SchedOut key_out, HeadsOut dq, float *__restrict__ lse2, float *__restrict__ minus_delta, float *__restrict__ parts)
{
    typedef AttnTile<ND> Tile;
    __shared__ __attribute__((aligned(1024))) char lds[4 * Tile::BYTES];
    if (blockIdx.x < with_keys) {                             // the first block makes the keys' list meanwhile
        auto &work = *reinterpret_cast<SchedLds<kAttnThreads, kSelfSeq> *>(lds);
        static_assert(sizeof(work) <= sizeof(lds));
        schedule(true, source.seq_start, source.seq_len, source.n_seq, sh.T, sh.G, sh.magic, sh.Hk, key_out, source.err_flag, work);
        return;
    }
    const int block = blockIdx.x - with_keys, at = block / sh.Hk, hk = block - at * sh.Hk;
    AttnUnit u;
    if (!source.find<false>(at, sh.G, sh.magic, u)) return;
    u.make_uniform();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), G = sh.G, d = sh.d;
    if (u.tile < 0) {
        const int pieces = G * d / 8;
        for (int i = threadIdx.x; i < u.len * pieces; i += kAttnThreads)
            *reinterpret_cast<uint4 *>(dq.p + (u.row0 + i / pieces) * dq.ld + (long long)hk * G * d + i % pieces * 8) = make_uint4(0, 0, 0, 0);
        return;
    }
    const int rows = u.len * G, first = u.tile * kRowTile + wave * 32;
    const int r = min(first + (lane & 31), rows - 1), tok = token_of(r, sh.magic), head = hk * G + r - tok * G;
    const int wave_lo = token_of(min(first, rows - 1), sh.magic), wave_hi = token_of(min(first + 31, rows - 1), sh.magic);
    const bool live = first + (lane & 31) < rows;

    const uint32_t row_lane = Tile::row_lane(lane), col_lane = Tile::col_lane(lane);
    TokenTiles<ND> kt(k, u, hk, d, wave, lane), vt(v, u, hk, d, wave, lane);
    kt.load_next(lds + (u.from & 1) * Tile::BYTES, wave);
    vt.load_next(lds + (2 + (u.from & 1)) * Tile::BYTES, wave);
    bf16x8_t qf[2 * ND], df[2 * ND];
    load_row<ND>(qf, q.p + (long long)(u.row0 + tok) * q.ld + head * d, d, lane);
    load_row<ND>(df, dout.p + (long long)(u.row0 + tok) * dout.ld + head * d, d, lane);
    float D = 0.0f;
    {
        bf16x8_t of[2 * ND];
        load_row<ND>(of, out.p + (long long)(u.row0 + tok) * out.ld + head * d, d, lane);
#pragma unroll
        for (int kk = 0; kk < 2 * ND; ++kk)
#pragma unroll
            for (int i = 0; i < 8; ++i) D = fmaf((float)of[kk][i], (float)df[kk][i], D);
        D = halves_sum(D);
    }
    const long long place = (long long)(u.row0 + tok) * sh.Hq + head;
    const float l2 = lse[place] * kLog2e, c = sh.scale * kLog2e;
    // a sequence's first row has one key and a constant softmax: its scores have no gradient (what rounding would leave is not stored)
    auto mask = [&](int t, int b, f32x16_t &s) __attribute__((always_inline)) {
        if (t * kKeyTile + kKeyTile - 1 > wave_lo) {
            rare();
            const int seen = (tok > 0 ? tok : -1) - t * kKeyTile - (lane >> 5) * 4;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (b * 32 + (i >> 2) * 8 + (i & 3) > seen) s[i] = -INFINITY;
        }
    };
    auto tiles_in = [&](int t) __attribute__((always_inline)) {       // step t's are there; the next ones go out
        tile_barrier();
        if (t + 1 < u.to) {
            kt.load_next(lds + (~t & 1) * Tile::BYTES, wave);
            vt.load_next(lds + (2 + (~t & 1)) * Tile::BYTES, wave);
        }
    };
    f32x16_t minus_D;
#pragma unroll
    for (int i = 0; i < 16; ++i) minus_D[i] = -D;
    // Few keys: first the sum of ds, which is what D lacks.  Both steps' tiles then stay where they are.
    const bool exact = u.to <= kExactSteps;
    if (exact) {
        float more = 0.0f;
#pragma unroll 1
        for (int t = 0; t < u.to; ++t) {
            tiles_in(t);
            if (t * kKeyTile > wave_hi) continue;
            const uint32_t key_rows = lds_at(lds + (t & 1) * Tile::BYTES, row_lane), val_rows = lds_at(lds + (2 + (t & 1)) * Tile::BYTES, row_lane);
#pragma unroll 1
            for (int b = 0; b < 2; ++b) {
                f32x16_t s, dp;
                score_pair<ND>(key_rows + b * 32 * Tile::ROW, val_rows + b * 32 * Tile::ROW, qf, df, minus_D, s, dp);
                mask(t, b, s);
#pragma unroll
                for (int i = 0; i < 16; ++i) more = fmaf(__builtin_amdgcn_exp2f(fmaf(s[i], c, -l2)), dp[i], more);
            }
        }
        D += halves_sum(more);
#pragma unroll
        for (int i = 0; i < 16; ++i) minus_D[i] = -D;
    }
    if (live && lane < 32 && u.from == 0) lse2[place] = l2, minus_delta[place] = -D;

    f32x16_t acc[ND];
#pragma unroll
    for (int n = 0; n < ND; ++n) acc[n] = zero16();
    for (int t = u.from; t < u.to; ++t) {
        if (!exact) tiles_in(t);
        if (t * kKeyTile > wave_hi) continue;
        const char *keys = lds + (t & 1) * Tile::BYTES, *vals = lds + (2 + (t & 1)) * Tile::BYTES;
        const uint32_t key_rows = lds_at(keys, row_lane), val_rows = lds_at(vals, row_lane), key_cols = lds_at(keys, col_lane);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            f32x16_t s, dp;
            score_pair<ND>(key_rows + b * 32 * Tile::ROW, val_rows + b * 32 * Tile::ROW, qf, df, minus_D, s, dp);
            mask(t, b, s);
            bf16x8_t f[ND];
            auto fetch = [&](int j) __attribute__((always_inline)) {
#pragma unroll
                for (int n = 0; n < ND; ++n) f[n] = Tile::cols(key_cols, n * 32, b * 32 + j * 16);
            };
            auto gradients = [&](int j) __attribute__((always_inline)) {
#pragma unroll
                for (int i = 8 * j; i < 8 * j + 8; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -l2)) * dp[i];
                return pack_half(s, j);
            };
            auto add = [&](const bf16x8_t &x) __attribute__((always_inline)) {
#pragma unroll
                for (int n = 0; n < ND; ++n) acc[n] = mfma16(f[n], x, acc[n]);
            };
            fetch(0);
            const bf16x8_t ds0 = gradients(0);
            in_order();
            add(ds0);
            const bf16x8_t ds1 = gradients(1);
            in_order();
            fetch(1);
            add(ds1);
            if (exact) {                                      // what the rounding of ds left
                rare();
                add(pack_rest(s, 1));
                fetch(0);
                add(pack_rest(s, 0));
            }
        }
    }
    if (u.slot >= 0) {
        Part<ND>::put(parts, u.slot * sh.Hk + hk, wave, lane, acc);
        return;
    }
    store_row<ND>(acc, sh.scale, dq.p + (long long)(u.row0 + tok) * dq.ld + head * d, d, lane, live);
}

// ---------------------------------------------------------------- backward: keys and values
// dk and dv of 64 keys over some of the packed rows behind the first of them.  Two waves share 32 keys: each works out p and ds for 32 of a step's
// 64 rows, hands the other the half that it needs, and adds up one of the two gradients over all 64 rows.  A wave for itself would hold both sums,
// 128 registers beside the operands' 64 and the scores' 32, and leave no room for a second wave on its SIMD (the long sequence 2260 -> 1190 us).
// Four products a step, two barriers: 1100 us, 1000 TFLOP/s for 8192 tokens of 32 heads with keys of their own; without any loads it took 930.  A step of a unit's two
// blocks takes 4200 cycles, in packed micro-batches, too; 2050 are products, and no other unit is busy for as long.  A quarter of a wave's time is waits and barriers.
template <int ND>
__global__ void __launch_bounds__(kAttnThreads, 2)
attn_dkv_kernel(AttnShape sh, HeadsIn q, HeadsIn k, HeadsIn v, HeadsIn dout, const float *__restrict__ lse2, const float *__restrict__ minus_delta,
                UnitSource source, HeadsOut dk, HeadsOut dv, float *__restrict__ parts)
{
    typedef AttnTile<ND, kRowStep> Tile;
    constexpr int STATS = 4 * Tile::BYTES, TRADE = STATS + 4 * kRowStep * 4, PAIR = 6 * 1024;
    // queries and their upstream, two steps each; the rows' lse and -D, two steps each; what the waves of a pair hand each other: p, or ds and its rest
    __shared__ __attribute__((aligned(1024))) char lds[TRADE + kAttnWaves / 2 * PAIR];
    const int at = blockIdx.x / sh.Hk, hk = blockIdx.x - at * sh.Hk;
    AttnUnit u;
    if (!source.find<true>(at, sh.G, sh.magic, u)) return;
    u.make_uniform();
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), role = wave & 1, G = sh.G, d = sh.d;   // role 0: dv, 1: dk
    if (u.tile < 0) {
        const int pieces = d / 8;
        for (int i = threadIdx.x; i < u.len * pieces; i += kAttnThreads) {
            *reinterpret_cast<uint4 *>(dk.p + (u.row0 + i / pieces) * dk.ld + (long long)hk * d + i % pieces * 8) = make_uint4(0, 0, 0, 0);
            *reinterpret_cast<uint4 *>(dv.p + (u.row0 + i / pieces) * dv.ld + (long long)hk * d + i % pieces * 8) = make_uint4(0, 0, 0, 0);
        }
        return;
    }
    const int rows = u.len * G, first = u.tile * kKeyRows + (wave >> 1) * 32, key = min(first + (lane & 31), u.len - 1);
    const int need = key * G;                                 // this key's first packed row; keys behind the sequence see what its last one sees
    const int pair_first = min(first, u.len - 1) * G, pair_last = min(first + 31, u.len - 1) * G;

    // This wave's loads of a step's packed rows, step after step downwards.  Where groups divide the rows between two loads, every load's rows lie as
    // those of the load before, so many tokens on: a lane's constant beside a uniform base that moves by a constant.  (Divisions for every load took a
    // quarter of a step's time.)  Other groups' and the last rows' are worked out lane by lane.
    constexpr int APART = kAttnWaves * Tile::RPB;
    const int sub = lane / Tile::SPR, col = min((lane % Tile::SPR) ^ Tile::swz(wave * Tile::RPB + sub), d / 8 - 1) * 8;
    const unsigned magic = sh.magic;
    const int apart = token_of(APART, magic), top = u.to * kRowStep - APART + wave * Tile::RPB, top_in = token_of(top, magic), top_tok = u.row0 + top_in;
    const int col0 = (hk * G + top - top_in * G) * d, sub_in = token_of(sub, magic), stat_in = token_of((u.to - 1) * kRowStep + lane, magic);
    const bool alike = apart * G == APART;
    const bf16_t *q_at = q.p + (long long)top_tok * q.ld + col0, *d_at = dout.p + (long long)top_tok * dout.ld + col0;
    const long long q_apart = (long long)apart * q.ld, d_apart = (long long)apart * dout.ld;
    const float *stat = wave == 0 ? lse2 : minus_delta, *stat_at = stat + (long long)(u.row0 + stat_in) * sh.Hq + hk * G + ((u.to - 1) * kRowStep + lane - stat_in * G);
    const uint32_t q_off = (uint32_t)(sub_in * q.ld + (sub - sub_in * G) * d + col) * 2u, d_off = (uint32_t)(sub_in * dout.ld + (sub - sub_in * G) * d + col) * 2u;
    auto load = [&](int t, int slot) __attribute__((always_inline)) {
        char *to = lds + slot * Tile::BYTES + wave * 1024, *stat_to = lds + STATS + (slot * 2 + wave) * kRowStep * 4;
        if (alike && t * kRowStep + kRowStep <= rows) {
#pragma unroll
            for (int i = Tile::LOADS - 1; i >= 0; --i) {
                load_lds16_sv(q_at, q_off, to + i * kAttnWaves * 1024);
                load_lds16_sv(d_at, d_off, to + 2 * Tile::BYTES + i * kAttnWaves * 1024);
                q_at -= q_apart;
                d_at -= d_apart;
            }
            if (wave < 2) load_lds4(stat_at, stat_to);
        } else {
            rare();
            int row0 = u.row0;
            asm volatile("" : "+s"(row0));                    // (nothing of this branch is kept in registers for it)
#pragma unroll
            for (int i = 0; i < Tile::LOADS; ++i) {
                const int r = min(t * kRowStep + (wave + i * kAttnWaves) * Tile::RPB + sub, rows - 1), tok = token_of(r, magic), c0 = (hk * G + r - tok * G) * d + col;
                load_lds16(q.p + (long long)(row0 + tok) * q.ld + c0, to + i * kAttnWaves * 1024);
                load_lds16(dout.p + (long long)(row0 + tok) * dout.ld + c0, to + 2 * Tile::BYTES + i * kAttnWaves * 1024);
                q_at -= q_apart;
                d_at -= d_apart;
            }
            if (wave < 2) {
                const int r = min(t * kRowStep + lane, rows - 1), tok = token_of(r, magic);
                load_lds4(stat + (long long)(row0 + tok) * sh.Hq + hk * G + r - tok * G, stat_to);
            }
        }
        stat_at -= (long long)(kRowStep / G) * sh.Hq;
    };
    const uint32_t row_lane = Tile::row_lane(lane) + role * 32 * Tile::ROW, col_lane = Tile::col_lane(lane);
    load(u.to - 1, (u.to - 1) & 1);
    bf16x8_t kf[2 * ND], vf[2 * ND];
    load_row<ND>(kf, k.p + (long long)(u.row0 + key) * k.ld + hk * d, d, lane);
    load_row<ND>(vf, v.p + (long long)(u.row0 + key) * v.ld + hk * d, d, lane);

    const float c = sh.scale * kLog2e;
    f32x16_t acc[ND];
#pragma unroll
    for (int n = 0; n < ND; ++n) acc[n] = zero16();
    char *give = lds + TRADE + (wave >> 1) * PAIR + (role ? 4096 : 0) + lane * 16;
    const char *take = lds + TRADE + (wave >> 1) * PAIR + (role ? 0 : 4096) + lane * 16;
    const int fine = kExactSteps * kKeyTile * G;              // rows before that see few keys
    // From the last rows to the first: the blocks of a head, which begin at different rows, then read the same ones at about the same time, out of L2.
    auto walk = [&](auto which) __attribute__((always_inline)) {
        constexpr int ROLE = decltype(which)::value;
        for (int t = u.to - 1; t >= u.from; --t) {
            tile_barrier();
            const int slot = t & 1, r0 = t * kRowStep;
            const char *qs = lds + slot * Tile::BYTES, *ds = qs + 2 * Tile::BYTES;
            const float *ls = reinterpret_cast<const float *>(lds + STATS + slot * 2 * kRowStep * 4) + ROLE * 32 + (lane >> 5) * 4, *Ds = ls + kRowStep;
            if (t > u.from) load(t - 1, slot ^ 1);
            const bool dead = r0 + kRowStep - 1 < pair_first; // all of these rows come before this pair's keys
            const uint32_t cols = lds_at(ROLE ? qs : ds, col_lane);
            bf16x8_t f[ND];
            auto fetch = [&](int half, int j) __attribute__((always_inline)) {
#pragma unroll
                for (int n = 0; n < ND; ++n) f[n] = Tile::cols(cols + half * 32 * Tile::ROW, n * 32, j * 16);
            };
            auto add = [&](const bf16x8_t &x) __attribute__((always_inline)) {
#pragma unroll
                for (int n = 0; n < ND; ++n) acc[n] = mfma16(f[n], x, acc[n]);
            };
            if (!dead) {
                f32x16_t s, dp, minus_D;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 D4 = *reinterpret_cast<const float4 *>(Ds + g * 8);
                    minus_D[4 * g] = D4.x, minus_D[4 * g + 1] = D4.y, minus_D[4 * g + 2] = D4.z, minus_D[4 * g + 3] = D4.w;
                }
                score_pair<ND>(lds_at(qs, row_lane), lds_at(ds, row_lane), kf, vf, minus_D, s, dp);
                if (r0 < max(pair_last, G) || r0 + kRowStep > rows) {
                    rare();
                    const int base = r0 + ROLE * 32 + (lane >> 5) * 4;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int r = base + (i >> 2) * 8 + (i & 3);
                        if (r < need || r >= rows) s[i] = -INFINITY;
                        if (r < G) dp[i] = 0.0f;              // the sequence's first token: one key, no gradient of its scores
                    }
                }
                // exponentials and gradients of 16 rows; the half that this wave adds up, and the other wave's to LDS
                auto gradients = [&](int j) __attribute__((always_inline)) {
#pragma unroll
                    for (int g = 2 * j; g < 2 * j + 2; ++g) {
                        const float4 l4 = *reinterpret_cast<const float4 *>(ls + g * 8);
                        const float lv[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            s[4 * g + i] = __builtin_amdgcn_exp2f(fmaf(s[4 * g + i], c, -lv[i]));
                            dp[4 * g + i] *= s[4 * g + i];
                        }
                    }
                    const bf16x8_t p = pack_half(s, j), e = pack_half(dp, j);
                    *reinterpret_cast<bf16x8_t *>(give + j * 1024) = ROLE ? p : e;
                    return ROLE ? e : p;
                };
                fetch(ROLE, 0);
                const bf16x8_t x0 = gradients(0);
                in_order();
                add(x0);
                const bf16x8_t x1 = gradients(1);
                in_order();
                fetch(ROLE, 1);
                add(x1);
                if (r0 < fine) {                              // what the rounding of ds left
                    rare();
                    if (ROLE) {
                        add(pack_rest(dp, 1));
                        fetch(ROLE, 0);
                        add(pack_rest(dp, 0));
                    } else {
#pragma unroll
                        for (int j = 0; j < 2; ++j) *reinterpret_cast<bf16x8_t *>(give + 2048 + j * 1024) = pack_rest(dp, j);
                    }
                }
                fetch(ROLE ^ 1, 0);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (dead) continue;
            const bf16x8_t y0 = *reinterpret_cast<const bf16x8_t *>(take), y1 = *reinterpret_cast<const bf16x8_t *>(take + 1024);
            add(y0);
            fetch(ROLE ^ 1, 1);
            add(y1);
            if (ROLE && r0 < fine) {
                rare();
                add(*reinterpret_cast<const bf16x8_t *>(take + 2048 + 1024));
                fetch(ROLE ^ 1, 0);
                add(*reinterpret_cast<const bf16x8_t *>(take + 2048));
            }
        }
    };
    if (role) walk(std::integral_constant<int, 1>{});
    else walk(std::integral_constant<int, 0>{});
    if (u.slot >= 0) {
        Part<ND>::put(parts, u.slot * sh.Hk + hk, wave, lane, acc);
        return;
    }
    const HeadsOut &to = role ? dk : dv;
    store_row<ND>(acc, role ? sh.scale : 1.0f, to.p + (long long)(u.row0 + key) * to.ld + hk * d, d, lane, first + (lane & 31) < u.len);
}

// Adds up the partial sums of the tiles that several blocks shared, in ascending order: those of rows, behind row_joins tiles' those of keys.
template <int ND>
__global__ void __launch_bounds__(kAttnThreads)
attn_join_kernel(AttnShape sh, int row_joins, const AttnList *__restrict__ rows, const AttnUnit *__restrict__ row_units, float *__restrict__ row_parts, HeadsOut dq,
                 const AttnList *__restrict__ keys, const AttnUnit *__restrict__ key_units, float *__restrict__ key_parts, HeadsOut dk, HeadsOut dv)
{
    const int n = blockIdx.x % ND, block = blockIdx.x / ND, tile = block / sh.Hk, hk = block - tile * sh.Hk, of_keys = tile >= row_joins, at = of_keys ? tile - row_joins : tile;
    if (at >= (of_keys ? keys : rows)->joins) return;
    const AttnUnit u = (of_keys ? key_units : row_units)[at];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float *parts = of_keys ? key_parts : row_parts;
    f32x16_t acc[1] = {zero16()};
#pragma unroll 4
    for (int c = 0; c < u.chunks; ++c) Part<ND>::add(parts, (u.slot + c) * sh.Hk + hk, wave, lane, n, 1.0f, acc[0]);
    const int first = of_keys ? u.tile * kKeyRows + (wave >> 1) * 32 : u.tile * kRowTile + wave * 32, count = of_keys ? u.len : u.len * sh.G;
    const int mine = min(first + (lane & 31), count - 1), tok = of_keys ? mine : token_of(mine, sh.magic), head = of_keys ? hk : hk * sh.G + mine - tok * sh.G;
    const HeadsOut &to = !of_keys ? dq : wave & 1 ? dk : dv;
    store_row<1>(acc, of_keys && !(wave & 1) ? 1.0f : sh.scale, to.p + (long long)(u.row0 + tok) * to.ld + head * sh.d + n * 32, sh.d - n * 32, lane, first + (lane & 31) < count);
}

// ---------------------------------------------------------------- host
inline int attn_nd(int d) { return (d + 31) / 32; }
// Lists: at most so many units, joined tiles and partial sums a key head, for rows and for keys.  A token is a sequence's or padding's, and padding
// takes no more places than it would as rows or keys, but for a tile a sequence.  Chunks have at least c steps: a fair share's worth (half of it: keys) of all steps, and a
// least number of them.  A tile of x > c steps has fewer than x / c + 1 < 2 x / c of them, all together fewer than twice their steps / c.
struct AttnSizes {
    int units, joins, slots;
    size_t part_bytes;
    size_t list_bytes() const { return round256(sizeof(AttnList) + (size_t)(units + joins) * sizeof(AttnUnit)); }
};
inline AttnSizes attn_sizes(long long tiles, long long most, long long whole, int min_chunk, int n_seq, int Hk, int d)
{
    AttnSizes s;
    whole = std::min(whole, tiles * most / min_chunk);
    s.joins = (int)std::min(whole, tiles);
    s.slots = (int)(2 * whole);
    s.units = (int)(tiles + n_seq + 2 * whole);
    s.part_bytes = round256((size_t)s.slots * Hk * kAttnWaves * attn_nd(d) * 16 * 64 * sizeof(float));
    return s;
}
inline AttnSizes row_sizes(int T, int n_seq, int Hq, int Hk, int d, bool bwd)
{
    const int G = Hq / Hk, most = tiles_of(T, kKeyTile);
    const long long rest = (long long)most * T * Hq / (kShareTiles * kRowTile);
    const bool share = most - rest >= (bwd ? kBwdShareSteps : kFwdShareSteps);
    return attn_sizes((long long)T * G / kRowTile + n_seq, most, share ? kAttnSlots / Hk + 1 : 0, kMinRowChunk, n_seq, Hk, d);
}
inline AttnSizes key_sizes(int T, int n_seq, int Hq, int Hk, int d)
{
    return attn_sizes(T / kKeyRows + n_seq, tiles_of((long long)T * (Hq / Hk), kRowStep), 2 * kAttnSlots / Hk + 1, kMinKeyChunk, n_seq, Hk, d);
}
// (a launch has fewer than 2^32 threads)
inline bool attn_takes(int T, int n_seq, int Hq, int Hk, int d)
{
    if (d % 8 || d > kAttnMaxDim || n_seq > kAttnMaxSeq || Hq / Hk > kAttnMaxGroup || Hq > 4096 || (long long)T * (Hq / Hk) > kAttnMaxRows) return false;
    return (long long)std::max(row_sizes(T, n_seq, Hq, Hk, d, true).units, key_sizes(T, n_seq, Hq, Hk, d).units) * Hk < (1ll << 32) / kAttnThreads - 1;
}
inline size_t row_sum_bytes(const AttnSizes &s, int Hk) { return round256((size_t)s.slots * Hk * kRowTile * sizeof(float2)); }
size_t attn_fwd_ws_bytes(int T, int n_seq, int Hq, int Hk, int d)
{
    if (T < 0 || n_seq < 0 || Hk < 1 || Hq < 1 || Hq % Hk || d < 8 || !attn_takes(T, n_seq, Hq, Hk, d)) return 0;
    const AttnSizes s = row_sizes(T, n_seq, Hq, Hk, d, false);
    return s.list_bytes() + s.part_bytes + row_sum_bytes(s, Hk);
}
size_t attn_bwd_ws_bytes(int T, int n_seq, int Hq, int Hk, int d)
{
    if (!attn_fwd_ws_bytes(T, n_seq, Hq, Hk, d)) return 0;
    const AttnSizes r = row_sizes(T, n_seq, Hq, Hk, d, true), k = key_sizes(T, n_seq, Hq, Hk, d);
    return r.list_bytes() + r.part_bytes + k.list_bytes() + k.part_bytes + 2 * round256((size_t)T * Hq * sizeof(float));
}
// A list in the workspace, and the next free byte behind it.
inline SchedOut sched_out(char *&ws, const AttnSizes &s)
{
    AttnList *head = (AttnList *)ws;
    AttnUnit *units = (AttnUnit *)(head + 1);
    ws += s.list_bytes();
    return SchedOut{head, units, units + s.units, s.slots > 0};
}
inline int check_attn(const int32_t *seq_start, int n_seq, int T, int Hq, int Hk, int d, float scale, const int32_t *err_flag)
{
    if (T < 0 || n_seq < 0 || Hq < 1 || Hk < 1 || Hq % Hk || d < 8 || !(scale > 0.0f) || scale > 1e38f) return RELIBRA_EINVAL;
    if (!attn_takes(T, n_seq, Hq, Hk, d)) return RELIBRA_EUNSUPPORTED;
    if (T > 0 && n_seq > 0 && (!seq_start || !err_flag)) return RELIBRA_EINVAL;
    return RELIBRA_OK;
}
template <class Fn> void attn_layout(int d, const Fn &fn)
{
    switch (attn_nd(d)) {
    case 1: fn(std::integral_constant<int, 1>{}); break;
    case 2: fn(std::integral_constant<int, 2>{}); break;
    case 3: fn(std::integral_constant<int, 3>{}); break;
    default: fn(std::integral_constant<int, 4>{}); break;
    }
}

}  // namespace relibra

using namespace relibra;

extern "C" int relibra_attention_fwd(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride, const int32_t *seq_start,
                                     const int32_t *seq_len, int n_seq, int T, int Hq, int Hk, int d, float scale, void *out, int64_t out_stride, float *lse,
                                     void *workspace, size_t workspace_bytes, int32_t *err_flag, relibra_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    const int rc = check_attn(seq_start, n_seq, T, Hq, Hk, d, scale, err_flag);
    if (rc != RELIBRA_OK) return rc;
    if (T == 0 || n_seq == 0) return RELIBRA_OK;
    const HeadRows in[3] = {{q, q_stride, Hq * d}, {k, k_stride, Hk * d}, {v, v_stride, Hk * d}}, to{out, out_stride, Hq * d};
    const Piece lse_all{lse, (size_t)T * Hq * sizeof(float)};
    if (!to.usable() || !lse || to.overlaps(lse_all, T)) return RELIBRA_EINVAL;
    for (const HeadRows &x : in)
        if (!x.usable() || x.overlaps(to, T) || x.overlaps(lse_all, T)) return RELIBRA_EINVAL;
    if (!aligned16(workspace)) return RELIBRA_EINVAL;
    const size_t need = attn_fwd_ws_bytes(T, n_seq, Hq, Hk, d);
    if (!workspace || workspace_bytes < need) return RELIBRA_EWORKSPACE;
    if (!pieces_apart(T, {in[0], in[1], in[2]}, {to}, {{seq_start, (n_seq + 1) * sizeof(int32_t)}, {seq_len, n_seq * sizeof(int32_t)}},
                      {lse_all, {workspace, need}, {err_flag, sizeof(int32_t)}}))
        return RELIBRA_EINVAL;
    const AttnSizes sz = row_sizes(T, n_seq, Hq, Hk, d, false);
    char *ws = (char *)workspace;
    const SchedOut rows = sched_out(ws, sz);
    float *parts = (float *)ws;
    float2 *sums = (float2 *)(ws + sz.part_bytes);
    const AttnShape sh{T, Hq, Hk, Hq / Hk, d, token_magic(Hq / Hk), scale};
    const HeadsOut oo{(bf16_t *)out, out_stride};
    const bool listed = sz.joins > 0 || n_seq > kSelfSeq;
    const UnitSource source{listed ? rows.head : nullptr, rows.units, seq_start, seq_len, n_seq, T, err_flag};
    if (listed)
        RELIBRA_LAUNCH(RELIBRA_K_ATTN_SCHED, stream, attn_sched_kernel<<<1, kSchedThreads, 0, stream>>>(seq_start, seq_len, n_seq, T, sh.G, sh.magic, Hk, rows, rows, err_flag));
    attn_layout(d, [&](auto nd) {
        constexpr int ND = decltype(nd)::value;
        RELIBRA_LAUNCH(RELIBRA_K_ATTN_FWD, stream, (attn_fwd_kernel<ND><<<sz.units * Hk, kAttnThreads, 0, stream>>>(
            sh, HeadsIn{(const bf16_t *)q, q_stride}, HeadsIn{(const bf16_t *)k, k_stride}, HeadsIn{(const bf16_t *)v, v_stride}, source, oo, lse, parts, sums)));
        if (listed && sz.joins > 0)
            RELIBRA_LAUNCH(RELIBRA_K_ATTN_JOIN, stream, (attn_join_out_kernel<ND><<<sz.joins * Hk * ND, kAttnThreads, 0, stream>>>(
                sh, rows.head, rows.joins, parts, sums, oo, lse)));
    });
    RELIBRA_HIP_TRY(launch_check());
    return RELIBRA_OK;
}

extern "C" int relibra_attention_bwd(const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride, const void *out,
                                     int64_t out_stride, const float *lse, const void *dout, int64_t dout_stride, const int32_t *seq_start, const int32_t *seq_len,
                                     int n_seq, int T, int Hq, int Hk, int d, float scale, void *dq, int64_t dq_stride, void *dk, int64_t dk_stride, void *dv,
                                     int64_t dv_stride, void *workspace, size_t workspace_bytes, int32_t *err_flag, relibra_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    const int rc = check_attn(seq_start, n_seq, T, Hq, Hk, d, scale, err_flag);
    if (rc != RELIBRA_OK) return rc;
    if (T == 0 || n_seq == 0) return RELIBRA_OK;
    const HeadRows in[5] = {{q, q_stride, Hq * d}, {k, k_stride, Hk * d}, {v, v_stride, Hk * d}, {out, out_stride, Hq * d}, {dout, dout_stride, Hq * d}};
    const HeadRows to[3] = {{dq, dq_stride, Hq * d}, {dk, dk_stride, Hk * d}, {dv, dv_stride, Hk * d}};
    const Piece lse_all{lse, (size_t)T * Hq * sizeof(float)};
    if (!lse) return RELIBRA_EINVAL;
    for (const HeadRows &x : in)
        if (!x.usable()) return RELIBRA_EINVAL;
    for (int i = 0; i < 3; ++i) {
        if (!to[i].usable() || to[i].overlaps(lse_all, T)) return RELIBRA_EINVAL;
        for (const HeadRows &x : in)
            if (x.overlaps(to[i], T)) return RELIBRA_EINVAL;
        for (int j = 0; j < i; ++j)
            if (to[j].overlaps(to[i], T)) return RELIBRA_EINVAL;
    }
    if (!aligned16(workspace)) return RELIBRA_EINVAL;
    const size_t need = attn_bwd_ws_bytes(T, n_seq, Hq, Hk, d);
    if (!workspace || workspace_bytes < need) return RELIBRA_EWORKSPACE;
    if (!pieces_apart(T, {in[0], in[1], in[2], in[3], in[4]}, {to[0], to[1], to[2]}, {{seq_start, (n_seq + 1) * sizeof(int32_t)}, {seq_len, n_seq * sizeof(int32_t)}, lse_all},
                      {{workspace, need}, {err_flag, sizeof(int32_t)}}))
        return RELIBRA_EINVAL;
    const AttnSizes rs = row_sizes(T, n_seq, Hq, Hk, d, true), ks = key_sizes(T, n_seq, Hq, Hk, d);
    char *ws = (char *)workspace;
    const SchedOut rows = sched_out(ws, rs), keys = sched_out(ws, ks);
    float *row_parts = (float *)ws, *key_parts = (float *)(ws += rs.part_bytes);
    float *lse2 = (float *)(ws += ks.part_bytes), *delta = (float *)(ws + round256((size_t)T * Hq * sizeof(float)));
    const AttnShape sh{T, Hq, Hk, Hq / Hk, d, token_magic(Hq / Hk), scale};
    const HeadsIn qi{(const bf16_t *)q, q_stride}, ki{(const bf16_t *)k, k_stride}, vi{(const bf16_t *)v, v_stride}, oi{(const bf16_t *)out, out_stride},
        di{(const bf16_t *)dout, dout_stride};
    const HeadsOut dqo{(bf16_t *)dq, dq_stride}, dko{(bf16_t *)dk, dk_stride}, dvo{(bf16_t *)dv, dv_stride};
    // Rows' units are found without a list where no tile of theirs is shared.  Keys' are where no tile can have more than 8 steps: those of 5 to 8 would be
    // shared with a list, but making it and joining costs about what that saves; beyond, the list is made beside dq.  One sequence backward, found / listed, us: 5
    // steps (320 tokens of 8 heads) 25 / 27, 8 steps (512 tokens of 2, 8, 32, 64 heads) 33.5 / 31.5, 34 / 33, 36 / 40, 40 / 51, 16 steps (1024 of 2, 8, 32) 54 / 44,
    // 55 / 52, 61 / 72.
    const bool rows_listed = rs.joins > 0 || n_seq > kSelfSeq;
    const bool keys_listed = rows_listed || tiles_of((long long)T * sh.G, kRowStep) > 2 * kMinKeyChunk;
    const int beside = keys_listed && !rows_listed;
    const UnitSource row_source{rows_listed ? rows.head : nullptr, rows.units, seq_start, seq_len, n_seq, T, err_flag};
    const UnitSource key_source{keys_listed ? keys.head : nullptr, keys.units, seq_start, seq_len, n_seq, T, err_flag};
    if (rows_listed)
        RELIBRA_LAUNCH(RELIBRA_K_ATTN_SCHED, stream, attn_sched_kernel<<<2, kSchedThreads, 0, stream>>>(seq_start, seq_len, n_seq, T, sh.G, sh.magic, Hk, rows, keys, err_flag));
    attn_layout(d, [&](auto nd) {
        constexpr int ND = decltype(nd)::value;
        RELIBRA_LAUNCH(RELIBRA_K_ATTN_DQ, stream, (attn_dq_kernel<ND><<<rs.units * Hk + beside, kAttnThreads, 0, stream>>>(
            sh, qi, ki, vi, oi, di, lse, row_source, beside, keys, dqo, lse2, delta, row_parts)));
        RELIBRA_LAUNCH(RELIBRA_K_ATTN_DKV, stream, (attn_dkv_kernel<ND><<<ks.units * Hk, kAttnThreads, 0, stream>>>(
            sh, qi, ki, vi, di, lse2, delta, key_source, dko, dvo, key_parts)));
        if (keys_listed && rs.joins + ks.joins > 0)
            RELIBRA_LAUNCH(RELIBRA_K_ATTN_JOIN, stream, (attn_join_kernel<ND><<<(rs.joins + ks.joins) * Hk * ND, kAttnThreads, 0, stream>>>(
                sh, rs.joins, rows.head, rows.joins, row_parts, dqo, keys.head, keys.joins, key_parts, dko, dvo)));
    });
    RELIBRA_HIP_TRY(launch_check());
    return RELIBRA_OK;
}
