// Orthogonalised updates: momentum and Newton-Schulz steps on a batch of matrices (the weight gradients of the experts).
//
//   M' = mu M + G,  U = G + mu M' (Nesterov) or M' (or G without momentum),  X = U / |U|_F, then five (`steps`) times
//   A = X X^T (over the longer side),  B = b A + c A^2,  X = a X + B X         and  out = scale X.
// The polynomial a s + b s^3 + c s^5 takes every singular value of at most 1 towards 1.
//
// Precision.  The products' operands are IEEE halves: 11 bits where bf16 has 8, at the same MFMA rate, and the range suffices
// because singular values stay below 1.3: everything is stored times 2^12 (kScale), which keeps the entries of a large matrix
// (about 1 / sqrt(m n)) out of the subnormals.  The linear term a X is another matter: what rounding puts outside of X's row and column
// spaces is multiplied by a = 3.4 in every step, by 485 in all, and a gradient of few tokens has few dimensions.  X is therefore
// kept as the sum of two halves, hi + lo (22 bits), of which only hi enters products.  Near the end X X^T is close to a multiple of
// I, and so is B (-2.4 I): the diagonals of A and B are kept apart in fp32 and the products' operands have a diagonal of zeros, so
// that what is rounded is small:  X' = (a + dB) hi + (a + w dB) lo + (B - dB) hi  row by row.  B hi stands for B X: what the
// product leaves out of lo is put back for the diagonal, w = 1, but only in the last three steps, since dB lo, unlike B lo, does leave X's
// row space.  Relative error of the result (norm) in a simulation against double precision, before the result's own
// rounding to bf16 (1.7e-3), with bf16 operands / halves alone / lo kept too / and the diagonals apart: 128 x 256 Gaussian 1.2e-2 /
// 1.7e-3 / 1.7e-3 / 5.9e-4, 64 x 1000 1.3e-2 / 1.8e-3 / 2.1e-3 / 3.1e-4, rank 1 1.2 / 0.15 / 4.0e-4 / 5.5e-4, rank 16 of 256 x 500
// 0.3 / 3e-2 / 5.5e-4 / 7.4e-4.
//
// Matrices are padded to multiples of 64 with zeros, which every step leaves zero.  X lies as the gradient does; the Gram matrix is
// taken over the longer side, along memory (wide) or across it (tall), and X is multiplied from the left or the right.  A and B
// are symmetric: only tiles on and below the diagonal are computed, and stored twice.
//
// 32 of 1536 x 4096 take 6.99 ms, of which 5 x (gram 343, poly 160, update 720 us) are products: 0.90, 0.73 and 0.86 PFLOP/s of what the
// formulas need (a large library product of halves reaches 1.37).  Gram and poly are bound by the matrix units, with 21 tiles of 256 x 256 for 18 tiles' worth
// and 2.6 rounds of the units paid as 3.  The update is bound by them and then by memory, one behind the other: its epilogue reads and writes hi and lo, 8 bytes a
// value, 1.6 GB a launch or about 320 us at the copy rate, while a workgroup that has its unit to itself multiplies nothing, and tiles of one
// length keep the units in step.  (The last step writes 2 bytes for 4: 655 us where the others take 735, traced.)
#include "gemm_tile.h"
#include "wave_ops.h"
#include "wave_stage.h"

#include <algorithm>

namespace relibra {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kScale = 4096.0f;
constexpr int kOrthoPad = 64;
constexpr int kMinParts = 16, kMaxParts = 1024;  // partial sums of a matrix's squares
constexpr int kOrthoMaxSide = 32768;
constexpr int kOrthoMaxSteps = 8;                // rank 1 of 256 x 500, simulated: an error of 1.5e-3 of the norm (outside of its space, times 3.44 a step)
constexpr int kComputeUnits = 256;

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));

struct OrthoShape {
    int n, rows, cols;                           // matrices, as the caller gives them
    int rp, cp;                                  // padded
    bool tall;                                   // rows > cols
};
// Workspace: two copies of X's first halves (a step reads one and writes the other), the second halves, A, B, their diagonals,
// parts of A where its contraction is split.
struct OrthoWs {
    uint16_t *x[2], *lo, *a, *b;
    float *da, *db, *part;
};
inline size_t ortho_x_bytes(const OrthoShape &s) { return round256((size_t)s.n * s.rp * s.cp * 2); }
inline size_t ortho_gram_bytes(const OrthoShape &s)
{
    const size_t m = s.tall ? s.cp : s.rp;
    return round256((size_t)s.n * m * m * 2);
}
inline size_t ortho_diag_bytes(const OrthoShape &s) { return round256((size_t)s.n * (s.tall ? s.cp : s.rp) * sizeof(float)); }
inline OrthoShape ortho_shape(int n, int rows, int cols)
{
    auto pad = [](int v) { return (v + kOrthoPad - 1) / kOrthoPad * kOrthoPad; };
    return OrthoShape{n, rows, cols, pad(rows), pad(cols), rows > cols};
}
// Blocks that share a matrix's squares: about 2048 over all matrices, each with 4096 values or more, but 16 a matrix at least (of small ones
// some have nothing to do) and 1024 at most.  With 64 a matrix one of 4096 x 4096 took 197 us (0.25 of the copy rate).
inline int norm_parts(int n, int rows, int cols)
{
    const size_t values = (size_t)rows * cols;
    return (int)std::min<size_t>(std::max<size_t>(std::min<size_t>((2048 + n - 1) / n, values / 4096), kMinParts), kMaxParts);
}
// ---------------------------------------------------------------- momentum, norm, first halves
enum { U_GRAD = 0, U_MOMENTUM = 1, U_NESTEROV = 2 };
__device__ __forceinline__ float update_of(float g, float m_new, float mu, int mode)
{
    return mode == U_GRAD ? g : mode == U_MOMENTUM ? m_new : fmaf(mu, m_new, g);
}

// M' and the sum of U^2, part blockIdx.x of matrix blockIdx.y.  Squares in double: no gradient is too large or small.  Eight values at a
// time, wherever the matrix starts.  Bound by memory: 32 of 1536 x 4096 in fp32 450 us, 2.4 GB at 5.4 TB/s.
template <class GT>
__global__ void __launch_bounds__(256)
ortho_momentum_kernel(const GT *__restrict__ g, const float *m, float mu, int mode, size_t per_matrix, float *m_out, double *__restrict__ parts)
{
    __shared__ double red[4];
    const size_t base = (size_t)blockIdx.y * per_matrix;
    double sum = 0.0;
    auto one = [&](float gv, float mv) __attribute__((always_inline)) {
        const float mn = mode == U_GRAD ? 0.0f : fmaf(mu, mv, gv);
        const double u = update_of(gv, mn, mu, mode);
        sum += u * u;
        return mn;
    };
    const size_t eights = per_matrix / 8, stride = (size_t)gridDim.x * 256;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < eights; i += stride) {
        float gv[8], mv[8] = {};
        unpack8(fetch8_any(g + base + i * 8), gv);
        if (mode != U_GRAD) unpack8(fetch8_any(m + base + i * 8), mv);
#pragma unroll
        for (int j = 0; j < 8; ++j) mv[j] = one(gv[j], mv[j]);
        if (mode != U_GRAD) store8_any(m_out + base + i * 8, mv);
    }
    const size_t rest = eights * 8 + threadIdx.x;
    if (blockIdx.x == 0 && rest < per_matrix) {
        const float mn = one(to_f32(g[base + rest]), mode != U_GRAD ? m[base + rest] : 0.0f);
        if (mode != U_GRAD) m_out[base + rest] = mn;
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) parts[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// X = kScale U / |U| as two halves, padding included.  A thread takes 8 consecutive padded columns of a row.  A pass of its own over G
// and M', since |U| is known only behind the first.  Bound by memory: 32 of 1536 x 4096 465 us, 2.4 GB at 5.2 TB/s.
template <class GT>
__global__ void __launch_bounds__(256)
ortho_load_kernel(const GT *__restrict__ g, const float *__restrict__ m_new, float mu, int mode, OrthoShape s, const double *__restrict__ parts,
                  int n_parts, uint16_t *__restrict__ hi, uint16_t *__restrict__ lo)
{
    __shared__ double scale_of;
    const int b = blockIdx.y;
    if (threadIdx.x < 64) {
        double sum = 0.0;
        for (int i = threadIdx.x; i < n_parts; i += 64) sum += parts[(size_t)b * n_parts + i];
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
        if (threadIdx.x == 0) scale_of = sum == 0.0 ? 0.0 : (double)kScale / sqrt(sum);
    }
    __syncthreads();
    const double scale = scale_of;
    const int per_row = s.cp / 8;
    const unsigned pieces = (unsigned)((size_t)s.rp * per_row);                     // at most 2^27: sides of at most 32768
    const size_t from = (size_t)b * s.rows * s.cols, to = (size_t)b * s.rp * s.cp;
    for (unsigned p = blockIdx.x * 256 + threadIdx.x; p < pieces; p += gridDim.x * 256) {
        const int r = p / (unsigned)per_row, c = p % (unsigned)per_row * 8;
        float gv[8] = {}, mv[8] = {}, u[8];
        const size_t at = from + (size_t)r * s.cols + c;
        const bool whole = r < s.rows && c + 8 <= s.cols;
        if (whole) {
            if (mode != U_MOMENTUM) unpack8(fetch8_any(g + at), gv);
            if (mode != U_GRAD) unpack8(fetch8_any(m_new + at), mv);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool in = r < s.rows && c + j < s.cols;
            if (!whole) {
                gv[j] = in && mode != U_MOMENTUM ? to_f32(g[at + j]) : 0.0f;
                mv[j] = in && mode != U_GRAD ? m_new[at + j] : 0.0f;
            }
            u[j] = in ? (float)((double)update_of(gv[j], mv[j], mu, mode) * scale) : 0.0f;
        }
        uint16_t h8[8], l8[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const _Float16 h = (_Float16)u[j];
            h8[j] = __builtin_bit_cast(uint16_t, h);
            l8[j] = __builtin_bit_cast(uint16_t, (_Float16)(u[j] - (float)h));
        }
        const size_t out = to + (size_t)r * s.cp + c;
        *reinterpret_cast<uint4 *>(hi + out) = *reinterpret_cast<const uint4 *>(h8);
        *reinterpret_cast<uint4 *>(lo + out) = *reinterpret_cast<const uint4 *>(l8);
    }
}

// ---------------------------------------------------------------- products
// A tile has BB rows (on the lanes) and BA columns (in the accumulator registers); a wave owns 64 rows and COLS columns.  ADEPTH, BDEPTH: values
// of the contraction in an LDS tile of the column and of the row operand.
template <int BA_, int BB_, int STAGES_, int OCC_, int ADEPTH_ = BK, int BDEPTH_ = ADEPTH_> struct OrthoCfg {
    static constexpr int BA = BA_, BB = BB_, WA = 2, WB = BB / 64, THREADS = WA * WB * 64, STAGES = STAGES_;
    static constexpr int COLS = BA / WA;                             // of a wave
    static constexpr int ADEPTH = ADEPTH_, BDEPTH = BDEPTH_;
    static constexpr int WAVES_PER_SIMD = OCC_ * WA * WB / 4;        // OCC_: workgroups per compute unit
    static constexpr bool DEEP = BDEPTH == 2 * ADEPTH;               // the row operand's tiles have a ring of their own
    static constexpr int SLABS = STAGES * (BA + (DEEP ? 0 : BB)) * ADEPTH * 2 + (DEEP ? (STAGES + 3) / 2 * BB * BDEPTH * 2 : 0);
    static constexpr int STAGING = WA * WB * 2 * WaveStage<64>::BYTES;
    static constexpr int LDS = SLABS > STAGING ? SLABS : STAGING;
    template <class AT, class BT = KcTile<BB, BDEPTH>> using Loop = KLoop<AT, BT, 1, 1, BA, BB, WA, WB, 1, false, STAGES, true, false, false, true>;
};

__device__ __forceinline__ uint2 pack4h(const float (&v)[4])
{
    const f16x4_t h = {(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
    return __builtin_bit_cast(uint2, h);
}
__device__ __forceinline__ void unpack4h(uint2 w, float (&v)[4])
{
    const f16x4_t h = __builtin_bit_cast(f16x4_t, w);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)h[i];
}

// Physical block -> tile: block % 8 is the XCD, each takes an eighth of the tile list, so neighbouring tiles share an L2.
__device__ __forceinline__ int xcd_tile(int block, int total)
{
    const int per_xcd = (total + 7) >> 3;
    const int t = (block & 7) * per_xcd + (block >> 3);
    return (block >> 3) < per_xcd && t < total ? t : -1;
}

// Symmetric product S = P P^T over k (P [m, k], k along memory: ACROSS = false; or P^T stored, [k, m]: ACROSS = true).
// POLY: out = b P + c P P / kScale instead of P P^T / kScale (P symmetric, m = k).  The diagonals are kept apart: `diag_out` takes
// the result's, out has zeros there; P = p + diag(diag_in) in the POLY form, so that P P = p p + (d_r + d_c) p_rc + d^2.
// Tiles that hold anything on or below the diagonal, row block after row block; of these the 64 x 64 blocks on or below it are
// stored, those below a second time with rows and columns exchanged, read back from the staging area by transposing LDS reads.
template <class CF> __host__ __device__ constexpr int gram_tiles_of_row(int i) { return ((i + 1) * CF::BB - 1) / CF::BA + 1; }
// Tile (i, j) of the triangle: which rows and columns.
template <class CF> __device__ __forceinline__ void gram_tile(int tile, int &row0, int &col0)
{
    int i = 0;
    while (tile >= gram_tiles_of_row<CF>(i)) tile -= gram_tiles_of_row<CF>(i++);
    row0 = i * CF::BB;
    col0 = tile * CF::BA;
}
// A wave's 64 x 64 block of sums (rows wrow0.., columns wcol0.. at most as far) to halves, diagonal apart, stored in both triangles.  buf: two
// staging areas.  src, din: P and its diagonal (POLY).
template <bool POLY>
__device__ __forceinline__ void gram_block(const f32x16_t (*sums)[2], char *buf, const uint16_t *src, const float *din, int m, int wrow0, int wcol0, uint16_t *dst,
                                           float *dout, int lane)
{
    using ST = WaveStage<64>;
    float d_r[2] = {0.0f, 0.0f}, d_c[2][4][4];
    if (POLY) {
#pragma unroll
        for (int ta = 0; ta < 2; ++ta)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<float4 *>(d_c[ta][q]) = *reinterpret_cast<const float4 *>(din + wcol0 + ta * 32 + q * 8 + (lane >> 5) * 4);
        ST::fill(buf, src, m, wrow0, m, wcol0, m, lane);
        d_r[0] = din[wrow0 + (lane & 31)];
        d_r[1] = din[wrow0 + 32 + (lane & 31)];
        wave_lds_fence();
    }
#pragma unroll
    for (int tb = 0; tb < 2; ++tb)
#pragma unroll
        for (int ta = 0; ta < 2; ++ta)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = tb * 32 + (lane & 31), c = ta * 32 + q * 8 + (lane >> 5) * 4;
                float v[4], old[4];
                if (POLY) unpack4h(ST::get(buf, r, c), old);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float s = sums[ta][tb][q * 4 + e];
                    v[e] = POLY ? kNsB * old[e] + (kNsC / kScale) * (s + (d_r[tb] + d_c[ta][q][e]) * old[e]) : s * (1.0f / kScale);
                    if (wrow0 == wcol0 && r == c + e) {
                        dout[wrow0 + r] = POLY ? kNsB * d_r[tb] + (kNsC / kScale) * (s + d_r[tb] * d_r[tb]) : v[e];
                        v[e] = 0.0f;
                    }
                }
                ST::put(buf, r, c, pack4h(v));
            }
    wave_lds_fence();
    ST::flush(buf, dst, m, wrow0, m, wcol0, m, lane);
    if (wrow0 != wcol0) {
        char *turned = buf + ST::BYTES;
#pragma unroll
        for (int r0 = 0; r0 < 64; r0 += 32)               // rows of the exchanged block: columns r0 .. r0 + 31 of the staged one
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const int bq = lane >> 4, iq = lane & 15;
                const int c = r0 + (bq & 1) * 16 + (iq & 3) * 4, r = kk * 16 + (bq >> 1) * 8 + (iq >> 2);
                const s16x4_t l = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)RELIBRA_LDS(buf + ST::acc_addr(r, c)));
                const s16x4_t h = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)RELIBRA_LDS(buf + ST::acc_addr(r + 4, c)));
                const s16x8_t v = __builtin_shufflevector(l, h, 0, 1, 2, 3, 4, 5, 6, 7);
                *reinterpret_cast<s16x8_t *>(turned + ST::acc_addr(r0 + (lane & 31), kk * 16 + (lane >> 5) * 8)) = v;
            }
        wave_lds_fence();
        ST::flush(turned, dst, m, wcol0, m, wrow0, m, lane);
    }
    wave_lds_fence();
}
template <class CF, bool POLY, class Acc>
__device__ __forceinline__ void gram_epilogue(const Acc &acc, char *lds, const uint16_t *src, const float *din, int m, int row0, int col0, uint16_t *dst, float *dout)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    __syncthreads();                                          // every wave is done with the operand slabs
    char *buf = lds + wave * 2 * WaveStage<64>::BYTES;
    const int wrow0 = row0 + (wave % CF::WB) * 64;
#pragma unroll
    for (int half = 0; half < CF::COLS / 64; ++half) {
        const int wcol0 = col0 + (wave / CF::WB) * CF::COLS + half * 64;
        if (wrow0 >= m || wcol0 > wrow0) break;               // uniform in the wave; padding is in whole runs of 64
        gram_block<POLY>(&acc[0][half * 2], buf, src, din, m, wrow0, wcol0, dst, dout, lane);
    }
}
template <class CF, bool ACROSS, bool POLY>
__global__ void __launch_bounds__(CF::THREADS, CF::WAVES_PER_SIMD)
ortho_gram_kernel(const uint16_t *__restrict__ p, const float *__restrict__ diag_in, int m, int k, int per_matrix, int total, int splits, int k_split,
                  uint16_t *__restrict__ out, float *__restrict__ diag_out, float *__restrict__ part)
{
    using KL = typename std::conditional<ACROSS, typename CF::template Loop<KsTile<CF::BA, CF::ADEPTH>, KsTile<CF::BB, CF::ADEPTH>>,
                                         typename CF::template Loop<KcTile<CF::BA, CF::ADEPTH>>>::type;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int t = xcd_tile(blockIdx.x, total);
    if (t < 0) return;
    const int tile = t / splits, split = t % splits, mat = tile / per_matrix;
    int row0, col0;
    gram_tile<CF>(tile % per_matrix, row0, col0);
    const uint16_t *src = p + (size_t)mat * m * k;
    const int ld = ACROSS ? m : k, k0 = split * k_split, depth = min(k - k0, k_split);
    const uint16_t *from = src + (ACROSS ? (size_t)k0 * m : (size_t)k0);
    const Operand A[1][1] = {{{from, ld, col0, m - 1}}}, B[1][1] = {{{from, ld, row0, m - 1}}};
    typename KL::Acc acc;
    KL::zero(acc);
    KL::run(acc, A, B, depth / CF::ADEPTH, depth, lds, threadIdx.x);
    if (!POLY && splits > 1) {
        float4 *to = reinterpret_cast<float4 *>(part) + ((size_t)t * CF::THREADS / 64 + (threadIdx.x >> 6)) * CF::COLS / 32 * 2 * 4 * 64 + (threadIdx.x & 63);
#pragma unroll
        for (int ta = 0; ta < CF::COLS / 32; ++ta)
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    to[((ta * 2 + tb) * 4 + q) * 64] = make_float4(acc[0][ta][tb][4 * q], acc[0][ta][tb][4 * q + 1], acc[0][ta][tb][4 * q + 2], acc[0][ta][tb][4 * q + 3]);
        return;
    }
    gram_epilogue<CF, POLY>(acc, lds, src, POLY ? diag_in + (size_t)mat * m : nullptr, m, row0, col0, out + (size_t)mat * m * m, diag_out + (size_t)mat * m);
}

// A 64 x 64 block of A (one wave's of a tile) from the parts of a split contraction: wave w adds up parts w, w + 4, .., then the first
// wave the four sums, always in this order.  (One workgroup a tile took 15 to 30 us: nothing but a wave's own loads in flight.)
template <class CF>
__global__ void __launch_bounds__(256)
ortho_join_kernel(const float *__restrict__ part, int m, int per_matrix, int splits, uint16_t *__restrict__ out, float *__restrict__ diag_out)
{
    static_assert(CF::COLS == 64, "a wave's block");
    constexpr int WAVES = CF::WA * CF::WB;
    __shared__ __attribute__((aligned(1024))) char lds[4 * 16 * 1024];
    const int tile = blockIdx.x / WAVES, of = blockIdx.x % WAVES, mat = tile / per_matrix, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int row0, col0;
    gram_tile<CF>(tile % per_matrix, row0, col0);
    const int wrow0 = row0 + of % CF::WB * 64, wcol0 = col0 + of / CF::WB * 64;
    if (wrow0 >= m || wcol0 > wrow0) return;
    f32x16_t sums[2][2];
#pragma unroll
    for (int i = 0; i < 64; ++i) sums[i >> 5][(i >> 4) & 1][i & 15] = 0.0f;
    auto add = [&](const float4 *from) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float4 v = from[i * 64 + lane];
            f32x16_t &to = sums[i >> 3][(i >> 2) & 1];
            to[4 * (i & 3)] += v.x;
            to[4 * (i & 3) + 1] += v.y;
            to[4 * (i & 3) + 2] += v.z;
            to[4 * (i & 3) + 3] += v.w;
        }
    };
#pragma unroll 2
    for (int s = wave; s < splits; s += 4) add(reinterpret_cast<const float4 *>(part) + (((size_t)tile * splits + s) * WAVES + of) * 16 * 64);
    float4 *mine = reinterpret_cast<float4 *>(lds + wave * 16 * 1024);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const f32x16_t &v = sums[i >> 3][(i >> 2) & 1];
        mine[i * 64 + lane] = make_float4(v[4 * (i & 3)], v[4 * (i & 3) + 1], v[4 * (i & 3) + 2], v[4 * (i & 3) + 3]);
    }
    __syncthreads();
    if (wave) return;
    for (int w = 1; w < 4; ++w) add(reinterpret_cast<const float4 *>(lds + w * 16 * 1024));
    wave_lds_fence();
    gram_block<false>(&sums[0], lds, nullptr, nullptr, m, wrow0, wcol0, out + (size_t)mat * m * m, diag_out + (size_t)mat * m, lane);
}

// X' = (a + d) hi + (a + w d) lo + B hi, d the diagonal of B kept apart.  Wide: X [m, n], B from the left, its rows on the lanes, X's
// columns across memory in the registers.  Tall: X [n, m], its rows on the lanes, B from the right, B's columns (which are its rows) in
// the registers.  The last step writes the caller's matrix instead.
struct OrthoLast {
    uint16_t *out;                               // bf16 [n, rows, cols], or nullptr: not the last step
    float scale;
    int vec;                                     // rows of 8-value pieces: 16-byte stores
};
template <class CF, bool TALL>
__global__ void __launch_bounds__(CF::THREADS, CF::WAVES_PER_SIMD)
ortho_update_kernel(const uint16_t *__restrict__ x, uint16_t *lo, const uint16_t *__restrict__ bmat, const float *__restrict__ diag, float w, OrthoShape s,
                    int tiles_r, int tiles_c, int total, uint16_t *__restrict__ x_out, OrthoLast last)
{
    using KL = typename CF::template Loop<typename std::conditional<TALL, KcTile<CF::BA, CF::ADEPTH>, KsTile<CF::BA, CF::ADEPTH>>::type>;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int t = xcd_tile(blockIdx.x, total);
    if (t < 0) return;
    const int per_matrix = tiles_r * tiles_c, mat = t / per_matrix, rem = t % per_matrix;
    // neighbouring tiles share a panel of X, B is shared by all
    const int i = TALL ? rem / tiles_c : rem % tiles_r, j = TALL ? rem % tiles_c : rem / tiles_r;
    const int m = TALL ? s.cp : s.rp;
    const uint16_t *X = x + (size_t)mat * s.rp * s.cp, *Bm = bmat + (size_t)mat * m * m;
    const int row0 = i * CF::BB, col0 = j * CF::BA;
    const Operand A[1][1] = {{TALL ? Operand{Bm, m, col0, m - 1} : Operand{X, s.cp, col0, s.cp - 1}}};
    const Operand B[1][1] = {{TALL ? Operand{X, s.cp, row0, s.rp - 1} : Operand{Bm, m, row0, m - 1}}};
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    typename KL::Acc acc;
    KL::zero(acc);
    KL::run(acc, A, B, m / CF::ADEPTH, m, lds, tid);
    __syncthreads();                                          // every wave is done with the operand slabs
    using ST = WaveStage<64>;
    char *buf_h = lds + wave * 2 * ST::BYTES, *buf_l = buf_h + ST::BYTES;
    uint16_t *L = lo + (size_t)mat * s.rp * s.cp, *Xo = x_out + (size_t)mat * s.rp * s.cp;
    const int wrow0 = row0 + (wave % CF::WB) * 64;
#pragma unroll
    for (int half = 0; half < CF::COLS / 64; ++half) {
        const int wcol0 = col0 + (wave / CF::WB) * CF::COLS + half * 64;
        if (wrow0 >= s.rp || wcol0 >= s.cp) break;
        ST::fill2(buf_h, buf_l, X, L, s.cp, wrow0, s.rp, wcol0, s.cp, lane);
        const float *d = diag + (size_t)mat * m;
        float d_r[2] = {0.0f, 0.0f};
        if (!TALL) {
            d_r[0] = d[wrow0 + (lane & 31)] * (1.0f / kScale);
            d_r[1] = d[wrow0 + 32 + (lane & 31)] * (1.0f / kScale);
        }
        wave_lds_fence();
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
#pragma unroll
            for (int ta = 0; ta < 2; ++ta)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int r = tb * 32 + (lane & 31), c = ta * 32 + q * 8 + (lane >> 5) * 4;
                    float h[4], l[4], v[4], d_c[4];
                    if (TALL) *reinterpret_cast<float4 *>(d_c) = *reinterpret_cast<const float4 *>(d + wcol0 + c);
                    unpack4h(ST::get(buf_h, r, c), h);
                    unpack4h(ST::get(buf_l, r, c), l);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float de = TALL ? d_c[e] * (1.0f / kScale) : d_r[tb];
                        v[e] = (kNsA + de) * h[e] + ((kNsA + w * de) * l[e] + acc[0][half * 2 + ta][tb][q * 4 + e] * (1.0f / kScale));
                    }
                    if (last.out) {
                        const float f = last.scale * (1.0f / kScale);
                        ST::put(buf_h, r, c, make_uint2(pack2bf(f * v[0], f * v[1]), pack2bf(f * v[2], f * v[3])));
                    } else {
                        const uint2 hp = pack4h(v);
                        unpack4h(hp, h);
#pragma unroll
                        for (int e = 0; e < 4; ++e) l[e] = v[e] - h[e];
                        ST::put(buf_h, r, c, hp);
                        ST::put(buf_l, r, c, pack4h(l));
                    }
                }
        wave_lds_fence();
        if (!last.out) {
            ST::flush(buf_h, Xo, s.cp, wrow0, s.rp, wcol0, s.cp, lane);
            ST::flush(buf_l, L, s.cp, wrow0, s.rp, wcol0, s.cp, lane);
        } else {
            uint16_t *O = last.out + (size_t)mat * s.rows * s.cols;
            if (last.vec) ST::flush(buf_h, O, s.cols, wrow0, s.rows, wcol0, s.cols, lane);
            else
#pragma unroll 1
                for (int r0 = 0; r0 < 64; r0 += 16) {         // 16 reads of LDS, then their stores
                    uint16_t v[16];
#pragma unroll
                    for (int r = 0; r < 16; ++r) v[r] = *reinterpret_cast<const uint16_t *>(buf_h + ST::acc_addr(r0 + r, lane & ~3) + (lane & 3) * 2);
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (wrow0 + r0 + r < s.rows && wcol0 + lane < s.cols) O[(size_t)(wrow0 + r0 + r) * s.cols + wcol0 + lane] = v[r];
                }
        }
        wave_lds_fence();
    }
}

template <class... Fs> int raise_lds_limits(int bytes, Fs... kernels)
{
    for (const void *f : {(const void *)kernels...})
        if (hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return RELIBRA_EHIP;
    return RELIBRA_OK;
}

inline unsigned xcd_grid(long long tiles) { return (unsigned)((tiles + 7) / 8 * 8); }

template <class CF> int gram_tiles(int n, int m)
{
    int per_matrix = 0;
    for (int i = 0; i * CF::BB < m; ++i) per_matrix += gram_tiles_of_row<CF>(i);
    return n * per_matrix;
}
struct GramSplit {
    int splits, depth;                           // parts of the contraction, values of each but the last (whole LDS tiles)
    float *part;
};
template <class CF, bool ACROSS, bool POLY, bool MAY_SPLIT = false>
int launch_gram(const uint16_t *p, const float *diag_in, int n, int m, int k, const GramSplit &sp, uint16_t *out, float *diag_out, hipStream_t stream)
{
    static const int limits = raise_lds_limits(CF::LDS, ortho_gram_kernel<CF, ACROSS, POLY>);
    if (limits != RELIBRA_OK) return limits;
    const int per_matrix = gram_tiles<CF>(1, m), tiles = n * per_matrix, total = tiles * sp.splits;
    RELIBRA_LAUNCH(POLY ? RELIBRA_K_ORTHO_POLY : RELIBRA_K_ORTHO_GRAM, stream, (ortho_gram_kernel<CF, ACROSS, POLY>
        <<<xcd_grid(total), CF::THREADS, CF::LDS, stream>>>(p, diag_in, m, k, per_matrix, total, sp.splits, sp.depth, out, diag_out, sp.part)));
    if constexpr (MAY_SPLIT)
        if (sp.splits > 1) {
            RELIBRA_LAUNCH(RELIBRA_K_ORTHO_JOIN, stream, (ortho_join_kernel<CF><<<tiles * CF::WA * CF::WB, 256, 0, stream>>>(sp.part, m, per_matrix, sp.splits, out, diag_out)));
        }
    return RELIBRA_OK;
}
template <class CF, bool TALL>
int launch_update(const OrthoShape &s, const OrthoWs &w, const uint16_t *x, uint16_t *x_out, float weight, const OrthoLast &last, hipStream_t stream)
{
    static const int limits = raise_lds_limits(CF::LDS, ortho_update_kernel<CF, TALL>);
    if (limits != RELIBRA_OK) return limits;
    const int tr = (s.rp + CF::BB - 1) / CF::BB, tc = (s.cp + CF::BA - 1) / CF::BA, total = s.n * tr * tc;
    RELIBRA_LAUNCH(RELIBRA_K_ORTHO_UPDATE, stream, (ortho_update_kernel<CF, TALL><<<xcd_grid(total), CF::THREADS, CF::LDS, stream>>>(
        x, w.lo, w.b, w.db, weight, s, tr, tc, total, x_out, last)));
    return RELIBRA_OK;
}

typedef OrthoCfg<256, 256, 4, 1> OrthoWide;
typedef OrthoCfg<256, 256, 3, 1, BK, 2 * BK> OrthoWideDeep;
typedef OrthoCfg<128, 128, 4, 2> OrthoNarrow;
typedef OrthoCfg<128, 128, 3, 1, 2 * BK> OrthoFew;
typedef OrthoCfg<128, 64, 3, 2, 2 * BK> OrthoFlat;

template <class CF> int update_tiles(const OrthoShape &s) { return s.n * ((s.rp + CF::BB - 1) / CF::BB) * ((s.cp + CF::BA - 1) / CF::BA); }

// Wide tiles where they occupy nearly half of the compute units or more, smaller ones where wide tiles would leave the rest idle.
// us a launch, 256 x 256 / 128 x 128 (wide tiles): A of 4096 x 4096 (136) 88 / 114, of 16 of 768 x 2048 (96) 48 / 40, of 64 of 256 x 512 (64)
// 17.9 / 11.8, of 2048 x 2048 (36) 42 / 23, of 2 of 1000 x 3000 (20) 54 / 27; X' of 16 of 768 x 2048 (384) 74 / 76, of 64 of 256 x 512 (128) 22.3 /
// 22.2, of 2048 x 2048 (64) 47 / 33.  The row operand twice as deep gains the wide X' 2 to 5 % (full lines of B) and costs A 3 %.  Half as
// many rows again (128 x 64) where X' has few tiles: 5 of 1001 x 333 (120 of 128 x 128) 15.3 -> 13.2, 8 of 512 x 512 (128) 13.9 -> 12.7, 2048 x 2048
// (256) 32.9 -> 34.4.
constexpr int kEnoughWideTiles = 112, kFewNarrowTiles = 192;
// Where even the small tiles are no more than the compute units, LDS tiles of twice the depth (half the barriers, a workgroup to
// itself): us a call, 2048 x 2048 375 -> 322, 2 of 1000 x 3000 348 -> 324, 300 x 4000 278 -> 225, level at 8 of 512 x 512; with more tiles the second workgroup of a
// unit is worth more, 16 of 768 x 2048 695 -> 716.  A long contraction of few tiles is split over the idle units besides, parts of
// kMinSplit or a little more, in whole LDS tiles, the last one what is left (2112: three of 576 and one of 384), and joined by a second launch: 300 x 4000 222 -> 168, 4 of 3000 x 200 208 -> 177, 2 of 300 x 2000 176 -> 162, level at 2 of 1000 x
// 3000 and 8 of 200 x 2048; contractions of 1024 that way: 8 of 256 x 1024 140 -> 155, 5 of 1001 x 333 166 -> 182.
constexpr int kMinSplit = 512, kSplitFrom = 2048;
inline GramSplit gram_split(int n, int m, int k)
{
    const int tiles = gram_tiles<OrthoFew>(n, m);
    if (gram_tiles<OrthoWide>(n, m) >= kEnoughWideTiles || k < kSplitFrom || 2 * tiles > kComputeUnits) return GramSplit{1, k, nullptr};
    const int splits = std::min(kComputeUnits / tiles, k / kMinSplit);
    const int depth = ((k + splits - 1) / splits + OrthoFew::ADEPTH - 1) / OrthoFew::ADEPTH * OrthoFew::ADEPTH;
    return GramSplit{(k + depth - 1) / depth, depth, nullptr};
}
inline size_t ortho_split_bytes(const OrthoShape &s)
{
    const int m = s.tall ? s.cp : s.rp, k = s.tall ? s.rp : s.cp;
    const GramSplit sp = gram_split(s.n, m, k);
    return sp.splits > 1 ? round256((size_t)gram_tiles<OrthoFew>(s.n, m) * sp.splits * OrthoFew::BA * OrthoFew::BB * sizeof(float)) : 0;
}

int ortho_steps(const OrthoShape &s, const OrthoWs &w, int steps, float scale, uint16_t *out, hipStream_t stream)
{
    const int m = s.tall ? s.cp : s.rp, k = s.tall ? s.rp : s.cp;
    const bool wide_gram = gram_tiles<OrthoWide>(s.n, m) >= kEnoughWideTiles, wide_update = update_tiles<OrthoWideDeep>(s) >= kEnoughWideTiles;
    const bool few_gram = gram_tiles<OrthoFew>(s.n, m) <= kComputeUnits, flat_update = update_tiles<OrthoNarrow>(s) <= kFewNarrowTiles;
    const GramSplit whole{1, m, nullptr};
    GramSplit split = gram_split(s.n, m, k);
    split.part = w.part;
    auto gram = [&](auto across, auto poly, const uint16_t *p, const float *d, int depth, const GramSplit &sp, uint16_t *out_, float *d_out) {
        constexpr bool AC = decltype(across)::value, PO = decltype(poly)::value;
        return wide_gram ? launch_gram<OrthoWide, AC, PO>(p, d, s.n, m, depth, sp, out_, d_out, stream)
               : few_gram ? launch_gram<OrthoFew, AC, PO, !PO>(p, d, s.n, m, depth, sp, out_, d_out, stream)
                          : launch_gram<OrthoNarrow, AC, PO>(p, d, s.n, m, depth, sp, out_, d_out, stream);
    };
    for (int i = 0; i < steps; ++i) {
        const uint16_t *x = w.x[i & 1];
        uint16_t *x_out = w.x[(i + 1) & 1];
        const float weight = i + 3 >= steps ? 1.0f : 0.0f;
        const OrthoLast last{i + 1 == steps ? out : nullptr, scale, s.cols % 8 == 0 && aligned16(out)};
        auto update = [&](auto tall) {
            constexpr bool T = decltype(tall)::value;
            return wide_update ? launch_update<OrthoWideDeep, T>(s, w, x, x_out, weight, last, stream)
                   : flat_update ? launch_update<OrthoFlat, T>(s, w, x, x_out, weight, last, stream)
                                 : launch_update<OrthoNarrow, T>(s, w, x, x_out, weight, last, stream);
        };
        int rc = s.tall ? gram(std::true_type{}, std::false_type{}, x, nullptr, k, split, w.a, w.da)
                        : gram(std::false_type{}, std::false_type{}, x, nullptr, k, split, w.a, w.da);
        if (rc == RELIBRA_OK) rc = gram(std::false_type{}, std::true_type{}, w.a, w.da, m, whole, w.b, w.db);
        if (rc == RELIBRA_OK) rc = s.tall ? update(std::true_type{}) : update(std::false_type{});
        if (rc != RELIBRA_OK) return rc;
    }
    return RELIBRA_OK;
}

// ---------------------------------------------------------------- thin matrices
// A side of at most 128: A and B fit into a workgroup's LDS, so one launch does a whole step.  The long side is cut into runs of rows,
// `runs` of them to a workgroup; it adds up the workgroups' partial A's, works out B (every workgroup of a matrix does: 128^3 at most),
// multiplies its own rows and takes their share of the next A while they are at hand.  X lies with the long side first whatever the
// gradient's layout, so that every product finds what it needs along memory or through transposing LDS reads; a workgroup alone
// reads and writes its rows, so they are updated in place.  Partial A's travel in accumulator order.  Where one workgroup holds a
// matrix it does all the steps in one launch.  us a call, tiles and 17 launches -> this: 8 of 128 x 256 102 -> 58, 4096 x 128 200 -> 79, 64 x 4096 172 -> 70,
// 128 of 128 x 2048 690 -> 433, 39 of 21 x 2499 238 -> 119.
// 16 waves, one 32 x 32 tile each in every phase: the phases are short chains of LDS round trips and conversions, and with four waves
// of four times the tiles a step of 128 x 128 took 16 us (nothing hides a wave's own latency) where 16 waves took 10.  Bound by LDS reads (products) and
// vector instructions (conversions), 15300 cycles a step: A to halves 1900, A A^T 1400, B to halves 1900, B X 2050, X' 2650, its
// Gram matrix and stores 3200, the rest waits.  Before images took the place of the tiles above the diagonal, and diagonals were taken out by the
// waves that hold one, 19000.
constexpr int kThinSide = 128, kThinWaves = 16, kThinThreads = kThinWaves * 64, kThinBatch = 2;
template <int MP> struct Thin {
    static constexpr int TILES = MP / 32;                    // of a side of A
    static constexpr int SPLIT = kThinWaves / (TILES * TILES);       // waves that share a tile of the rows' Gram matrix, a part of the rows each
    static constexpr int ROWS = kThinWaves / TILES * 32;     // of a run
    static constexpr int KK = MP / 16, AB = MP * MP * 2, STAGE = ROWS * MP * 2, DIAG = 3 * MP * (int)sizeof(float),
                         CARRY = SPLIT > 1 ? kThinWaves * 4096 : 0, LDS = AB + 2 * STAGE + DIAG + CARRY;     // CARRY: the waves' parts of A's tiles
    typedef WaveStage<MP> ST;                    // (row, column) -> place in the A / B buffer and in the staged rows of X
    static constexpr int PIECES = MP / 8, PER_THREAD = ROWS * PIECES / kThinThreads;         // 16-byte pieces of a row, of a run for each thread

    // A run's rows straight to the stage: a wave's 64 pieces fill 1 KiB of consecutive LDS, so each lane fetches the piece whose
    // place is its own.  Not waited for here.
    static __device__ __forceinline__ void request_rows(const uint16_t *rows, char *stage, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) {
            const int first = (i * kThinWaves + wave) * 64, r = (first + lane) / PIECES, piece = ((first + lane) ^ r) & (PIECES - 1);
            load_lds16(rows + (size_t)r * MP + piece * 8, stage + first * 16);
        }
    }

    static __device__ __forceinline__ f32x16_t mfma(bf16x8_t a, bf16x8_t b, f32x16_t c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16_t zero()
    {
        f32x16_t z;
#pragma unroll
        for (int v = 0; v < 16; ++v) z[v] = 0.0f;
        return z;
    }
    static __device__ __forceinline__ bf16x8_t frag(const char *ab, int row0, int kk, int lane)
    {
        return *reinterpret_cast<const bf16x8_t *>(ab + ST::acc_addr(row0 + (lane & 31), kk * 16 + (lane >> 5) * 8));
    }
    // rows contracted over: value k of column c0 + (lane & 31), k = kk * 16 + (lane / 32) * 8 .. + 7, by transposing LDS reads
    static __device__ __forceinline__ bf16x8_t frag_across(const char *stage, int c0, int kk, int lane)
    {
        const int b = lane >> 4, i = lane & 15, c = c0 + (b & 1) * 16 + (i & 3) * 4, r = kk * 16 + (b >> 1) * 8 + (i >> 2);
        const s16x4_t l = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)RELIBRA_LDS(stage + ST::acc_addr(r, c)));
        const s16x4_t h = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t *)RELIBRA_LDS(stage + ST::acc_addr(r + 4, c)));
        return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(l, h, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // Tile of a symmetric matrix -> its place: columns a0 .. in the registers, rows b0 .. on the lanes.  Only tiles with b0 <= a0 are
    // worked out (half the LDS reads, which bound these products: those on the diagonal need one operand); the order of the first TILES leaves
    // no SIMD with more than three of the ten.
    static __device__ __forceinline__ int a_of(int tile) { return tile / TILES * 32; }
    static __device__ __forceinline__ int b_of(int tile) { return (tile + (tile < TILES)) % TILES * 32; }
    static __device__ __forceinline__ bool lower(int tile) { return b_of(tile) <= a_of(tile); }
    // g += this wave's tile of the staged rows' Gram matrix, over its part of the rows
    static __device__ __forceinline__ f32x16_t gram(f32x16_t g, const char *stage, int wave, int lane)
    {
        const int tile = wave / SPLIT, a0 = a_of(tile), b0 = b_of(tile), k0 = wave % SPLIT * (ROWS / SPLIT / 16);
        if (a0 == b0) {
#pragma unroll
            for (int kk = 0; kk < ROWS / SPLIT / 16; ++kk) {
                if (kk % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                const bf16x8_t f = frag_across(stage, a0, k0 + kk, lane);
                g = mfma(f, f, g);
            }
        } else if (b0 < a0) {
#pragma unroll
            for (int kk = 0; kk < ROWS / SPLIT / 16; ++kk) {
                if (kk % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                g = mfma(frag_across(stage, a0, k0 + kk, lane), frag_across(stage, b0, k0 + kk, lane), g);
            }
        }
        return g;
    }
    // The image of a tile below the diagonal that this wave has put into `ab`: read back transposed, 8 values of a column at a time.
    static __device__ __forceinline__ void put_image(char *ab, int a0, int b0, int lane)
    {
        wave_lds_fence();
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
            *reinterpret_cast<bf16x8_t *>(ab + ST::acc_addr(a0 + (lane & 31), b0 + kk * 16 + (lane >> 5) * 8)) = frag_across(ab, a0, b0 / 16 + kk, lane);
    }
    // second halves lie in accumulator order: [32 x 32 tile of the run][4 registers of a lane][lane] of 4 values
    static __device__ __forceinline__ int lo_at(int tile, int q, int lane) { return ((tile * 4 + q) * 64 + lane) * 4; }
    // a partial A: [tile][part of the rows][4 registers of a lane][lane], of which tiles above the diagonal are left out
    static __device__ __forceinline__ size_t part_at(size_t chunk, int tile_and_split, int q, int lane) { return ((chunk * kThinWaves + tile_and_split) * 4 + q) * 64 + lane; }
    static __device__ __forceinline__ void store_part(const f32x16_t &g, float *part, size_t chunk, int wave, int lane)
    {
        if (!lower(wave / SPLIT)) return;
#pragma unroll
        for (int q = 0; q < 4; ++q) reinterpret_cast<float4 *>(part)[part_at(chunk, wave, q, lane)] = make_float4(g[4 * q], g[4 * q + 1], g[4 * q + 2], g[4 * q + 3]);
    }
};
struct ThinShape {
    int n, rows, cols;                           // as the caller gives them
    int mp, run_rows, chunks, runs;              // short side padded to 64 or 128; rows of a run, workgroups of a matrix, runs of each
    bool tall;
    __host__ __device__ int longs() const { return tall ? rows : cols; }
    __host__ __device__ int shorts() const { return tall ? cols : rows; }
    __host__ __device__ size_t x_at(int mat) const { return (size_t)mat * chunks * runs * run_rows * mp; }
};
inline bool is_thin(int rows, int cols) { return std::min(rows, cols) <= kThinSide; }
// One run to a workgroup as far as there are compute units (a workgroup fills one).  Every workgroup of a matrix reads all partial
// A's (40 KiB apiece, two in flight, about 1 us each): of more than kThinDirect, or where the workgroups read more than kThinReads altogether, a
// kernel of its own makes one first.  us a call, without / with it: 128 x 700 (6 workgroups) 67 / 73, 8 of 128 x 700 79 / 81, 32 of 100 x 700 104 / 97,
// 128 x 1000 (8) 72 / 69, 32 of 128 x 500 (4) 79 / 90, 64 of 128 x 500 110 / 106, 16 of 100 x 1000 (8) 97 / 88.
constexpr int kThinDirect = 6, kThinReads = 768;
inline ThinShape thin_shape(int n, int rows, int cols)
{
    ThinShape s{n, rows, cols, 128, Thin<128>::ROWS, 1, 1, rows > cols};
    if (std::min(rows, cols) <= 64) s.mp = 64, s.run_rows = Thin<64>::ROWS;
    const int all = (s.longs() + s.run_rows - 1) / s.run_rows;
    const int chunks = std::max(1, std::min(kComputeUnits / n, all));
    s.runs = (all + chunks - 1) / chunks;
    s.chunks = (all + s.runs - 1) / s.runs;
    return s;
}
inline bool thin_summed(const ThinShape &s) { return s.chunks > kThinDirect || (s.chunks > 1 && s.n * s.chunks * s.chunks > kThinReads); }
struct ThinWs {
    uint16_t *hi, *lo;
    float *part[2], *sum;
    double *parts;
};
inline size_t thin_x_bytes(const ThinShape &s) { return round256(s.x_at(s.n) * sizeof(uint16_t)); }
inline size_t thin_part_bytes(const ThinShape &s) { return round256((size_t)s.n * s.chunks * kThinWaves * 1024 * sizeof(float)); }

inline size_t thin_sum_bytes(const ThinShape &s) { return thin_summed(s) ? round256((size_t)s.n * kThinWaves * 1024 * sizeof(float)) : 0; }

// Rows of a run, 8 values of the short side at a time, lanes along the memory of the caller's matrix: fn(row of the run, first value).
template <int MP, int UNROLL, class Fn> __device__ __forceinline__ void thin_pieces(bool tall, int tid, const Fn &fn)
{
    constexpr int PIECES = Thin<MP>::PIECES, ROWS = Thin<MP>::ROWS;
#pragma unroll UNROLL
    for (int p = tid; p < ROWS * PIECES; p += kThinThreads) {
        if (tall) fn(p / PIECES, p % PIECES * 8);
        else fn(p % ROWS, p / ROWS * 8);
    }
}

// First halves of a workgroup's rows and their partial A.
template <class GT, int MP>
__global__ void __launch_bounds__(kThinThreads)
ortho_thin_load_kernel(const GT *__restrict__ g, const float *__restrict__ m_new, float mu, int mode, ThinShape s, const double *__restrict__ parts, int n_parts,
                       uint16_t *__restrict__ hi, uint16_t *__restrict__ lo, float *__restrict__ part)
{
    using TH = Thin<MP>;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    __shared__ double scale_of;
    int tid = threadIdx.x;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), mat = blockIdx.y;
    if (tid < 64) {
        double sum = 0.0;
        for (int i = tid; i < n_parts; i += 64) sum += parts[(size_t)mat * n_parts + i];
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
        if (tid == 0) scale_of = sum == 0.0 ? 0.0 : (double)kScale / sqrt(sum);
    }
    __syncthreads();
    const double scale = scale_of;
    const size_t from = (size_t)mat * s.rows * s.cols;
    const int longs = s.longs(), shorts = s.shorts();
    f32x16_t acc = TH::zero();
    for (int run = 0; run < s.runs; ++run) {
        const int row0 = (blockIdx.x * s.runs + run) * TH::ROWS;
        asm volatile("" : "+v"(tid));                         // (opaque: else the addresses of a run are kept in registers from run to run)
        thin_pieces<MP, 2>(s.tall, tid, [&](int i, int j0) __attribute__((always_inline)) {
            const int li = row0 + i;
            float gv[8] = {}, mv[8] = {};
            if (s.tall && li < longs && j0 + 8 <= shorts) {
                const size_t at = from + (size_t)li * s.cols + j0;
                if (mode != U_MOMENTUM) unpack8(fetch8_any(g + at), gv);
                if (mode != U_GRAD) unpack8(fetch8_any(m_new + at), mv);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (li < longs && j0 + j < shorts) {
                        const size_t at = from + (s.tall ? (size_t)li * s.cols + j0 + j : (size_t)(j0 + j) * s.cols + li);
                        if (mode != U_MOMENTUM) gv[j] = to_f32(g[at]);
                        if (mode != U_GRAD) mv[j] = m_new[at];
                    }
            }
            uint16_t h8[8], l8[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = li < longs && j0 + j < shorts;
                const float u = in ? (float)((double)update_of(gv[j], mv[j], mu, mode) * scale) : 0.0f;
                const _Float16 h = (_Float16)u;
                h8[j] = __builtin_bit_cast(uint16_t, h);
                l8[j] = __builtin_bit_cast(uint16_t, (_Float16)(u - (float)h));
            }
            *reinterpret_cast<uint4 *>(hi + s.x_at(mat) + (size_t)li * MP + j0) = *reinterpret_cast<const uint4 *>(h8);
            uint16_t *l = lo + s.x_at(mat) + (size_t)row0 * MP + TH::lo_at(i / 32 * TH::TILES + j0 / 32, j0 % 32 / 8, i % 32);
            *reinterpret_cast<uint2 *>(l) = *reinterpret_cast<const uint2 *>(l8);
            *reinterpret_cast<uint2 *>(l + 32 * 4) = *reinterpret_cast<const uint2 *>(l8 + 4);
            *reinterpret_cast<uint4 *>(lds + TH::ST::acc_addr(i, j0)) = *reinterpret_cast<const uint4 *>(h8);
        });
        __syncthreads();
        acc = TH::gram(acc, lds, wave, lane);
        __syncthreads();
    }
    TH::store_part(acc, part, (size_t)mat * s.chunks + blockIdx.x, wave, lane);
}

// One partial A of a matrix from those of its workgroups, in ascending order: blockIdx.x of kThinWaves blocks of 1024 values.
template <int MP>
__global__ void __launch_bounds__(256)
ortho_thin_sum_kernel(const float4 *__restrict__ part, int chunks, float4 *__restrict__ sum)
{
    if (!Thin<MP>::lower(blockIdx.x / Thin<MP>::SPLIT)) return;
    const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x, base = (size_t)blockIdx.y * chunks * kThinWaves * 256 + at;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int c = 0; c < chunks; ++c) {
        const float4 v = part[base + (size_t)c * kThinWaves * 256];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    sum[(size_t)blockIdx.y * kThinWaves * 256 + at] = s;
}

__device__ __forceinline__ void add4(f32x16_t &to, int q, const float4 &v)
{
    to[4 * q] += v.x;
    to[4 * q + 1] += v.y;
    to[4 * q + 2] += v.z;
    to[4 * q + 3] += v.w;
}

// Of a 32 x 32 accumulator tile on the diagonal: whether the lane holds one of its elements, and that element, with 0 left in its place.
__device__ __forceinline__ bool holds_diagonal(int lane) { return ((lane >> 2) & 1) == lane >> 5; }
__device__ __forceinline__ float take_diagonal(f32x16_t &v, int lane)
{
    const int at = (lane & 31) - (lane >> 5) * 4;
    float d = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const bool here = at == i / 4 * 8 + i % 4;
        d = here ? v[i] : d;
        v[i] = here ? 0.0f : v[i];
    }
    return d;
}

// Steps first .. first + count - 1 of `steps` (count > 1 with one workgroup a matrix only).
template <int MP>
__global__ void __launch_bounds__(kThinThreads)
ortho_thin_step_kernel(ThinShape s, int first, int count, int steps, uint16_t *hi, uint16_t *lo, const float *__restrict__ part_in, int n_in,
                       float *__restrict__ part_out, float out_scale, int vec,
                       uint16_t *__restrict__ out)
{
    using TH = Thin<MP>;
    using ST = typename TH::ST;
    constexpr int KK = TH::KK, TILES = TH::TILES, SPLIT = TH::SPLIT;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    char *ab = lds;
    float *da = reinterpret_cast<float *>(lds + TH::AB + 2 * TH::STAGE), *hi_by = da + MP, *lo_by = hi_by + MP;     // diagonal of A; a + d and a + w d, d that of B
    float4 *carry = reinterpret_cast<float4 *>(lds + TH::AB + 2 * TH::STAGE + TH::DIAG);
    f32x16_t acc = TH::zero();                                // this wave's tile of the next A over the workgroup's rows
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), mat = blockIdx.y;
    // this wave's tile of A and B (those of the first TILES^2 waves that have one) and of a run's rows of X
    const bool has_tile = wave < TILES * TILES && TH::lower(wave);
    const int a0 = TH::a_of(wave), b0 = TH::b_of(wave), x_col = wave % TILES * 32;
    for (int step = first; step < first + count; ++step) {
        const float w = step + 3 >= steps ? 1.0f : 0.0f;
        const bool last = step + 1 == steps;
        int lane = tid & 63, cols = s.cols;                   // (opaque: else every address of a step is kept in registers through all steps)
        asm volatile("" : "+v"(lane), "+s"(cols));
        const int r_ab = b0 + (lane & 31), half = (lane >> 5) * 4;
        // the first run's rows are on their way while A and B are worked out, the next one's while a run is finished
        uint2 lv[4];
        auto fetch = [&](int run, int t) __attribute__((always_inline)) {
            const size_t at_run = s.x_at(mat) + (size_t)(blockIdx.x * s.runs + run) * TH::ROWS * MP;
            TH::request_rows(hi + at_run, lds + TH::AB + (run & 1) * TH::STAGE, wave, t & 63);
#pragma unroll
            for (int q = 0; q < 4; ++q) lv[q] = *reinterpret_cast<const uint2 *>(lo + at_run + TH::lo_at(wave, q, t & 63));
        };
        fetch(0, tid);
        // A: every wave adds up its part over the workgroups of the matrix, in ascending order, several at a time so that a memory
        // round trip is paid once for all; the parts of a tile meet in LDS
        if (step == first) {
            const float4 *src = reinterpret_cast<const float4 *>(part_in);
            acc = TH::zero();
#pragma unroll 1
            for (int c0 = 0; TH::lower(wave / SPLIT) && c0 < n_in; c0 += kThinBatch) {
                float4 v[kThinBatch][4];
#pragma unroll
                for (int u = 0; u < kThinBatch; ++u)
                    if (c0 + u < n_in)
#pragma unroll
                        for (int q = 0; q < 4; ++q) v[u][q] = src[TH::part_at((size_t)mat * n_in + c0 + u, wave, q, lane)];
#pragma unroll
                for (int u = 0; u < kThinBatch; ++u)
                    if (c0 + u < n_in)
#pragma unroll
                        for (int q = 0; q < 4; ++q) add4(acc, q, v[u][q]);
            }
        }
        if (SPLIT > 1) {
#pragma unroll
            for (int q = 0; q < 4; ++q) carry[TH::part_at(0, wave, q, lane)] = make_float4(acc[4 * q], acc[4 * q + 1], acc[4 * q + 2], acc[4 * q + 3]);
            __syncthreads();
        }
        uint2 at[4];
        if (has_tile) {
            f32x16_t sum = SPLIT > 1 ? TH::zero() : acc;
            if (SPLIT > 1)
#pragma unroll
                for (int c = 0; c < SPLIT; ++c)
#pragma unroll
                    for (int q = 0; q < 4; ++q) add4(sum, q, carry[TH::part_at(0, wave * SPLIT + c, q, lane)]);
            // A: its diagonal apart, the rest as halves
#pragma unroll
            for (int i = 0; i < 16; ++i) sum[i] *= 1.0f / kScale;
            if (a0 == b0) {
                const float d = take_diagonal(sum, lane);
                if (holds_diagonal(lane)) da[r_ab] = d;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float v[4] = {sum[4 * q], sum[4 * q + 1], sum[4 * q + 2], sum[4 * q + 3]};
                at[q] = pack4h(v);
                ST::put(ab, r_ab, a0 + q * 8 + half, at[q]);
            }
            if (b0 < a0) TH::put_image(ab, a0, b0, lane);
        }
        __syncthreads();
        f32x16_t p = TH::zero();
        if (has_tile && a0 == b0) {
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                if (kk % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                const bf16x8_t f = TH::frag(ab, a0, kk, lane);
                p = TH::mfma(f, f, p);
            }
        } else if (has_tile) {
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                if (kk % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                p = TH::mfma(TH::frag(ab, a0, kk, lane), TH::frag(ab, b0, kk, lane), p);
            }
        }
        __syncthreads();                                      // A has been read: B takes its place
        if (has_tile) {
            const float d_r = da[r_ab], by_r = fmaf(kNsC / kScale, d_r, kNsB);
            if (a0 == b0) {
                const float d = (kNsB * d_r + (kNsC / kScale) * (take_diagonal(p, lane) + d_r * d_r)) * (1.0f / kScale);
                if (holds_diagonal(lane)) {
                    hi_by[r_ab] = kNsA + d;
                    lo_by[r_ab] = kNsA + w * d;
                }
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {                     // (on the diagonal both p and the half of A are 0 by now)
                const int c = a0 + q * 8 + half;
                const float4 d_c = *reinterpret_cast<const float4 *>(da + c);
                const float dc[4] = {d_c.x, d_c.y, d_c.z, d_c.w};
                float old[4], v[4];
                unpack4h(at[q], old);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = fmaf(fmaf(kNsC / kScale, dc[e], by_r), old[e], (kNsC / kScale) * p[4 * q + e]);
                ST::put(ab, r_ab, c, pack4h(v));
            }
            if (b0 < a0) TH::put_image(ab, a0, b0, lane);
        }
        __syncthreads();
        acc = TH::zero();
        for (int run = 0; run < s.runs; ++run) {
            const int row0 = (blockIdx.x * s.runs + run) * TH::ROWS;
            int t = tid;
            asm volatile("" : "+v"(t), "+s"(cols));
            const int lane = t & 63, half = (lane >> 5) * 4, x_row = wave / TILES * 32 + (lane & 31);
            const size_t at_run = s.x_at(mat) + (size_t)row0 * MP;
            char *stage = lds + TH::AB + (run & 1) * TH::STAGE;
            wait_vm_lgkm0<0>();                               // this wave's share of the rows is there
            __syncthreads();
            f32x16_t x = TH::zero();
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                if (kk % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                x = TH::mfma(TH::frag(ab, x_col, kk, lane), TH::frag(stage, wave / TILES * 32, kk, lane), x);
            }
            uint2 h_now[4], l_now[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                h_now[q] = ST::get(stage, x_row, x_col + q * 8 + half);
                l_now[q] = lv[q];
            }
            __syncthreads();                                  // the rows have been read: X' takes their place
            if (run + 1 < s.runs) fetch(run + 1, t);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = x_col + q * 8 + half;
                const float4 bh = *reinterpret_cast<const float4 *>(hi_by + c), bl = *reinterpret_cast<const float4 *>(lo_by + c);
                const float by_h[4] = {bh.x, bh.y, bh.z, bh.w}, by_l[4] = {bl.x, bl.y, bl.z, bl.w};
                float h[4], l[4], v[4];
                unpack4h(h_now[q], h);
                unpack4h(l_now[q], l);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = fmaf(by_h[e], h[e], fmaf(by_l[e], l[e], x[4 * q + e] * (1.0f / kScale)));
                uint2 hp = pack4h(v);
                if (!last) {
                    unpack4h(hp, h);
#pragma unroll
                    for (int e = 0; e < 4; ++e) l[e] = v[e] - h[e];
                    *reinterpret_cast<uint2 *>(lo + at_run + TH::lo_at(wave, q, lane)) = pack4h(l);
                } else {
                    const float f = out_scale * (1.0f / kScale);
                    hp = make_uint2(pack2bf(f * v[0], f * v[1]), pack2bf(f * v[2], f * v[3]));
                }
                ST::put(stage, x_row, c, hp);
            }
            __syncthreads();
            if (!last) {
#pragma unroll
                for (int i = 0; i < TH::PER_THREAD; ++i) {
                    const int p = i * kThinThreads + t;
                    reinterpret_cast<uint4 *>(hi + at_run)[p] = *reinterpret_cast<const uint4 *>(stage + ST::acc_addr(p / TH::PIECES, p % TH::PIECES * 8));
                }
                acc = TH::gram(acc, stage, wave, lane);
            } else {
                uint16_t *o = out + (size_t)mat * s.rows * s.cols;
                thin_pieces<MP, 1>(s.tall, t, [&](int i, int j0) __attribute__((always_inline)) {
                    if (row0 + i >= s.longs() || j0 >= s.shorts()) return;
                    uint16_t v[8];
                    *reinterpret_cast<uint4 *>(v) = *reinterpret_cast<const uint4 *>(stage + ST::acc_addr(i, j0));
                    if (s.tall && vec) *reinterpret_cast<uint4 *>(o + (size_t)(row0 + i) * cols + j0) = *reinterpret_cast<const uint4 *>(v);
                    else
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (j0 + j < s.shorts()) o[s.tall ? (size_t)(row0 + i) * cols + j0 + j : (size_t)(j0 + j) * cols + row0 + i] = v[j];
                });
            }
            __syncthreads();                                  // the stage is free for the run after the next
        }
        if (step + 1 < first + count) {                       // one workgroup holds the matrix: the next A stays here
            wait_vm_lgkm0<0>();
            __syncthreads();                                  // the rows are where the next step finds them; B has been read
        } else if (!last) TH::store_part(acc, part_out, (size_t)mat * s.chunks + blockIdx.x, wave, lane);
    }
}

template <class GT, int MP>
int thin_run(const ThinShape &s, const ThinWs &w, const GT *g, const float *m_new, float mu, int mode, int n_parts, int steps, float scale, uint16_t *out,
             hipStream_t stream)
{
    using TH = Thin<MP>;
    static const int limits = raise_lds_limits(TH::LDS, ortho_thin_load_kernel<GT, MP>, ortho_thin_step_kernel<MP>);
    if (limits != RELIBRA_OK) return limits;
    const dim3 grid(s.chunks, s.n);
    RELIBRA_LAUNCH(RELIBRA_K_ORTHO_LOAD, stream, (ortho_thin_load_kernel<GT, MP><<<grid, kThinThreads, TH::STAGE, stream>>>(
        g, m_new, mu, mode, s, w.parts, n_parts, w.hi, w.lo, w.part[0])));
    const int each = s.chunks == 1 ? steps : 1, vec = s.cols % 8 == 0 && aligned16(out);
    for (int i = 0; i < steps; i += each) {
        const bool summed = thin_summed(s);
        if (summed) RELIBRA_LAUNCH(RELIBRA_K_ORTHO_POLY, stream, ortho_thin_sum_kernel<MP><<<dim3(kThinWaves, s.n), 256, 0, stream>>>(
            (const float4 *)w.part[i & 1], s.chunks, (float4 *)w.sum));
        RELIBRA_LAUNCH(RELIBRA_K_ORTHO_THIN, stream, (ortho_thin_step_kernel<MP><<<grid, kThinThreads, TH::LDS, stream>>>(
            s, i, each, steps, w.hi, w.lo, summed ? w.sum : w.part[i & 1], summed ? 1 : s.chunks, w.part[(i + 1) & 1], scale, vec, out)));
    }
    return RELIBRA_OK;
}

// (2^30 tiles of 64 x 64: tile numbers are ints)
inline bool ortho_takes(int n, int rows, int cols)
{
    return n <= 65535 && rows <= kOrthoMaxSide && cols <= kOrthoMaxSide && (long long)n * ((rows + 63) / 64) * ((cols + 63) / 64) < 1 << 30;
}
size_t ortho_ws_bytes(int n, int rows, int cols)
{
    if (rows < 1 || cols < 1 || !ortho_takes(n, rows, cols)) return 0;
    const size_t parts = round256((size_t)n * norm_parts(n, rows, cols) * sizeof(double));
    if (is_thin(rows, cols)) {
        const ThinShape s = thin_shape(n, rows, cols);
        return parts + 2 * thin_x_bytes(s) + 2 * thin_part_bytes(s) + thin_sum_bytes(s);
    }
    const OrthoShape s = ortho_shape(n, rows, cols);
    return parts + 3 * ortho_x_bytes(s) + 2 * ortho_gram_bytes(s) + 2 * ortho_diag_bytes(s) + ortho_split_bytes(s);
}

template <class GT>
int ortho_run(int n, int rows, int cols, const GT *g, const float *m, float mu, float scale, int steps, int mode, float *m_out, uint16_t *out, char *ws, hipStream_t stream)
{
    const size_t per_matrix = (size_t)rows * cols;
    const int n_parts = norm_parts(n, rows, cols);
    double *parts = (double *)ws;
    ws += round256((size_t)n * n_parts * sizeof(double));
    RELIBRA_LAUNCH(RELIBRA_K_ORTHO_NORM, stream, ortho_momentum_kernel<GT><<<dim3(n_parts, n), 256, 0, stream>>>(
        g, m, mu, mode, per_matrix, m_out, parts));
    if (is_thin(rows, cols)) {
        const ThinShape s = thin_shape(n, rows, cols);
        ThinWs w;
        w.parts = parts;
        w.hi = (uint16_t *)ws;
        w.lo = (uint16_t *)(ws += thin_x_bytes(s));
        w.part[0] = (float *)(ws += thin_x_bytes(s));
        w.part[1] = (float *)(ws += thin_part_bytes(s));
        w.sum = (float *)(ws + thin_part_bytes(s));
        return s.mp == 64 ? thin_run<GT, 64>(s, w, g, m_out, mu, mode, n_parts, steps, scale, out, stream)
                          : thin_run<GT, 128>(s, w, g, m_out, mu, mode, n_parts, steps, scale, out, stream);
    }
    const OrthoShape s = ortho_shape(n, rows, cols);
    OrthoWs w;
    w.x[0] = (uint16_t *)ws;
    w.x[1] = (uint16_t *)(ws += ortho_x_bytes(s));
    w.lo = (uint16_t *)(ws += ortho_x_bytes(s));
    w.a = (uint16_t *)(ws += ortho_x_bytes(s));
    w.b = (uint16_t *)(ws += ortho_gram_bytes(s));
    w.da = (float *)(ws += ortho_gram_bytes(s));
    w.db = (float *)(ws += ortho_diag_bytes(s));
    w.part = (float *)(ws + ortho_diag_bytes(s));
    const unsigned pieces = (unsigned)((size_t)s.rp * s.cp / 8), blocks = std::min((pieces + 255) / 256, std::max(32u, (4096u + n - 1) / n));
    RELIBRA_LAUNCH(RELIBRA_K_ORTHO_LOAD, stream, ortho_load_kernel<GT><<<dim3(blocks, n), 256, 0, stream>>>(
        g, m_out, mu, mode, s, parts, n_parts, w.x[0], w.lo));
    return ortho_steps(s, w, steps, scale, out, stream);
}

}  // namespace relibra

using namespace relibra;

extern "C" int relibra_orthogonalize(const void *grad, const float *momentum, int n, int rows, int cols, float mu, float scale, int steps, int flags,
                                     float *momentum_out, void *out, void *workspace, size_t workspace_bytes, relibra_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    if (n < 0 || rows < 0 || cols < 0 || steps < 1 || (flags & ~(RELIBRA_ORTHO_BF16 | RELIBRA_ORTHO_NESTEROV))) return RELIBRA_EINVAL;
    if (!ortho_takes(n, rows, cols) || steps > kOrthoMaxSteps) return RELIBRA_EUNSUPPORTED;
    if ((momentum != nullptr) != (momentum_out != nullptr) || (!momentum && (flags & RELIBRA_ORTHO_NESTEROV))) return RELIBRA_EINVAL;
    if (n == 0 || rows == 0 || cols == 0) return RELIBRA_OK;
    if (!grad || !out) return RELIBRA_EINVAL;
    if (!workspace || workspace_bytes < ortho_ws_bytes(n, rows, cols)) return RELIBRA_EWORKSPACE;
    if (!aligned16(workspace)) return RELIBRA_EINVAL;
    // a momentum written over the gradient would be read as the gradient by the pass that divides by the norm
    const size_t halves = (size_t)n * rows * cols * 2, floats = 2 * halves, grad_bytes = flags & RELIBRA_ORTHO_BF16 ? halves : floats;
    if (overlap(out, halves, grad, grad_bytes)) return RELIBRA_EINVAL;
    if (momentum && (overlap(out, halves, momentum, floats) || overlap(out, halves, momentum_out, floats) || overlap(momentum_out, floats, grad, grad_bytes) ||
                     (momentum_out != momentum && overlap(momentum_out, floats, momentum, floats)))) return RELIBRA_EINVAL;
    const int mode = !momentum ? U_GRAD : flags & RELIBRA_ORTHO_NESTEROV ? U_NESTEROV : U_MOMENTUM;
    const int rc = flags & RELIBRA_ORTHO_BF16
                       ? ortho_run(n, rows, cols, (const bf16_t *)grad, momentum, mu, scale, steps, mode, momentum_out, (uint16_t *)out, (char *)workspace, stream)
                       : ortho_run(n, rows, cols, (const float *)grad, momentum, mu, scale, steps, mode, momentum_out, (uint16_t *)out, (char *)workspace, stream);
    if (rc != RELIBRA_OK) return rc;
    RELIBRA_HIP_TRY(launch_check());
    return RELIBRA_OK;
}
