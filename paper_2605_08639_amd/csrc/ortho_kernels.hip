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

typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));

struct OrthoShape {
    int n, rows, cols;                           // matrices, as the caller gives them
    int rp, cp;                                  // padded
    bool tall;                                   // rows > cols
};
// Workspace: two copies of X's first halves (a step reads one and writes the other), the second halves, A, B, their diagonals, partial sums.
struct OrthoWs {
    uint16_t *x[2], *lo, *a, *b;
    float *da, *db;
    double *parts;
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
// Blocks that share a matrix's squares: 2048 over all matrices, each with at least 4096 values.  With 64 a matrix one of
// 4096 x 4096 took 197 us (0.25 of the copy rate).
inline int norm_parts(const OrthoShape &s)
{
    const size_t values = (size_t)s.rows * s.cols;
    return (int)std::min<size_t>(std::max<size_t>(std::min<size_t>((2048 + s.n - 1) / s.n, values / 4096), kMinParts), kMaxParts);
}
size_t ortho_ws_bytes(int n, int rows, int cols)
{
    const OrthoShape s = ortho_shape(n, rows, cols);
    return 3 * ortho_x_bytes(s) + 2 * ortho_gram_bytes(s) + 2 * ortho_diag_bytes(s) + round256((size_t)n * norm_parts(s) * sizeof(double));
}

// ---------------------------------------------------------------- momentum, norm, first halves
enum { U_GRAD = 0, U_MOMENTUM = 1, U_NESTEROV = 2 };
__device__ __forceinline__ float update_of(float g, float m_new, float mu, int mode)
{
    return mode == U_GRAD ? g : mode == U_MOMENTUM ? m_new : fmaf(mu, m_new, g);
}

// M' and the sum of U^2, part blockIdx.x of matrix blockIdx.y.  Squares in double: no gradient is too large or small.
// vec: elements per matrix and all pointers allow 16-byte accesses (four fp32 or eight bytes of bf16 at a time).
template <class GT>
__global__ void __launch_bounds__(256)
ortho_momentum_kernel(const GT *__restrict__ g, const float *m, float mu, int mode, size_t per_matrix, int vec, float *m_out, double *__restrict__ parts)
{
    __shared__ double red[4];
    const size_t base = (size_t)blockIdx.y * per_matrix;
    double sum = 0.0;
    auto one = [&](GT gv, float mv) __attribute__((always_inline)) {
        const float mn = mode == U_GRAD ? 0.0f : fmaf(mu, mv, to_f32(gv));
        const double u = update_of(to_f32(gv), mn, mu, mode);
        sum += u * u;
        return mn;
    };
    if (vec) {
        const size_t quads = per_matrix / 4, stride = (size_t)gridDim.x * 256;
        for (size_t q = (size_t)blockIdx.x * 256 + threadIdx.x; q < quads; q += stride) {
            GT gv[4];
            if constexpr (sizeof(GT) == 4) *reinterpret_cast<float4 *>(gv) = *reinterpret_cast<const float4 *>(g + base + q * 4);
            else *reinterpret_cast<uint2 *>(gv) = *reinterpret_cast<const uint2 *>(g + base + q * 4);
            float4 mv = make_float4(0.f, 0.f, 0.f, 0.f);
            if (mode != U_GRAD) mv = *reinterpret_cast<const float4 *>(m + base + q * 4);
            const float4 mn = make_float4(one(gv[0], mv.x), one(gv[1], mv.y), one(gv[2], mv.z), one(gv[3], mv.w));
            if (mode != U_GRAD) *reinterpret_cast<float4 *>(m_out + base + q * 4) = mn;
        }
    } else {
        for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < per_matrix; i += (size_t)gridDim.x * 256) {
            const float mn = one(g[base + i], mode != U_GRAD ? m[base + i] : 0.0f);
            if (mode != U_GRAD) m_out[base + i] = mn;
        }
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) parts[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// X = kScale U / |U| as two halves, padding included.  A thread takes 8 consecutive padded columns of a row.
template <class GT>
__global__ void __launch_bounds__(256)
ortho_load_kernel(const GT *__restrict__ g, const float *__restrict__ m_new, float mu, int mode, OrthoShape s, int vec, const double *__restrict__ parts,
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
    const size_t pieces = (size_t)s.rp * per_row;
    const size_t from = (size_t)b * s.rows * s.cols, to = (size_t)b * s.rp * s.cp;
    for (size_t p = (size_t)blockIdx.x * 256 + threadIdx.x; p < pieces; p += (size_t)gridDim.x * 256) {
        const int r = (int)(p / per_row), c = (int)(p % per_row) * 8;
        float gv[8] = {}, mv[8] = {}, u[8];
        const size_t at = from + (size_t)r * s.cols + c;
        const bool whole = vec && r < s.rows && c < s.cols;          // cols % 8 == 0 then
        if (whole) {
            if (mode != U_MOMENTUM) load8(g + at, gv);
            if (mode != U_GRAD) load8(m_new + at, mv);
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
// A tile has BB rows (on the lanes) and BA columns (in the accumulator registers); a wave owns 64 rows and BA / WA_ columns.
template <int BA_, int BB_, int STAGES_, int OCC_, bool DEEP_ = false, int WA_ = 2> struct OrthoCfg {
    static constexpr int BA = BA_, BB = BB_, WA = WA_, WB = BB / 64, THREADS = WA * WB * 64, STAGES = STAGES_;
    static constexpr int COLS = BA / WA;                             // of a wave
    static constexpr int BDEPTH = DEEP_ ? 2 * BK : BK;               // of the row operand's LDS tiles
    static constexpr int WAVES_PER_SIMD = OCC_ * WA * WB / 4;        // OCC_: workgroups per compute unit
    static constexpr int SLABS = STAGES * (BA + (DEEP_ ? 0 : BB)) * BK * 2 + (DEEP_ ? (STAGES + 3) / 2 * BB * BDEPTH * 2 : 0);
    static constexpr int STAGING = WA * WB * 2 * WaveStage<64>::BYTES;
    static constexpr int LDS = SLABS > STAGING ? SLABS : STAGING;
    template <class AT> using Loop = KLoop<AT, KcTile<BB, BDEPTH>, 1, 1, BA, BB, WA, WB, 1, false, STAGES, true, false, false, true>;
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
template <class CF, bool ACROSS, bool POLY>
__global__ void __launch_bounds__(CF::THREADS, CF::WAVES_PER_SIMD)
ortho_gram_kernel(const uint16_t *__restrict__ p, const float *__restrict__ diag_in, int m, int k, int per_matrix, int total, uint16_t *__restrict__ out,
                  float *__restrict__ diag_out)
{
    using KL = typename std::conditional<ACROSS, KLoop<KsTile<CF::BA>, KsTile<CF::BB>, 1, 1, CF::BA, CF::BB, CF::WA, CF::WB, 1, false, CF::STAGES, true, false, false, true>,
                                         typename CF::template Loop<KcTile<CF::BA>>>::type;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int t = xcd_tile(blockIdx.x, total);
    if (t < 0) return;
    const int mat = t / per_matrix;
    int i = 0, j = t % per_matrix;
    while (j >= gram_tiles_of_row<CF>(i)) j -= gram_tiles_of_row<CF>(i++);
    const uint16_t *src = p + (size_t)mat * m * k;
    uint16_t *dst = out + (size_t)mat * m * m;
    const int ld = ACROSS ? m : k, row0 = i * CF::BB, col0 = j * CF::BA;
    const Operand A[1][1] = {{{src, ld, col0, m - 1}}}, B[1][1] = {{{src, ld, row0, m - 1}}};
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    typename KL::Acc acc;
    KL::zero(acc);
    KL::run(acc, A, B, k / BK, k, lds, tid);
    __syncthreads();                                          // every wave is done with the operand slabs
    using ST = WaveStage<64>;
    char *buf = lds + wave * 2 * ST::BYTES;
    const int wrow0 = row0 + (wave % CF::WB) * 64;
#pragma unroll
    for (int half = 0; half < CF::COLS / 64; ++half) {
        const int wcol0 = col0 + (wave / CF::WB) * CF::COLS + half * 64;
        if (wrow0 >= m || wcol0 > wrow0) break;               // uniform in the wave; padding is in whole runs of 64
        const float *din = diag_in + (size_t)mat * m;
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
                        const float s = acc[0][half * 2 + ta][tb][q * 4 + e];
                        v[e] = POLY ? kNsB * old[e] + (kNsC / kScale) * (s + (d_r[tb] + d_c[ta][q][e]) * old[e]) : s * (1.0f / kScale);
                        if (wrow0 == wcol0 && r == c + e) {
                            diag_out[(size_t)mat * m + wrow0 + r] = POLY ? kNsB * d_r[tb] + (kNsC / kScale) * (s + d_r[tb] * d_r[tb]) : v[e];
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
    using KL = typename CF::template Loop<typename std::conditional<TALL, KcTile<CF::BA>, KsTile<CF::BA>>::type>;
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
    KL::run(acc, A, B, m / BK, m, lds, tid);
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
                for (int r = 0; r < 64 && wrow0 + r < s.rows; ++r)
                    if (wcol0 + lane < s.cols)
                        O[(size_t)(wrow0 + r) * s.cols + wcol0 + lane] = *reinterpret_cast<const uint16_t *>(buf_h + ST::acc_addr(r, lane & ~3) + (lane & 3) * 2);
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
template <class CF, bool ACROSS, bool POLY>
int launch_gram(const uint16_t *p, const float *diag_in, int n, int m, int k, uint16_t *out, float *diag_out, hipStream_t stream)
{
    static const int limits = raise_lds_limits(CF::LDS, ortho_gram_kernel<CF, ACROSS, POLY>);
    if (limits != RELIBRA_OK) return limits;
    const int per_matrix = gram_tiles<CF>(1, m);
    RELIBRA_LAUNCH(POLY ? RELIBRA_K_ORTHO_POLY : RELIBRA_K_ORTHO_GRAM, stream, (ortho_gram_kernel<CF, ACROSS, POLY>
        <<<xcd_grid((long long)n * per_matrix), CF::THREADS, CF::LDS, stream>>>(p, diag_in, m, k, per_matrix, n * per_matrix, out, diag_out)));
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
typedef OrthoCfg<256, 256, 3, 1, true> OrthoWideDeep;
typedef OrthoCfg<128, 128, 4, 2> OrthoNarrow;
typedef OrthoCfg<128, 64, 4, 2> OrthoFlat;

template <class CF> int update_tiles(const OrthoShape &s) { return s.n * ((s.rp + CF::BB - 1) / CF::BB) * ((s.cp + CF::BA - 1) / CF::BA); }

// Wide tiles where they occupy nearly half of the compute units or more, smaller ones where wide tiles would leave the rest idle.
// us a launch, 256 x 256 / 128 x 128 (wide tiles): A of 4096 x 4096 (136) 88 / 114, of 16 of 768 x 2048 (96) 48 / 40, of 64 of 256 x 512 (64)
// 17.9 / 11.8, of 2048 x 2048 (36) 42 / 23, of 2 of 1000 x 3000 (20) 54 / 27; X' of 16 of 768 x 2048 (384) 74 / 76, of 64 of 256 x 512 (128) 22.3 /
// 22.2, of 2048 x 2048 (64) 47 / 33.  The row operand twice as deep gains the wide X' 2 to 5 % (full lines of B) and costs A 3 %.  Half as
// many rows again (128 x 64) where X' has few tiles: 5 of 1001 x 333 (120 of 128 x 128) 15.3 -> 13.2, 8 of 512 x 512 (128) 13.9 -> 12.7, 2048 x 2048
// (256) 32.9 -> 34.4.
constexpr int kEnoughWideTiles = 112, kFewNarrowTiles = 192;

int ortho_steps(const OrthoShape &s, const OrthoWs &w, int steps, float scale, uint16_t *out, hipStream_t stream)
{
    const int m = s.tall ? s.cp : s.rp, k = s.tall ? s.rp : s.cp;
    const bool wide_gram = gram_tiles<OrthoWide>(s.n, m) >= kEnoughWideTiles, wide_update = update_tiles<OrthoWideDeep>(s) >= kEnoughWideTiles;
    const bool flat_update = update_tiles<OrthoNarrow>(s) <= kFewNarrowTiles;
    auto gram = [&](auto across, auto poly, const uint16_t *p, const float *d, int depth, uint16_t *out_, float *d_out) {
        return wide_gram ? launch_gram<OrthoWide, decltype(across)::value, decltype(poly)::value>(p, d, s.n, m, depth, out_, d_out, stream)
                         : launch_gram<OrthoNarrow, decltype(across)::value, decltype(poly)::value>(p, d, s.n, m, depth, out_, d_out, stream);
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
        int rc = s.tall ? gram(std::true_type{}, std::false_type{}, x, nullptr, k, w.a, w.da) : gram(std::false_type{}, std::false_type{}, x, nullptr, k, w.a, w.da);
        if (rc == RELIBRA_OK) rc = gram(std::false_type{}, std::true_type{}, w.a, w.da, m, w.b, w.db);
        if (rc == RELIBRA_OK) rc = s.tall ? update(std::true_type{}) : update(std::false_type{});
        if (rc != RELIBRA_OK) return rc;
    }
    return RELIBRA_OK;
}

template <class GT>
void ortho_load(const OrthoShape &s, const OrthoWs &w, const GT *g, const float *m, float mu, int mode, float *m_out, hipStream_t stream)
{
    const size_t per_matrix = (size_t)s.rows * s.cols;
    const int parts = norm_parts(s);
    const bool aligned = aligned16(g) && (mode == U_GRAD || (aligned16(m) && aligned16(m_out)));
    RELIBRA_LAUNCH(RELIBRA_K_ORTHO_NORM, stream, ortho_momentum_kernel<GT><<<dim3(parts, s.n), 256, 0, stream>>>(
        g, m, mu, mode, per_matrix, aligned && per_matrix % 4 == 0, m_out, w.parts));
    const size_t pieces = (size_t)s.rp * s.cp / 8;
    RELIBRA_LAUNCH(RELIBRA_K_ORTHO_LOAD, stream, ortho_load_kernel<GT><<<dim3((unsigned)std::min<size_t>((pieces + 255) / 256, 256), s.n), 256, 0, stream>>>(
        g, m_out, mu, mode, s, aligned && s.cols % 8 == 0, w.parts, parts, w.x[0], w.lo));
}

}  // namespace relibra

using namespace relibra;

extern "C" int relibra_orthogonalize(const void *grad, const float *momentum, int n, int rows, int cols, float mu, float scale, int steps, int flags,
                                     float *momentum_out, void *out, void *workspace, size_t workspace_bytes, relibra_stream stream_)
{
    hipStream_t stream = (hipStream_t)stream_;
    if (n < 0 || rows < 0 || cols < 0 || steps < 1 || (flags & ~(RELIBRA_ORTHO_BF16 | RELIBRA_ORTHO_NESTEROV))) return RELIBRA_EINVAL;
    if (n > 65535 || rows > kOrthoMaxSide || cols > kOrthoMaxSide || steps > 64) return RELIBRA_EUNSUPPORTED;
    if ((momentum != nullptr) != (momentum_out != nullptr) || (!momentum && (flags & RELIBRA_ORTHO_NESTEROV))) return RELIBRA_EINVAL;
    if (n == 0 || rows == 0 || cols == 0) return RELIBRA_OK;
    if (!grad || !out || out == grad) return RELIBRA_EINVAL;
    const OrthoShape s = ortho_shape(n, rows, cols);
    const long long t = 128;
    if ((long long)n * ((s.rp + t - 1) / t) * ((s.cp + t - 1) / t) > 0x3fffffff) return RELIBRA_EUNSUPPORTED;
    if (!workspace || workspace_bytes < ortho_ws_bytes(n, rows, cols)) return RELIBRA_EWORKSPACE;
    if (!aligned16(workspace)) return RELIBRA_EINVAL;
    OrthoWs w;
    char *p = (char *)workspace;
    w.x[0] = (uint16_t *)p;
    w.x[1] = (uint16_t *)(p += ortho_x_bytes(s));
    w.lo = (uint16_t *)(p += ortho_x_bytes(s));
    w.a = (uint16_t *)(p += ortho_x_bytes(s));
    w.b = (uint16_t *)(p += ortho_gram_bytes(s));
    w.da = (float *)(p += ortho_gram_bytes(s));
    w.db = (float *)(p += ortho_diag_bytes(s));
    w.parts = (double *)(p + ortho_diag_bytes(s));
    const int mode = !momentum ? U_GRAD : flags & RELIBRA_ORTHO_NESTEROV ? U_NESTEROV : U_MOMENTUM;
    if (flags & RELIBRA_ORTHO_BF16) ortho_load(s, w, (const bf16_t *)grad, momentum, mu, mode, momentum_out, stream);
    else ortho_load(s, w, (const float *)grad, momentum, mu, mode, momentum_out, stream);
    const int rc = ortho_steps(s, w, steps, scale, (uint16_t *)out, stream);
    if (rc != RELIBRA_OK) return rc;
    RELIBRA_HIP_TRY(launch_check());
    return RELIBRA_OK;
}
