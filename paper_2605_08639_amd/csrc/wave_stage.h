// Row-major staging of 16-bit accumulator tiles through a wave's own LDS, shared by the GEMM epilogues.
#pragma once
#include "common.h"

namespace relibra {

// LDS operations of one wave execute in order; this keeps the compiler from moving them across
// the hand-over between the two layouts and waits for the data.
__device__ __forceinline__ void wave_lds_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_s_waitcnt(0xC07F);          // lgkmcnt(0)
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Per-wave LDS staging between the accumulator layout (a lane holds 4 consecutive columns of
// its row) and the row-major layout (a row's columns spread over consecutive lanes), so that
// global accesses of the epilogue are 16 bytes per lane along rows: full cache lines.
// A wave stages 64 rows x NCOLS bf16; 16-byte pieces of a row are XOR-ed with the row number.
template <int NCOLS>
struct WaveStage {
    static constexpr int PIECES = NCOLS / 8;
    static constexpr int BYTES = 64 * NCOLS * 2;
    static constexpr int ROWS_PER_PASS = 64 / PIECES;
    static constexpr int PASSES = 64 / ROWS_PER_PASS;

    // accumulator side: 8 bytes = columns col..col+3 (col % 4 == 0) of `row`
    static __device__ __forceinline__ int acc_addr(int row, int col)
    {
        return row * (NCOLS * 2) + ((((col >> 3) ^ row) & (PIECES - 1)) << 4) + ((col >> 2) & 1) * 8;
    }
    static __device__ __forceinline__ void put(char *buf, int row, int col, uint2 v) { *reinterpret_cast<uint2 *>(buf + acc_addr(row, col)) = v; }
    static __device__ __forceinline__ uint2 get(const char *buf, int row, int col) { return *reinterpret_cast<const uint2 *>(buf + acc_addr(row, col)); }

    // row-major side: stage -> global, rows grow0.. of a tensor with leading dimension ld.
    // All LDS reads first, then the (predicated) stores: left to itself the compiler moves every
    // read into the branch of its store, and each store then waits for its own read in turn.
    // Only columns col_from <= c < n_dim are stored.
    static __device__ __forceinline__ void flush(const char *buf, bf16_t *out, int ld, int grow0, int row_end,
                                                 int gcol0, int n_dim, int lane, int col_from = 0)
    {
        uint4 v[PASSES];
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = p * ROWS_PER_PASS + lane / PIECES, piece = lane % PIECES;
            v[p] = *reinterpret_cast<const uint4 *>(buf + r * (NCOLS * 2) + (((piece ^ r) & (PIECES - 1)) << 4));
        }
#pragma unroll
        for (int p = 0; p < PASSES; ++p)          // the values are needed here: the reads stay above
            asm volatile("" : "+v"(v[p].x), "+v"(v[p].y), "+v"(v[p].z), "+v"(v[p].w));
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = p * ROWS_PER_PASS + lane / PIECES, piece = lane % PIECES;
            if (grow0 + r < row_end && gcol0 + piece * 8 < n_dim && gcol0 + piece * 8 >= col_from)
                *reinterpret_cast<uint4 *>(out + (size_t)(grow0 + r) * ld + gcol0 + piece * 8) = v[p];
        }
    }
    // global -> stage.  Rows and columns beyond the tensor are read from clamped (valid) addresses
    // instead of being skipped: what lands in their places is never stored by flush, and without
    // the predicates all loads of the fill are in flight together (predicated, every load was
    // waited for before the next one went out: one memory round trip per pass).
    // Needs grow0 < row_end and n_dim >= 8.
    // two tensors of the same shape into two staging areas, all loads in flight together
    static __device__ __forceinline__ void fill2(char *buf0, char *buf1, const bf16_t *in0, const bf16_t *in1, int ld, int grow0,
                                                 int row_end, int gcol0, int n_dim, int lane)
    {
        uint4 v0[PASSES], v1[PASSES];
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = p * ROWS_PER_PASS + lane / PIECES, piece = lane % PIECES;
            const size_t at = (size_t)min(grow0 + r, row_end - 1) * ld + min(gcol0 + piece * 8, n_dim - 8);
            v0[p] = *reinterpret_cast<const uint4 *>(in0 + at);
            v1[p] = *reinterpret_cast<const uint4 *>(in1 + at);
        }
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = p * ROWS_PER_PASS + lane / PIECES, piece = lane % PIECES;
            const int at = r * (NCOLS * 2) + (((piece ^ r) & (PIECES - 1)) << 4);
            *reinterpret_cast<uint4 *>(buf0 + at) = v0[p];
            *reinterpret_cast<uint4 *>(buf1 + at) = v1[p];
        }
    }
    static __device__ __forceinline__ void fill(char *buf, const bf16_t *in, int ld, int grow0, int row_end,
                                                int gcol0, int n_dim, int lane)
    {
        uint4 v[PASSES];
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = p * ROWS_PER_PASS + lane / PIECES, piece = lane % PIECES;
            const int gr = min(grow0 + r, row_end - 1), gc = min(gcol0 + piece * 8, n_dim - 8);
            v[p] = *reinterpret_cast<const uint4 *>(in + (size_t)gr * ld + gc);
        }
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int r = p * ROWS_PER_PASS + lane / PIECES, piece = lane % PIECES;
            *reinterpret_cast<uint4 *>(buf + r * (NCOLS * 2) + (((piece ^ r) & (PIECES - 1)) << 4)) = v[p];
        }
    }
};

}  // namespace relibra
