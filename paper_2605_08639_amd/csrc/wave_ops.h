// Reductions over aligned groups of lanes of a 64-lane wave: every lane of a group gets the group's result.  Up to 16 lanes
// they are DPP moves (no LDS, no index registers), beyond that the row and half swaps of gfx950.
#pragma once
#include "common.h"
#include "wave_stage.h"

namespace relibra {

template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}

struct SumOp {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
struct MaxOp {
    static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); }
};

// LANES: 1, 2, 4, .. 64.  The order of the additions is the same for every lane and every call.
template <int LANES, class Op> __device__ __forceinline__ float group_reduce(float v)
{
    static_assert(LANES >= 1 && LANES <= 64 && (LANES & (LANES - 1)) == 0, "a power of two");
    if constexpr (LANES >= 2) v = Op::of(v, dpp<0xB1>(v));         // quad_perm 1,0,3,2
    if constexpr (LANES >= 4) v = Op::of(v, dpp<0x4E>(v));         // quad_perm 2,3,0,1
    if constexpr (LANES >= 8) v = Op::of(v, dpp<0x141>(v));        // row_half_mirror: the quads hold their own result by now
    if constexpr (LANES >= 16) v = Op::of(v, dpp<0x140>(v));       // row_mirror
    if constexpr (LANES >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
        v = Op::of(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
    }
    if constexpr (LANES >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
        v = Op::of(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
    }
    return v;
}
template <int LANES> __device__ __forceinline__ float group_sum(float v) { return group_reduce<LANES, SumOp>(v); }
template <int LANES> __device__ __forceinline__ float group_max(float v) { return group_reduce<LANES, MaxOp>(v); }

// Sum over the lanes of a wave that have the same place in their group of LANES (4, 8, 16); every lane gets its place's.
template <int LANES> __device__ __forceinline__ float place_sum(float v)
{
    static_assert(LANES == 4 || LANES == 8 || LANES == 16, "group size");
    if constexpr (LANES <= 8) v += dpp<0x128>(v);                  // row_ror 8
    if constexpr (LANES <= 4) v += dpp<0x124>(v);                  // row_ror 4
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    v = __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
    const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    return __builtin_bit_cast(float, (unsigned)s[0]) + __builtin_bit_cast(float, (unsigned)s[1]);
}

// Sums over a wave's lanes up to each lane: shifts within rows of 16, then the rows before.
__device__ __forceinline__ int wave_scan(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);   // row_shr 1, 2, 4, 8: zeros come in
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    const int lane = threadIdx.x & 63, a = __builtin_amdgcn_readlane(v, 15), b = __builtin_amdgcn_readlane(v, 31), c = __builtin_amdgcn_readlane(v, 47);
    return v + (lane >= 48 ? a + b + c : lane >= 32 ? a + b : lane >= 16 ? a : 0);
}

// Eight consecutive values of memory (16-byte aligned) as loaded, as fp32, and back (one rounding to bf16).
template <class T> struct Raw8;
template <> struct Raw8<bf16_t> {
    uint4 q;
};
template <> struct Raw8<float> {
    float4 a, b;
};
__device__ __forceinline__ Raw8<bf16_t> fetch8(const bf16_t *p) { return Raw8<bf16_t>{*reinterpret_cast<const uint4 *>(p)}; }
__device__ __forceinline__ Raw8<float> fetch8(const float *p)
{
    return Raw8<float>{reinterpret_cast<const float4 *>(p)[0], reinterpret_cast<const float4 *>(p)[1]};
}
template <class T> __device__ __forceinline__ Raw8<T> zero8()
{
    if constexpr (sizeof(T) == 2) return Raw8<T>{make_uint4(0, 0, 0, 0)};
    else return Raw8<T>{make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
}
__device__ __forceinline__ void unpack8(const Raw8<bf16_t> &r, float (&v)[8])
{
    const uint32_t w[4] = {r.q.x, r.q.y, r.q.z, r.q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack8(const Raw8<float> &r, float (&v)[8])
{
    v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w;
    v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
}
// The same at any alignment of the element type (the memory pipeline takes such accesses).
__device__ __forceinline__ Raw8<bf16_t> fetch8_any(const bf16_t *p)
{
    typedef uint32_t any4 __attribute__((ext_vector_type(4), aligned(2)));
    return Raw8<bf16_t>{__builtin_bit_cast(uint4, *reinterpret_cast<const any4 *>(p))};
}
__device__ __forceinline__ Raw8<float> fetch8_any(const float *p)
{
    typedef float any4 __attribute__((ext_vector_type(4), aligned(4)));
    return Raw8<float>{__builtin_bit_cast(float4, reinterpret_cast<const any4 *>(p)[0]), __builtin_bit_cast(float4, reinterpret_cast<const any4 *>(p)[1])};
}
template <class T> __device__ __forceinline__ void load8(const T *p, float (&v)[8]) { unpack8(fetch8(p), v); }
__device__ __forceinline__ void store8(bf16_t *p, const float (&v)[8])
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack2bf(v[0], v[1]), pack2bf(v[2], v[3]), pack2bf(v[4], v[5]), pack2bf(v[6], v[7]));
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8_any(bf16_t *p, const float (&v)[8])
{
    typedef uint32_t any4 __attribute__((ext_vector_type(4), aligned(2)));
    *reinterpret_cast<any4 *>(p) = any4{pack2bf(v[0], v[1]), pack2bf(v[2], v[3]), pack2bf(v[4], v[5]), pack2bf(v[6], v[7])};
}
__device__ __forceinline__ void store8_any(float *p, const float (&v)[8])
{
    typedef float any4 __attribute__((ext_vector_type(4), aligned(4)));
    reinterpret_cast<any4 *>(p)[0] = any4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<any4 *>(p)[1] = any4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ float to_f32(bf16_t b) { return bf2f(b); }
__device__ __forceinline__ float to_f32(float f) { return f; }
__device__ __forceinline__ void from_f32(bf16_t *p, float f) { *p = f2bf(f); }
__device__ __forceinline__ void from_f32(float *p, float f) { *p = f; }

}  // namespace relibra
