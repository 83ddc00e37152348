// What the attention kernels share: matrix products by cache type, conversions
// and reductions over lane groups.
#pragma once

#include "kv_cache.h"

namespace attn {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr float NEG_INF = -__builtin_inff();
constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;

// The 16-bit type that products of a cache type are taken in.
constexpr bool is_f16(int type) { return type == SAE_KV_F16; }

template <bool F16>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <bool F16>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Two values rounded to the 16-bit type (nearest even).
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if constexpr (F16) return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
    else return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

// The two values of a packed pair.
template <bool F16>
__device__ __forceinline__ float low(uint32_t x)
{
    if constexpr (F16) return (float)__builtin_bit_cast(f16x2, x)[0];
    else return __uint_as_float(x << 16);
}
template <bool F16>
__device__ __forceinline__ float high(uint32_t x)
{
    if constexpr (F16) return (float)__builtin_bit_cast(f16x2, x)[1];
    else return __uint_as_float(x & 0xFFFF0000u);
}

// Two e4m3 values, bytes 0 and 1 or 2 and 3, times a power of two, as bf16 (exact but
// for results under 2^-126).
template <bool HIGH>
__device__ __forceinline__ uint32_t widen2(uint32_t x, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, HIGH));
}
__device__ __forceinline__ u32x2 widen4(uint32_t x, float scale) { return u32x2{widen2<false>(x, scale), widen2<true>(x, scale)}; }
__device__ __forceinline__ u32x4 widen8(uint32_t lo, uint32_t hi, float scale)
{
    const u32x2 a = widen4(lo, scale), b = widen4(hi, scale);
    return u32x4{a[0], a[1], b[0], b[1]};
}

// 2^(s - 127) for byte i of a word of scale bytes.
__device__ __forceinline__ float scale_of(uint32_t word, int i) { return __uint_as_float(((word >> (8 * i)) & 0xFFu) << 23); }

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }

// Maximum over lanes l and l ^ 32.
__device__ __forceinline__ float max_halves(float x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
// Maximum over the four lanes that agree mod 16.
__device__ __forceinline__ float max_groups(float x)
{
    x = max_halves(x);
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// The reference of weights for a maximum of `top` (both in powers of two): `bias` under it.
// Sums, outputs and parts are under the same reference, so nothing is corrected after.
// f16 loses bits under 2^-14 and everything under 2^-25, and keys that far below the
// largest may make up an output together (one key of a high score and a small value
// before many others): f16 weights use the type's range above 1.  Where fp32 does not
// hold top - bias to a few bits their reference is the maximum.
template <bool F16>
__device__ __forceinline__ float reference(float top, float bias)
{
    return top - (!F16 || fabsf(top) < 0x1p19f ? bias : 0.0f);
}

// A value that all lanes hold, in a scalar register.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long uniform(long long x)
{
    return (long long)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

// Exclusive scan over a workgroup of NW waves; total in every thread.  lds: NW
// values that nothing else uses.
template <int NW, typename T>
__device__ __forceinline__ T scan(T v, T &total, T *lds)
{
    const int lane = (int)__lane_id(), wave = threadIdx.x / SAE_WAVE;
    T s = v;
#pragma unroll
    for (int o = 1; o < SAE_WAVE; o <<= 1) {
        const T u = __shfl_up(s, o);
        if (lane >= o) s += u;
    }
    if (lane == SAE_WAVE - 1) lds[wave] = s;
    __syncthreads();
    T before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        if (w < wave) before += lds[w];
        total += lds[w];
    }
    return before + s - v;
}

}  // namespace attn
