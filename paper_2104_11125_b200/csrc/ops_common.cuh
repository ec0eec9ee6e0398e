// Shared helpers of the learner-side operators: element types, vector access, waits.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/scalecom_operators.h"
#include "common.cuh"

namespace sc {

template <typename T> struct Elem;
template <> struct Elem<float> {
    static constexpr int id = SCALECOM_F32;
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
};
template <> struct Elem<__half> {
    static constexpr int id = SCALECOM_F16;
    static __device__ __forceinline__ float up(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half down(float v) { return __float2half_rn(v); }
};
template <> struct Elem<__nv_bfloat16> {
    static constexpr int id = SCALECOM_BF16;
    static __device__ __forceinline__ float up(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 down(float v) { return __float2bfloat16_rn(v); }
};

// N elements of T as the words that a single load or store moves (N * sizeof(T) <= 16). Built-in vector types on purpose: a struct
// of 16-bit elements is copied element by element (measured: a bf16 layer norm at 1.5 TB/s).
template <int BYTES> struct Words;
template <> struct Words<16> { typedef uint4 type; };
template <> struct Words<8> { typedef uint2 type; };
template <> struct Words<4> { typedef uint32_t type; };
template <> struct Words<2> { typedef uint16_t type; };
template <typename T, int N> using Pack = typename Words<N * sizeof(T)>::type;

__device__ __forceinline__ uint32_t word_of(const uint4& p, int i) { return i == 0 ? p.x : i == 1 ? p.y : i == 2 ? p.z : p.w; }
__device__ __forceinline__ uint32_t word_of(const uint2& p, int i) { return i == 0 ? p.x : p.y; }
__device__ __forceinline__ uint32_t word_of(const uint32_t& p, int) { return p; }
__device__ __forceinline__ uint32_t word_of(const uint16_t& p, int) { return p; }
__device__ __forceinline__ void set_word(uint4& p, int i, uint32_t v) { (i == 0 ? p.x : i == 1 ? p.y : i == 2 ? p.z : p.w) = v; }
__device__ __forceinline__ void set_word(uint2& p, int i, uint32_t v) { (i == 0 ? p.x : p.y) = v; }
__device__ __forceinline__ void set_word(uint32_t& p, int, uint32_t v) { p = v; }
__device__ __forceinline__ void set_word(uint16_t& p, int, uint32_t v) { p = uint16_t(v); }

// element i of a pack (i a constant after unrolling)
template <typename T, int N> __device__ __forceinline__ float pack_get(const Pack<T, N>& p, int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(word_of(p, i));
    const uint32_t w = word_of(p, i / 2);
    if constexpr (Elem<T>::id == SCALECOM_BF16) return __uint_as_float((i & 1) ? w & 0xFFFF0000u : w << 16);
    return __half2float(__ushort_as_half(uint16_t((i & 1) ? w >> 16 : w & 0xFFFFu)));
}
template <typename T> __device__ __forceinline__ uint32_t bits_of(float v) {
    if constexpr (Elem<T>::id == SCALECOM_F32) return __float_as_uint(v);
    else if constexpr (Elem<T>::id == SCALECOM_BF16) return __bfloat16_as_ushort(__float2bfloat16_rn(v));
    else return __half_as_ushort(__float2half_rn(v));
}
template <typename T, int N>
__device__ __forceinline__ void load_up(const T* p, float (&v)[N]) {
    const Pack<T, N> t = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = pack_get<T, N>(t, i);
}
template <typename T, int N>
__device__ __forceinline__ void store_down(T* p, const float (&v)[N]) {
    Pack<T, N> t;
    if constexpr (sizeof(T) == 4 || N == 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) set_word(t, i, bits_of<T>(v[i]));
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            if constexpr (Elem<T>::id == SCALECOM_BF16) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[i], v[i + 1]);
                set_word(t, i / 2, *reinterpret_cast<const uint32_t*>(&h));
            } else {
                const __half2 h = __floats2half2_rn(v[i], v[i + 1]);
                set_word(t, i / 2, *reinterpret_cast<const uint32_t*>(&h));
            }
        }
    }
    *reinterpret_cast<Pack<T, N>*>(p) = t;
}

// 32 consecutive elements of one row: 16-byte accesses where the address and the row's end allow it
template <typename T>
__device__ __forceinline__ void load_row32(const T* p, float* v, int ncols) {
    constexpr int N = 16 / sizeof(T);
    if (ncols >= 32 && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < 32; i += N) {
            float t[N];
            load_up<T, N>(p + i, t);
#pragma unroll
            for (int j = 0; j < N; ++j) v[i + j] = t[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = i < ncols ? Elem<T>::up(p[i]) : 0.0f;
    }
}

__device__ __forceinline__ float warp_sum_f(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    return v;
}

// ---- chains of launches ------------------------------------------------------------------------------
// Every kernel of an operator is launched with programmatic stream serialisation: its blocks may start while the
// kernel before it drains, and each waits here, before its first access to global memory, until that kernel has
// completed and its writes are visible.
__device__ __forceinline__ void chain_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void chain_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- power-of-two scales of fp32 operands --------------------------------------------------------------
// A tensor's largest finite magnitude (bits in a device word) gives the scale 2^(14 - e), e its exponent: the
// scaled values are below 2^15, inside fp16's range with room for rounding up.
__device__ __forceinline__ int plane_shift(uint32_t amax_bits) {
    const int e = int(amax_bits >> 23) - 127;        // -127 for zero and denormals
    return amax_bits == 0u ? 0 : min(14 - e, 126);   // 126: both 2^s and 2^-s are normal numbers
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(uint32_t(e + 127) << 23); }      // -126 .. 127
__device__ __forceinline__ float plane_scale(uint32_t amax_bits) { return power_of_two(plane_shift(amax_bits)); }
// 2^e takes the scales of two operands out of their product again: -252 .. 226
__device__ __forceinline__ int plane_unshift(uint32_t amax_a, uint32_t amax_b) { return -plane_shift(amax_a) - plane_shift(amax_b); }
// It is applied as two factors, one after the other: a product that fp32 holds must neither pass infinity nor zero on its way. The second
// is 1 unless the first cannot hold it all.
struct Unscale { float first, second; };
__device__ __forceinline__ Unscale plane_unscale(int e) {
    const int h = e < -126 || e > 127 ? e / 2 : e;
    return {power_of_two(h), power_of_two(e - h)};
}

__device__ __forceinline__ uint32_t finite_bits(float v) {
    const uint32_t b = mag_key(v);
    return b < 0x7F800000u ? b : 0u;
}

// v as two fp16 values hi + lo (22 mantissa bits); an infinity or NaN stays in hi alone
__device__ __forceinline__ void split_planes(float v, __half& hi, __half& lo) {
    hi = __float2half_rn(v);
    const float r = v - __half2float(hi);
    lo = __float2half_rn((mag_key(r) < 0x7F800000u) ? r : 0.0f);
}

}  // namespace sc
