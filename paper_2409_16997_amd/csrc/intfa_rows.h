// Rows of activations, 8 consecutive elements to a lane: loads widened to fp32, the row's largest magnitude, INT8 codes, the Walsh-Hadamard transform.
// Shared by the quantizers of whole tensors and those that write into a cache (gfx950 only; not part of the C ABI).
#ifndef INTFA_ROWS_H
#define INTFA_ROWS_H

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <hip/hip_bf16.h>
#include <stdint.h>
#include <type_traits>

namespace ifa_rows {

// ---- 8 consecutive elements of any supported dtype, as loaded and widened exactly to fp32 -------
template <typename T> struct Raw8 {                   // fp16, bf16: one 128-bit load
    uint4 raw;
    // held as loaded: the compiler may not keep the widened values (twice the registers) in its place
    __device__ __forceinline__ void hold() { asm volatile("" : "+v"(raw.x), "+v"(raw.y), "+v"(raw.z), "+v"(raw.w)); }
    template <typename I> __device__ __forceinline__ void load(const void *p, I idx) { raw = *reinterpret_cast<const uint4 *>(static_cast<const T *>(p) + idx); }
    template <typename I> __device__ __forceinline__ void load_once(const void *p, I idx) {      // with the non-temporal hint
        typedef unsigned u4 __attribute__((ext_vector_type(4)));
        const u4 v = __builtin_nontemporal_load(reinterpret_cast<const u4 *>(static_cast<const T *>(p) + idx));
        raw = make_uint4(v[0], v[1], v[2], v[3]);
    }
    __device__ __forceinline__ void widen(float (&x)[8]) const {
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same_v<T, __half>) {
                const float2 f = __half22float2(__builtin_bit_cast(__half2, w[i]));
                x[2 * i] = f.x;
                x[2 * i + 1] = f.y;
            } else {                                  // bf16 -> fp32 is a 16-bit shift
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
};
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void hold() {
        asm volatile("" : "+v"(a.x), "+v"(a.y), "+v"(a.z), "+v"(a.w), "+v"(b.x), "+v"(b.y), "+v"(b.z), "+v"(b.w));
    }
    template <typename I> __device__ __forceinline__ void load_once(const void *p, I idx) {
        typedef float f4 __attribute__((ext_vector_type(4)));
        const f4 *q = reinterpret_cast<const f4 *>(static_cast<const float *>(p) + idx);
        const f4 v = __builtin_nontemporal_load(q), w = __builtin_nontemporal_load(q + 1);
        a = make_float4(v[0], v[1], v[2], v[3]);
        b = make_float4(w[0], w[1], w[2], w[3]);
    }
    template <typename I> __device__ __forceinline__ void load(const void *p, I idx) {
        const float4 *q = reinterpret_cast<const float4 *>(static_cast<const float *>(p) + idx);
        a = q[0];
        b = q[1];
    }
    __device__ __forceinline__ void widen(float (&x)[8]) const {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
};
template <typename T, typename I> __device__ __forceinline__ void load8(const void *p, I idx, float (&x)[8]) {
    Raw8<T> r;
    r.load(p, idx);
    r.widen(x);
}

__device__ __forceinline__ float absmax8(const float (&x)[8]) {
    float a = fmaxf(fabsf(x[0]), fabsf(x[1]));
#pragma unroll
    for (int i = 2; i < 8; ++i) a = fmaxf(a, fabsf(x[i]));
    return a;
}

// The conversion as the hardware does it, which C++ leaves undefined: NaN becomes 0, what is too large the nearest integer.
__device__ __forceinline__ int to_int(float t) {
    int i;
    asm("v_cvt_i32_f32 %0, %1" : "=v"(i) : "v"(t));
    return i;
}
// q = clamp(rint(x * inv), -127, 127) for 8 values, packed little-endian into two dwords.  For rows below 127 / max fp32 inv is infinite: every number but 0 is +-127, and 0 times it, NaN, is 0.
__device__ __forceinline__ uint2 quant8(const float (&x)[8], float inv) {
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int t = to_int(rintf(x[i] * inv));
        w[i >> 2] |= (static_cast<uint32_t>(t < -127 ? -127 : t > 127 ? 127 : t) & 0xffu) << (8 * (i & 3));
    }
    return make_uint2(w[0], w[1]);
}

// max over the aligned group of `LPR` adjacent lanes (LPR a power of two <= 64), result in all.
template <int LPR>
__device__ __forceinline__ float group_max(float a) {
    // quad_perm [1,0,3,2] and [2,3,0,1], then mirrors inside 8 and 16 lanes: DPP, no LDS.
    if (LPR >= 2) a = fmaxf(a, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(a), 0xB1, 0xf, 0xf, true)));
    if (LPR >= 4) a = fmaxf(a, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(a), 0x4E, 0xf, 0xf, true)));
    if (LPR >= 8) a = fmaxf(a, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(a), 0x141, 0xf, 0xf, true)));  // row_half_mirror
    if (LPR >= 16) a = fmaxf(a, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(a), 0x140, 0xf, 0xf, true))); // row_mirror
    if (LPR >= 32) a = fmaxf(a, __shfl_xor(a, 16));
    if (LPR >= 64) a = fmaxf(a, __shfl_xor(a, 32));
    return a;
}

// value held by lane ^ M (M a power of two < 64): DPP inside a quad, the LDS crossbar (no memory access) beyond
template <int M> __device__ __forceinline__ float lane_xor(float x) {
    const int v = __float_as_int(x);
    if (M == 1) return __int_as_float(__builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true));        // quad_perm [1,0,3,2]
    if (M == 2) return __int_as_float(__builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true));        // quad_perm [2,3,0,1]
    if (M == 4) return __int_as_float(__builtin_amdgcn_ds_swizzle(v, 0x101F));                   // bit mode: xor 4
    if (M == 8) return __int_as_float(__builtin_amdgcn_ds_swizzle(v, 0x201F));
    if (M == 16) return __int_as_float(__builtin_amdgcn_ds_swizzle(v, 0x401F));
    return __shfl_xor(x, 32);
}

// One butterfly stage of the Walsh-Hadamard transform across lanes: elements 8*sub + i and 8*(sub ^ M) + i.
// The lane with bit M clear holds a and keeps a + b, the other holds b and keeps a - b.
template <int M, int LPR> __device__ __forceinline__ void hadamard_lane_stage(float (&x)[8], int sub) {
    if (M < LPR) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = lane_xor<M>(x[i]);
            x[i] = (sub & M) ? (p - x[i]) : (x[i] + p);
        }
    }
}

// Unnormalized Walsh-Hadamard transform (Sylvester order) of a row of 8*LPR elements spread over LPR lanes,
// stages h = 1, 2, 4 inside the lane's 8 registers, then h = 8, 16, ... across lanes, all in fp32.
template <int LPR> __device__ __forceinline__ void hadamard_row(float (&x)[8], int sub) {
#pragma unroll
    for (int h = 1; h < 8; h <<= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((i & h) == 0) {
                const float a = x[i], b = x[i + h];
                x[i] = a + b;
                x[i + h] = a - b;
            }
    hadamard_lane_stage<1, LPR>(x, sub);
    hadamard_lane_stage<2, LPR>(x, sub);
    hadamard_lane_stage<4, LPR>(x, sub);
    hadamard_lane_stage<8, LPR>(x, sub);
    hadamard_lane_stage<16, LPR>(x, sub);
    hadamard_lane_stage<32, LPR>(x, sub);
}

}  // namespace ifa_rows

#endif  // INTFA_ROWS_H
