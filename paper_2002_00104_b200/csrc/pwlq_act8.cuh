// What the kernels on 8-bit activation checkpoints share: typed loads and stores of eight values,
// the group's constants, and a value's byte and back.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pwlq_common.cuh"

namespace pwlq {

constexpr float kAct8Levels = 63.0f;            // L of the 7-bit scheme
constexpr float kAct8Tiny = 7.8886090522101181e-31f;   // 2^-100: a smaller range is held as 0
constexpr uint32_t kInfBits = 0x7f800000u;

// ------------------------------------------------------------------------------ typed access
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) {
    return __float2bfloat16_rn(v);
}
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ void unpack16(uint32_t w, float& lo, float& hi, __nv_bfloat16) {
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack16(uint32_t w, float& lo, float& hi, __half) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    lo = f.x;
    hi = f.y;
}
__device__ __forceinline__ uint32_t pack16(float lo, float hi, __nv_bfloat16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack16(float lo, float hi, __half) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// Eight consecutive values as they lie in memory (16 bytes of a 16-bit type, 32 of binary32), kept
// packed between the load and the arithmetic so that rows requested ahead cost few registers.
template <typename T> struct Raw8 {
    uint4 w;
    __device__ __forceinline__ void get(float* v) const {
        unpack16(w.x, v[0], v[1], T());
        unpack16(w.y, v[2], v[3], T());
        unpack16(w.z, v[4], v[5], T());
        unpack16(w.w, v[6], v[7], T());
    }
    __device__ __forceinline__ void set(const float* v) {
        w.x = pack16(v[0], v[1], T());
        w.y = pack16(v[2], v[3], T());
        w.z = pack16(v[4], v[5], T());
        w.w = pack16(v[6], v[7], T());
    }
    __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint4*>(p) = w; }
    __device__ __forceinline__ void clear() { w = make_uint4(0u, 0u, 0u, 0u); }
};
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void get(float* v) const {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    __device__ __forceinline__ void set(const float* v) {
        a = make_float4(v[0], v[1], v[2], v[3]);
        b = make_float4(v[4], v[5], v[6], v[7]);
    }
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const float4*>(p);
        b = *reinterpret_cast<const float4*>(p + 4);
    }
    __device__ __forceinline__ void store(float* p) const {
        *reinterpret_cast<float4*>(p) = a;
        *reinterpret_cast<float4*>(p + 4) = b;
    }
    __device__ __forceinline__ void clear() { a = b = make_float4(0.0f, 0.0f, 0.0f, 0.0f); }
};

// The first `valid` (<= 8, may be <= 0) of eight values; the others read as 0 and are not stored.
// VEC: whole chunks start on 16-byte boundaries.
template <bool VEC, typename T>
__device__ __forceinline__ void load8(Raw8<T>& raw, const T* p, int valid) {
    if (VEC && valid >= 8) { raw.load(p); return; }
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < valid ? to_f32(p[i]) : 0.0f;
    raw.set(v);
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(const float* v, T* p, int valid) {
    if (VEC && valid >= 8) {
        Raw8<T> raw;
        raw.set(v);
        raw.store(p);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < valid) p[i] = from_f32<T>(v[i]);
}

// -------------------------------------------------------------------------------- the format
// Range of a group from the largest magnitude bits among its values (an unsigned maximum orders
// finite < Inf < NaN): NaN for a non-finite one, 0 below 2^-100.
__device__ __forceinline__ float act8_range(uint32_t max_bits) {
    if (max_bits >= kInfBits) return __uint_as_float(0x7fc00000u);
    const float m = __uint_as_float(max_bits);
    return m < kAct8Tiny ? 0.0f : m;
}

// Maximum over the aligned `lanes` (power of two <= 32) lanes that hold one group.
__device__ __forceinline__ uint32_t group_max(uint32_t v, int lanes) {
    for (int o = 1; o < lanes; o <<= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// Constants of a group.  Every thread makes them for the 8 or 16 values it holds, so they are formed
// with one reciprocal per piece and products; the quotients of make_params would cost more than the
// values' own arithmetic.  A piece with a non-positive range gets 0.
__device__ __forceinline__ PieceParams act8_params(float m, float ratio) {
    PieceParams P;
    P.p = __fmul_rn(m, ratio);
    const float d = __fsub_rn(m, P.p);
    P.s1 = __fmul_rn(P.p, 1.0f / kAct8Levels);
    P.s2 = __fmul_rn(d, 1.0f / kAct8Levels);          // NaN ranges make every step NaN
    P.inv1 = P.p > 0.0f ? __fmul_rn(__frcp_rn(P.p), kAct8Levels) : 0.0f;
    P.inv2 = d > 0.0f ? __fmul_rn(__frcp_rn(d), kAct8Levels) : 0.0f;
    return P;
}

// Byte of a value; P = act8_params of a group with a range that is neither 0 nor NaN.  The level sits
// in the low mantissa bits after 1.5 * 2^23 was added (see quantize_mag).
__device__ __forceinline__ uint32_t act8_byte(float x, const PieceParams& P) {
    const float a = fabsf(x);
    const bool tail = a > P.p;
    const float u = __fsub_rn(a, tail ? P.p : 0.0f);
    const float r = __fadd_rn(__fmul_rn(u, tail ? P.inv2 : P.inv1), 12582912.0f);
    const int q = min(__float_as_int(r) - 0x4B400000, 63);
    return (x < 0.0f ? 128u : 0u) | (tail ? 64u : 0u) | (uint32_t)q;
}

// Four bytes, the first in the low bits; 0 for a group that holds nothing.
__device__ __forceinline__ uint32_t act8_word(const float* x, float m, const PieceParams& P) {
    if (!(m > 0.0f)) return 0u;
    return act8_byte(x[0], P) | act8_byte(x[1], P) << 8 | act8_byte(x[2], P) << 16 |
           act8_byte(x[3], P) << 24;
}

__device__ __forceinline__ float act8_value(uint32_t byte, const PieceParams& P) {
    const float q = (float)(byte & 63u);
    const float v = (byte & 64u) ? __fadd_rn(__fmul_rn(q, P.s2), P.p) : __fmul_rn(q, P.s1);
    return __uint_as_float(__float_as_uint(v) ^ ((byte & 128u) << 24));
}
__device__ __forceinline__ void act8_values(uint32_t word, const PieceParams& P, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = act8_value((word >> (8 * i)) & 0xffu, P);
}

}  // namespace pwlq
