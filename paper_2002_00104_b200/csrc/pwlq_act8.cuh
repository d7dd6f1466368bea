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

// A kernel that was launched as the dependent of the one before it may start once all blocks of that
// one have called allow_dependents (or have ended), and must call await_previous before it touches
// anything that the earlier kernel writes or reads.
__device__ __forceinline__ void allow_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void await_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

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
    __device__ __forceinline__ void from_words(const uint32_t* x) { w = make_uint4(x[0], x[1], x[2], x[3]); }
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
    __device__ __forceinline__ void from_words(const uint32_t* x) {
        a = make_float4(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]), __uint_as_float(x[3]));
        b = make_float4(__uint_as_float(x[4]), __uint_as_float(x[5]), __uint_as_float(x[6]), __uint_as_float(x[7]));
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

// Moves a window of 32-bit words `bytes` bytes (a multiple of the value size, < 16) towards its front;
// the caller does not use what would have to come from behind it.
template <int WORDS, bool HALVES>
__device__ __forceinline__ void shift_window(uint32_t (&w)[WORDS], int bytes) {
#pragma unroll
    for (int i = 0; i + 2 < WORDS; ++i) w[i] = bytes & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i + 1 < WORDS; ++i) w[i] = bytes & 4 ? w[i + 1] : w[i];
    if (HALVES)
#pragma unroll
        for (int i = 0; i + 1 < WORDS; ++i) w[i] = __byte_perm(w[i], w[i + 1], bytes & 2 ? 0x5432 : 0x3210);
}

// Values from p - o on, o = how many values past a 16-byte boundary p is.
template <typename T> __device__ __forceinline__ int past_boundary(const T* p) {
    return (int)(((uintptr_t)p & 15) / sizeof(T));
}

// Eight values at p.  `valid` of them exist (may be <= 0 or > 8; the others read as 0) and `before`
// values of the same row lie before p.  VEC: p is on a 16-byte boundary.  Off it, the aligned 16-byte
// words around the eight values are read, where all of them lie inside the row, and shifted into
// place; the row's ends are read value by value, so nothing outside the row is touched.
template <bool VEC, typename T>
__device__ __forceinline__ void load8(Raw8<T>& raw, const T* p, int valid, int before) {
    if (VEC && valid >= 8) { raw.load(p); return; }
    if (!VEC) {
        constexpr int kPer = 16 / sizeof(T), kVecs = sizeof(T) == 4 ? 3 : 2;
        const int o = past_boundary(p);
        if (o == 0 && valid >= 8) { raw.load(p); return; }
        if (before >= o && valid >= kVecs * kPer - o) {
            uint32_t w[4 * kVecs];
            const uint4* q = reinterpret_cast<const uint4*>(p - o);
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                const uint4 x = q[i];
                w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
            }
            shift_window<4 * kVecs, sizeof(T) == 2>(w, o * (int)sizeof(T));
            raw.from_words(w);
            return;
        }
    }
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < valid ? to_f32(p[i]) : 0.0f;
    raw.set(v);
}

// The first `valid` of eight values to p, value by value.
template <typename T>
__device__ __forceinline__ void store8_each(const float* v, T* p, int valid) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < valid) p[i] = from_f32<T>(v[i]);
}

// The same for a whole warp at once: every lane calls.  VEC: p is on a 16-byte boundary where
// valid >= 8.  Off the boundary, lanes that hold consecutive parts of one row (valid counts to the
// row's end in all of them) turn their values in shared memory, so that a warp writes 32 neighbours at
// a time; parts of several rows are written value by value.
template <bool VEC, typename T>
__device__ __forceinline__ void store8(const float* v, T* p, int valid) {
    if (VEC) {
        if (valid >= 8) {
            Raw8<T> raw;
            raw.set(v);
            raw.store(p);
        } else {
            store8_each(v, p, valid);
        }
        return;
    }
    constexpr unsigned kAll = 0xffffffffu;
    __shared__ Raw8<T> turn[32][32];
    const int lane = threadIdx.x & 31;
    Raw8<T>* const mine = turn[threadIdx.x >> 5];
    T* const p0 = reinterpret_cast<T*>(__shfl_sync(kAll, (uintptr_t)p, 0));
    const int valid0 = __shfl_sync(kAll, valid, 0);
    if (!__all_sync(kAll, p == p0 + 8 * lane && (valid == valid0 - 8 * lane || (valid <= 0 && valid0 <= 8 * lane)))) {
        store8_each(v, p, valid);
        return;
    }
    Raw8<T> raw;
    raw.set(v);
    __syncwarp();
    mine[lane] = raw;
    __syncwarp();
    const T* from = reinterpret_cast<const T*>(mine);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (32 * i + lane < valid0) p0[32 * i + lane] = from[32 * i + lane];
}

// Two binary32 lanes at a time (see fma2 in pwlq_common.cuh).
__device__ __forceinline__ u64 mul2(u64 a, u64 b) {
    u64 d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d;
}
__device__ __forceinline__ u64 both(float v) { return pack2(v, v); }
__device__ __forceinline__ float lo2(u64 v) { float a, b; unpack2(v, a, b); return a; }
__device__ __forceinline__ float hi2(u64 v) { float a, b; unpack2(v, a, b); return b; }

// 32 bytes at once: eight binary32 or sixteen 16-bit values, on a 32-byte boundary.
struct Raw32 { uint32_t w[8]; };
__device__ __forceinline__ void store32(void* p, const Raw32& r) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]), "r"(r.w[4]), "r"(r.w[5]),
                   "r"(r.w[6]), "r"(r.w[7]) : "memory");
}
__device__ __forceinline__ Raw32 load32_global(const void* p) {   // on a 32-byte boundary
    Raw32 r;
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]),
                   "=r"(r.w[6]), "=r"(r.w[7]) : "l"(p) : "memory");
    return r;
}
__device__ __forceinline__ Raw32 load32(const void* p) {          // two 16-byte reads: any memory
    const uint4 a = reinterpret_cast<const uint4*>(p)[0], b = reinterpret_cast<const uint4*>(p)[1];
    return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
// The values of 32 bytes in pairs, and back.
template <typename T> constexpr int kPairs32 = 16 / sizeof(T);
template <typename T>
__device__ __forceinline__ void pairs32(const Raw32& r, u64* v, T) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float a, b;
        unpack16(r.w[i], a, b, T());
        v[i] = pack2(a, b);
    }
}
__device__ __forceinline__ void pairs32(const Raw32& r, u64* v, float) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack2(__uint_as_float(r.w[2 * i]), __uint_as_float(r.w[2 * i + 1]));
}
template <typename T>
__device__ __forceinline__ Raw32 raw32(const u64* v, T) {
    Raw32 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.w[i] = pack16(lo2(v[i]), hi2(v[i]), T());
    return r;
}
__device__ __forceinline__ Raw32 raw32(const u64* v, float) {
    Raw32 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.w[2 * i] = __float_as_uint(lo2(v[i]));
        r.w[2 * i + 1] = __float_as_uint(hi2(v[i]));
    }
    return r;
}

// -------------------------------------------------------------------------------- the format
// Larger of two magnitudes; NaN wins.
__device__ __forceinline__ float max_abs(float top, float v) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(top), "f"(fabsf(v)));
    return r;
}
// Range of a group from its largest magnitude: NaN for a non-finite one, 0 below 2^-100.
__device__ __forceinline__ float act8_range(float top) {
    if (!(top < __uint_as_float(kInfBits))) return __uint_as_float(0x7fc00000u);
    return top < kAct8Tiny ? 0.0f : top;
}

// Maximum over the aligned `lanes` (power of two <= 32) lanes that hold one group.
__device__ __forceinline__ float group_max(float v, int lanes) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
        if (o < lanes) v = max_abs(v, __shfl_xor_sync(0xffffffffu, v, o));
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

// The same for a group that is spread over an even number of lanes from an even lane on, all of which
// call together: a pair of lanes shares the two reciprocals, the encoder's most expensive part.
__device__ __forceinline__ PieceParams act8_params_paired(float m, float ratio) {
    PieceParams P;
    P.p = __fmul_rn(m, ratio);
    const float d = __fsub_rn(m, P.p);
    const bool odd = threadIdx.x & 1;
    const float of = odd ? d : P.p;
    const float mine = of > 0.0f ? __fmul_rn(__frcp_rn(of), kAct8Levels) : 0.0f;
    const float other = __shfl_xor_sync(0xffffffffu, mine, 1);
    P.inv1 = odd ? other : mine;
    P.inv2 = odd ? mine : other;
    return P;
}

// Eight bytes of eight values of a group with range m; P = act8_params(m).  Both pieces' levels are
// formed and one is taken: adding 1.5 * 2^23 (+ 64 in the tail) rounds the product to an integer,
// ties to even, and leaves region * 64 + level in the low byte of the sum.  No clamp is needed: a
// product exceeds 63 by its own rounding at most.
__device__ __forceinline__ uint2 act8_bytes8(const float* x, float m, const PieceParams& P) {
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t r[4], s[4];
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const float* y = x + 4 * h + i;
            float c[2], t[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                c[k] = __fmul_rn(fabsf(y[k]), P.inv1);
                t[k] = __fmul_rn(__fsub_rn(fabsf(y[k]), P.p), P.inv2);
            }
            const u64 center = add2(pack2(c[0], c[1]), both(12582912.0f));
            const u64 tail = add2(pack2(t[0], t[1]), both(12582912.0f + 64.0f));
            r[i] = __float_as_uint(fabsf(y[0]) > P.p ? lo2(tail) : lo2(center));
            r[i + 1] = __float_as_uint(fabsf(y[1]) > P.p ? hi2(tail) : hi2(center));
            s[i] = __float_as_uint(y[0]);
            s[i + 1] = __float_as_uint(y[1]);
        }
        const uint32_t low = __byte_perm(__byte_perm(r[0], r[1], 0x0040), __byte_perm(r[2], r[3], 0x0040), 0x5410);
        const uint32_t top = __byte_perm(__byte_perm(s[0], s[1], 0x0073), __byte_perm(s[2], s[3], 0x0073), 0x5410);
        w[h] = low | (top & 0x80808080u);
    }
    return m > 0.0f ? make_uint2(w[0], w[1]) : make_uint2(0u, 0u);
}

// The eight values of eight bytes times a factor, in pairs, to within a few roundings (the gradients'
// use; act8_values8 gives the format's own bits).  f = 128 + j from a byte permutation; the pieces are
// the lines s1 * (f - 128) and p + s2 * (f - 192), one fused operation each.  192 steps of the tail must not
// overflow: m * factor <= 1.1e38.
struct Act8Lines { u64 s1, z1, s2, z2; };
__device__ __forceinline__ Act8Lines act8_lines(float m, float ratio, float factor) {
    const float p = m * ratio, s1 = p * (1.0f / kAct8Levels) * factor, s2 = (m - p) * (1.0f / kAct8Levels) * factor;
    return {both(s1), both(-128.0f * s1), both(s2), both(fmaf(-192.0f, s2, p * factor))};
}
__device__ __forceinline__ void act8_scaled8(uint2 bytes, const Act8Lines& L, u64* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? bytes.x : bytes.y, j = w & 0x7f7f7f7fu;
        const float f0 = __uint_as_float(__byte_perm(j, 0x43000000u, i & 1 ? 0x7244 : 0x7044));
        const float f1 = __uint_as_float(__byte_perm(j, 0x43000000u, i & 1 ? 0x7344 : 0x7144));
        const u64 f = pack2(f0, f1), c = fma2(f, L.s1, L.z1), t = fma2(f, L.s2, L.z2);
        const float v0 = f0 >= 192.0f ? lo2(t) : lo2(c), v1 = f1 >= 192.0f ? hi2(t) : hi2(c);
        const uint32_t n0 = w << (i & 1 ? 8 : 24), n1 = i & 1 ? w : w << 16;
        v[i] = pack2(__uint_as_float(__float_as_uint(v0) ^ (n0 & 0x80000000u)),
                     __uint_as_float(__float_as_uint(v1) ^ (n1 & 0x80000000u)));
    }
}

// The eight values of eight bytes, in pairs.  A byte permutation puts j = region * 64 + level into
// the upper mantissa of f = 128 + j, so no integer is converted; f * s - 128 * s in one fused operation
// is exact before its one rounding (128 * s is exact, 192 * s would not be), so the products are the
// format's.  Both pieces are formed and one is taken.  Not for ranges above kAct8Big, where 128 * s may
// overflow.
constexpr float kAct8Big = 1.0e38f;
__device__ __forceinline__ void act8_values8(uint2 bytes, const PieceParams& P, u64* v) {
    const u64 s1 = both(P.s1), z1 = both(-128.0f * P.s1), s2 = both(P.s2), z2 = both(-128.0f * P.s2), p = both(P.p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? bytes.x : bytes.y, j = w & 0x7f7f7f7fu;
        const float f0 = __uint_as_float(__byte_perm(j, 0x43000000u, i & 1 ? 0x7244 : 0x7044));
        const float f1 = __uint_as_float(__byte_perm(j, 0x43000000u, i & 1 ? 0x7344 : 0x7144));
        const u64 f = pack2(f0, f1), c = fma2(f, s1, z1);
        const u64 t = add2(fma2(add2(f, both(-64.0f)), s2, z2), p);
        const float v0 = f0 >= 192.0f ? lo2(t) : lo2(c), v1 = f1 >= 192.0f ? hi2(t) : hi2(c);
        const uint32_t n0 = w << (i & 1 ? 8 : 24), n1 = i & 1 ? w : w << 16;
        v[i] = pack2(__uint_as_float(__float_as_uint(v0) ^ (n0 & 0x80000000u)),
                     __uint_as_float(__float_as_uint(v1) ^ (n1 & 0x80000000u)));
    }
}
// The 8 * N values of 8 * N bytes of a group with any range: above kAct8Big the constants are those of
// m / 256 and the values are scaled back, exactly.
template <int N>
__device__ __forceinline__ void act8_decode(const uint2* bytes, float m, float ratio, u64* v) {
    const bool big = m > kAct8Big;
    const PieceParams P = act8_params(big ? m * 0.00390625f : m, ratio);
#pragma unroll
    for (int i = 0; i < N; ++i) act8_values8(bytes[i], P, v + 4 * i);
    if (big)
#pragma unroll
        for (int k = 0; k < 4 * N; ++k) v[k] = mul2(v[k], both(256.0f));
}

}  // namespace pwlq
