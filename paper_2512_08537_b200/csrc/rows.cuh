// Rows of 16- or 32-bit values as the aligned 16-byte pieces inside them, for the kernels that take rows of logits.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/ardiff.h"

namespace ardiff {

template <typename T> struct Piece { static constexpr int N = 16 / (int)sizeof(T); };   // values a piece

// A piece of a row. The kernels are launched early: the one that writes the logits may still run when they start, and the gradient may lie
// where the logits do. So these are ordinary loads, which stay behind begin_kernel(): read-only ones (__ldg, or through __restrict__) want data
// that does not change while the kernel runs and may be moved in front of it.
__device__ __forceinline__ uint4 load_piece(const uint4* p) { return *p; }

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ void unpack(const uint4& p, float (&v)[4], float) {
    v[0] = __uint_as_float(p.x); v[1] = __uint_as_float(p.y); v[2] = __uint_as_float(p.z); v[3] = __uint_as_float(p.w);
}
__device__ __forceinline__ void unpack(const uint4& p, float (&v)[8], __nv_bfloat16) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void unpack(const uint4& p, float (&v)[8], __half) {
    const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 h = *reinterpret_cast<const __half2*>(&w[i]);
        const float2 f = __half22float2(h);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
// Values h .. h + 3 of a piece, h a multiple of 4.
__device__ __forceinline__ void unpack4(const uint4& p, int, float (&v)[4], float) { unpack(p, v, 0.f); }
__device__ __forceinline__ void unpack4(const uint4& p, int h, float (&v)[4], __nv_bfloat16) {
    const uint32_t a = h ? p.z : p.x, b = h ? p.w : p.y;
    v[0] = __uint_as_float(a << 16);
    v[1] = __uint_as_float(a & 0xffff0000u);
    v[2] = __uint_as_float(b << 16);
    v[3] = __uint_as_float(b & 0xffff0000u);
}
__device__ __forceinline__ void unpack4(const uint4& p, int h, float (&v)[4], __half) {
    const uint32_t a = h ? p.z : p.x, b = h ? p.w : p.y;
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&a)), y = __half22float2(*reinterpret_cast<const __half2*>(&b));
    v[0] = x.x;
    v[1] = x.y;
    v[2] = y.x;
    v[3] = y.y;
}

// The largest value of a piece; NaN if one is.
__device__ __forceinline__ float piece_max(const uint4& p, float) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(p.x)), "f"(__uint_as_float(p.y)));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(r) : "f"(__uint_as_float(p.z)));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(r) : "f"(__uint_as_float(p.w)));
    return r;
}
__device__ __forceinline__ float piece_max(const uint4& p, __nv_bfloat16) {
    uint32_t a, b;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(p.x), "r"(p.y));
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(p.z), "r"(p.w));
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(a << 16)), "f"(__uint_as_float(a & 0xffff0000u)));
    return r;
}
__device__ __forceinline__ float piece_max(const uint4& p, __half) {
    uint32_t a, b;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(a) : "r"(p.x), "r"(p.y));
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(b) : "r"(p.z), "r"(p.w));
    asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&a));
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(f.x), "f"(f.y));
    return r;
}
__device__ __forceinline__ uint4 pack(const float (&v)[4], float) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 pack(const float (&v)[8], __nv_bfloat16) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack(const float (&v)[8], __half) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// A row of V values: `lead` values before the first 16-byte boundary, `pieces` whole pieces, the rest.
template <typename T> struct Row {
    const T* x;
    int V, lead, pieces;
    __device__ __forceinline__ Row(const T* row, int v) : x(row), V(v) {
        lead = min(v, (int)(((16u - (unsigned)(reinterpret_cast<uintptr_t>(row) & 15u)) & 15u) / sizeof(T)));
        pieces = (v - lead) / Piece<T>::N;
    }
    __device__ __forceinline__ const uint4* body() const { return reinterpret_cast<const uint4*>(x + lead); }
    __device__ __forceinline__ int tail() const { return lead + pieces * Piece<T>::N; }    // the first value behind the pieces
};

// A value's place in the host's list of types; 0 for one that there is none of.
inline int value_size(int32_t dtype) {
    return dtype == ARDIFF_F32 ? 4 : dtype == ARDIFF_BF16 || dtype == ARDIFF_F16 ? 2 : 0;
}

__device__ __forceinline__ float ex2(float y) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
    return r;
}

// Two fp32 values in a register pair, and the instructions that take them as one.
struct Two {
    unsigned long long v;
};
__device__ __forceinline__ Two two(float a, float b) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 apart(Two a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ Two operator+(Two a, Two b) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Two operator*(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}

}  // namespace ardiff
