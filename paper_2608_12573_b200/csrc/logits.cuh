// Element types of the logits kernels (fp32, bf16, fp16): 16-byte vectors to fp32 values and back, and the scalar
// helpers of a softmax whose statistics are kept in fp32.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace profk {

template <typename T> struct Logit;

template <> struct Logit<float> {
    static __device__ __forceinline__ uint4 masked() { return make_uint4(0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u); }   // all -inf
    // Largest element of a vector in the form in which such maxima are joined cheaply (NaN never wins).
    using Top = float;
    static __device__ __forceinline__ Top top_of(const uint4& v) { return vec_max(v); }
    static __device__ __forceinline__ Top join(Top a, Top b) { return fmaxf(a, b); }
    static __device__ __forceinline__ float value(Top t) { return t; }
    static constexpr int VEC = 4;
    static __device__ __forceinline__ float to_float(float v) { return v; }
    static __device__ __forceinline__ float from_float(float v) { return v; }
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
        x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
    // Largest element (NaN never wins).
    static __device__ __forceinline__ float vec_max(const uint4& v) {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
};

template <> struct Logit<__nv_bfloat16> {
    static __device__ __forceinline__ uint4 masked() { return make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u); }
    using Top = __nv_bfloat162;
    static __device__ __forceinline__ Top top_of(const uint4& v) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
        return __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    }
    static __device__ __forceinline__ Top join(Top a, Top b) { return __hmax2(a, b); }
    static __device__ __forceinline__ float value(Top t) { return fmaxf(__low2float(t), __high2float(t)); }
    static constexpr int VEC = 8;
    static __device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16(v); }
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float vec_max(const uint4& v) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
        const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
};

template <> struct Logit<__half> {
    static __device__ __forceinline__ uint4 masked() { return make_uint4(0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u, 0xFC00FC00u); }
    using Top = __half2;
    static __device__ __forceinline__ Top top_of(const uint4& v) {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
        return __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    }
    static __device__ __forceinline__ Top join(Top a, Top b) { return __hmax2(a, b); }
    static __device__ __forceinline__ float value(Top t) { return fmaxf(__low2float(t), __high2float(t)); }
    static constexpr int VEC = 8;
    static __device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half from_float(float v) { return __float2half(v); }
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(h[i]);
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ float vec_max(const uint4& v) {
        const __half2* h = reinterpret_cast<const __half2*>(&v);
        const __half2 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
        return fmaxf(__low2float(m), __high2float(m));
    }
};

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LOWEST = -3.402823466e38f;      // start of a running maximum: finite, so that -inf - LOWEST is no NaN
constexpr float FAR_BELOW = -1e28f;             // stands in for differences of -inf where they meet a factor of zero (times 2^31 still finite)

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two fp32 lanes in one 64-bit register: the packed forms halve the issue slots of the elementwise arithmetic.
struct F32x2 { unsigned long long v; };
__device__ __forceinline__ F32x2 f2_make(float a, float b) {
    F32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void f2_split(F32x2 x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x.v)); }
__device__ __forceinline__ F32x2 f2_add(F32x2 a, F32x2 b) {
    F32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F32x2 f2_mul(F32x2 a, F32x2 b) {
    F32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F32x2 f2_fma(F32x2 a, F32x2 b, F32x2 c) {
    F32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ uint4 ld_stream_u4(const void* p) { return ld_stream(reinterpret_cast<const uint4*>(p)); }
// ... of memory that the same kernel may write (not through the read-only path).
__device__ __forceinline__ uint4 ld_once_u4(const void* p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void st_stream_u4(void* p, const uint4& v) {
    asm volatile("st.global.L1::no_allocate.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

}  // namespace profk
