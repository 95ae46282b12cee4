// Element types of logits and gradients: 16-byte vectors of them, and single ones.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <string.h>
#include <type_traits>

#include "common.cuh"
#include "sr_train.h"

namespace sr {

// Kernels here read with plain loads and with these.  What the compiler may take for constant while the kernel runs (__ldg, const
// __restrict__) it may also load before grid_begin() has waited for the kernel that writes it: the first row start of a batch was
// read too early that way.  Statements that are volatile stay in their order.
__device__ __forceinline__ uint4 load_once(const uint4* p) {            // not read again soon
    uint4 v;
    asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void store_once(uint4* p, const uint4& v) { __stcs(p, v); }

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x);             // to nearest even
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// Two fp32 numbers in one register pair: one instruction for both, each rounded as by itself.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 two(float lo, float hi) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ f32x2 two(float x) { return two(x, x); }
__device__ __forceinline__ float low_of(f32x2 x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float high_of(f32x2 x) { return __uint_as_float((uint32_t)(x >> 32)); }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// The elements of a 16-byte vector, in order.
template <typename T>
struct Vec {
    static constexpr int kElems = 16 / (int)sizeof(T);
};
__device__ __forceinline__ void unpack(const uint4& v, float (&x)[4], float) {
    x[0] = __uint_as_float(v.x); x[1] = __uint_as_float(v.y); x[2] = __uint_as_float(v.z); x[3] = __uint_as_float(v.w);
}
__device__ __forceinline__ void unpack(const uint4& v, float (&x)[8], __nv_bfloat16) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        x[2 * k] = __uint_as_float(w[k] << 16);
        x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void unpack(const uint4& v, float (&x)[8], __half) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        __half2 h;
        memcpy(&h, &w[k], 4);
        const float2 f = __half22float2(h);
        x[2 * k] = f.x;
        x[2 * k + 1] = f.y;
    }
}
__device__ __forceinline__ uint4 pack(const float (&x)[4], float) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ uint4 pack(const float (&x)[8], __nv_bfloat16) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
        memcpy(&w[k], &h, 4);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack(const float (&x)[8], __half) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const __half2 h = __floats2half2_rn(x[2 * k], x[2 * k + 1]);
        memcpy(&w[k], &h, 4);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Largest elements of vectors, a NaN only where there is nothing else: kept packed as long as more come.
template <typename T>
struct VecMax;
template <>
struct VecMax<float> {
    float m;
    __device__ __forceinline__ explicit VecMax(float first) : m(first) {}
    __device__ __forceinline__ void take(const uint4& v) {
        m = fmaxf(fmaxf(m, fmaxf(__uint_as_float(v.x), __uint_as_float(v.y))), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    __device__ __forceinline__ float value() const { return m; }
};
template <>
struct VecMax<__nv_bfloat16> {
    __nv_bfloat162 m;
    __device__ __forceinline__ explicit VecMax(float first) : m(__float2bfloat162_rn(first)) {}
    __device__ __forceinline__ void take(const uint4& v) {
        __nv_bfloat162 h[4];
        memcpy(h, &v, 16);
        m = __hmax2(m, __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
    }
    __device__ __forceinline__ float value() const { return fmaxf(__low2float(m), __high2float(m)); }
};
template <>
struct VecMax<__half> {
    __half2 m;
    __device__ __forceinline__ explicit VecMax(float first) : m(__float2half2_rn(first)) {}
    __device__ __forceinline__ void take(const uint4& v) {
        __half2 h[4];
        memcpy(h, &v, 16);
        m = __hmax2(m, __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3])));
    }
    __device__ __forceinline__ float value() const { return fmaxf(__low2float(m), __high2float(m)); }
};

inline int dtype_bytes(int32_t dtype) { return dtype == SR_DTYPE_F32 ? 4 : dtype == SR_DTYPE_BF16 || dtype == SR_DTYPE_F16 ? 2 : 0; }

// logprob.cu
struct LogitsArgs {
    const void* logits;
    int32_t dtype, n_tokens, vocab;
    int64_t pitch;
    const int32_t* targets;
    double temperature;
};
int launch_token_logprob(const LogitsArgs& a, float* logp, float* row_stats, float* entropy, int32_t* status, cudaStream_t s);
int launch_token_logprob_backward(const LogitsArgs& a, const float* row_stats, const float* entropy, const float* d_logp, const float* d_entropy, void* d_logits,
                                  int64_t d_pitch, cudaStream_t s);

// grads.cu
constexpr int kGradPiece = 16384;    // bytes of a tensor that a CTA takes at a time; pieces of a call are numbered in 32 bits: 32 TB
inline int64_t grad_pieces(int64_t count, int32_t dtype) {      // count >= 0
    const int64_t per = kGradPiece / dtype_bytes(dtype);
    return count / per + (count % per != 0);
}
size_t grad_norm_workspace_bytes(int32_t n_tensors);
int launch_grad_norm(const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t n_tensors, float* norm, void* ws, cudaStream_t s);
int launch_clip_grads(const void* const* grads, const int64_t* counts, const int32_t* dtypes, int32_t n_tensors, const float* norm, float max_norm,
                      void* const* out, int32_t* status, cudaStream_t s);

}  // namespace sr
