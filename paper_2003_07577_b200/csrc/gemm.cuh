// Shared pieces of the real-valued operators (linear.cu, orthogonalize.cu): element types, activations, what happens to a
// sum on its way out.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ebs_internal.cuh"

namespace ebs {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

inline size_t element_size(int dtype) { return dtype == EBS_F32 ? 4 : 2; }
inline bool real_dtype(int dtype) { return dtype == EBS_F32 || dtype == EBS_F16 || dtype == EBS_BF16; }

// The logistic function of v and its complement, neither taken as a difference: both keep their relative accuracy.
__device__ __forceinline__ void logistic(float v, float& s, float& rest) {
    const float t = expf(-fabsf(v)), r = 1.0f / (1.0f + t), tr = t * r;
    s = v >= 0.0f ? r : tr;
    rest = v >= 0.0f ? tr : r;
}
// act(z) and act'(z) as include/ebs.h states them.  (1 + tanh u) / 2 is the logistic function of 2u.
__device__ __forceinline__ float activation(float z, int act) {
    switch (act) {
        case EBS_ACT_RELU: return z > 0.0f ? z : 0.0f;
        case EBS_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678f));
        case EBS_ACT_GELU_TANH: return z / (1.0f + expf(-1.59576912f * (z + 0.044715f * z * z * z)));
        case EBS_ACT_SILU: return z / (1.0f + expf(-z));
        default: return z;
    }
}
__device__ __forceinline__ float activation_slope(float z, int act) {
    float s, rest;
    switch (act) {
        case EBS_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
        case EBS_ACT_GELU: return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * (0.39894228f * expf(-0.5f * z * z));
        case EBS_ACT_GELU_TANH:
            logistic(1.59576912f * (z + 0.044715f * z * z * z), s, rest);
            return s * (1.0f + z * rest * (1.59576912f * (1.0f + 0.134145f * z * z)));
        case EBS_ACT_SILU:
            logistic(z, s, rest);
            return s * (1.0f + z * rest);
        default: return 1.0f;
    }
}

// What becomes of the sum v of output (row, col).
//   linear:  z = v + bias[col]; y = act(z) + residual
//   otherwise: y = alpha * v + beta * c   (c fp32, read at the output's place)
struct GemmOut {
    const void* bias = nullptr;
    const void* residual = nullptr;
    void* z = nullptr;
    void* y = nullptr;
    const float* c = nullptr;
    long long ldr = 0, ldz = 0, ldy = 0, batch_y = 0;   // batch_y: elements between the matrices of a batch (y and c)
    float alpha = 1.0f, beta = 0.0f;
    int act = EBS_ACT_NONE;
};

template <typename T>
__device__ __forceinline__ void gemm_store(const GemmOut& o, int batch, long long row, int col, float v) {
    const long long at = batch * o.batch_y + row * o.ldy + col;
    if (o.c) v = o.alpha * v + o.beta * o.c[at];
    else if (o.alpha != 1.0f) v *= o.alpha;
    if (o.bias) v += to_f32(static_cast<const T*>(o.bias)[col]);
    if (o.z) static_cast<T*>(o.z)[row * o.ldz + col] = from_f32<T>(v);
    if (o.act) v = activation(v, o.act);
    if (o.residual) v += to_f32(static_cast<const T*>(o.residual)[row * o.ldr + col]);
    static_cast<T*>(o.y)[at] = from_f32<T>(v);
}

// D[i][j] = sum_r A(i, r) B(r, j) over elements at a[i * a_row + r * a_red] and b[j * b_col + r * b_red].
struct GemmIn {
    const void *a, *b;
    long long a_row, a_red, b_col, b_red, batch_a = 0, batch_b = 0;
    int rows, cols, red, batch = 1;
};

// dtype: type of both operands, out_dtype: of y, z, bias and residual.
int launch_gemm(const GemmIn& in, const GemmOut& out, int dtype, int out_dtype, cudaStream_t st);

}  // namespace ebs
