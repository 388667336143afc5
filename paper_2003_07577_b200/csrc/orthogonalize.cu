// Newton-Schulz orthogonalisation of update matrices.  See include/ebs.h.
#include <math.h>

#include "gemm.cuh"

namespace ebs {

static size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }

// X = G / (|G|_F + eps), one thread block a matrix, the sum of squares in 64 bits in a fixed order.
template <typename T>
__global__ void __launch_bounds__(1024) normalize_kernel(const T* g, long long count, float eps, float* x) {
    __shared__ double part[1024];
    g += blockIdx.x * count;
    x += blockIdx.x * count;
    double s = 0.0;
    for (long long i = threadIdx.x; i < count; i += 1024) { const double v = to_f32(g[i]); s += v * v; }
    part[threadIdx.x] = s;
    __syncthreads();
    for (int o = 512; o > 0; o >>= 1) {
        if (threadIdx.x < o) part[threadIdx.x] += part[threadIdx.x + o];
        __syncthreads();
    }
    const double inv = 1.0 / (sqrt(part[0]) + (double)eps);
    for (long long i = threadIdx.x; i < count; i += 1024) x[i] = (float)(to_f32(g[i]) * inv);
}
template <typename T>
__global__ void __launch_bounds__(256) scale_out_kernel(const float* x, long long count, float scale, T* out) {
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < count; i += gridDim.x * 256LL) out[i] = from_f32<T>(scale * x[i]);
}

// Bounds of the singular values after every step; false if they could leave 2^-60 .. 2^60.
static bool bounded(int steps, const float* c) {
    double s = 1.0;
    for (int i = 0; i < steps; ++i) {
        double top = 0.0;
        for (int j = 1; j <= 4096; ++j) {
            const double v = s * j / 4096.0, v2 = v * v, p = fabs(v * (c[0] + v2 * (c[1] + v2 * (double)c[2])));
            top = p > top ? p : top;
        }
        s = top;
        if (!(s < 0x1p60 && s > 0x1p-60)) return false;
    }
    return true;
}

struct OrthoBuffers {
    size_t x, a, total;
};
static OrthoBuffers ortho_buffers(int batch, int rows, int cols) {
    const size_t side = rows < cols ? rows : cols;
    OrthoBuffers b;
    b.x = round256((size_t)batch * rows * cols * 4);
    b.a = round256((size_t)batch * side * side * 4);
    b.total = 2 * b.x + 2 * b.a;
    return b;
}
static int check_shape(int batch, int rows, int cols, int dtype, int steps) {
    if (batch < 1 || rows < 1 || cols < 1 || !real_dtype(dtype) || steps < 0 || steps > 64) return EBS_ERR_INVALID_ARG;
    if (batch > 65535 || (long long)rows * cols > (1LL << 36) / batch) return EBS_ERR_OVERFLOW;
    return EBS_OK;
}

}  // namespace ebs

using namespace ebs;

extern "C" {

size_t ebs_orthogonalize_workspace_bytes(int batch, int rows, int cols, int dtype, int steps) {
    if (check_shape(batch, rows, cols, dtype, steps)) return 0;
    return ortho_buffers(batch, rows, cols).total;
}

int ebs_orthogonalize(const void* g, int batch, int rows, int cols, int dtype, int steps, const float* coeff, float eps, float scale, void* out,
                      void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_shape(batch, rows, cols, dtype, steps);
    if (rc) return rc;
    if (!g || !out || !workspace || !coeff || !(eps >= 0.0f) || !isfinite(eps) || !isfinite(scale)) return EBS_ERR_INVALID_ARG;
    if (((uintptr_t)g & 15) || ((uintptr_t)out & 15) || ((uintptr_t)workspace & 15)) return EBS_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (!isfinite(coeff[i])) return EBS_ERR_INVALID_ARG;
    if (!bounded(steps, coeff)) return EBS_ERR_UNSUPPORTED;
    const OrthoBuffers b = ortho_buffers(batch, rows, cols);
    if (workspace_bytes < b.total) return EBS_ERR_INVALID_ARG;
    const size_t bytes = (size_t)batch * rows * cols * element_size(dtype);
    const uintptr_t pg = (uintptr_t)g, po = (uintptr_t)out, pw = (uintptr_t)workspace;
    if (pg != po && pg < po + bytes && po < pg + bytes) return EBS_ERR_INVALID_ARG;
    if ((pw < pg + bytes && pg < pw + b.total) || (pw < po + bytes && po < pw + b.total)) return EBS_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    float* x = static_cast<float*>(workspace);
    float* x2 = reinterpret_cast<float*>(static_cast<char*>(workspace) + b.x);
    float* A = reinterpret_cast<float*>(static_cast<char*>(workspace) + 2 * b.x);
    float* B = reinterpret_cast<float*>(static_cast<char*>(workspace) + 2 * b.x + b.a);
    const long long count = (long long)rows * cols;
    if (dtype == EBS_F32) normalize_kernel<float><<<batch, 1024, 0, st>>>(static_cast<const float*>(g), count, eps, x);
    else if (dtype == EBS_F16) normalize_kernel<__half><<<batch, 1024, 0, st>>>(static_cast<const __half*>(g), count, eps, x);
    else normalize_kernel<__nv_bfloat16><<<batch, 1024, 0, st>>>(static_cast<const __nv_bfloat16*>(g), count, eps, x);
    if ((rc = check_cuda(cudaGetLastError()))) return rc;
    const bool tall = rows > cols;                            // then X X^T X is taken as X (X^T X): the smaller product
    const int m = tall ? cols : rows, n = tall ? rows : cols;
    const long long sq = (long long)m * m;
    for (int s = 0; s < steps; ++s) {
        const long long mi = tall ? 1 : cols, ni = tall ? cols : 1;      // element strides of the short and the long side
        GemmIn ga{x, x, mi, ni, mi, ni, count, count, m, m, n, batch};
        GemmOut oa;
        oa.y = A; oa.ldy = m; oa.batch_y = sq;
        if ((rc = launch_gemm(ga, oa, EBS_F32, EBS_F32, st))) return rc;
        GemmIn gb{A, A, m, 1, 1, m, sq, sq, m, m, m, batch};
        GemmOut ob;
        ob.y = B; ob.ldy = m; ob.batch_y = sq; ob.c = A; ob.alpha = coeff[2]; ob.beta = coeff[1];
        if ((rc = launch_gemm(gb, ob, EBS_F32, EBS_F32, st))) return rc;
        GemmIn gx = tall ? GemmIn{x, B, cols, 1, m, 1, count, sq, rows, cols, m, batch} : GemmIn{B, x, m, 1, 1, cols, sq, count, rows, cols, m, batch};
        GemmOut ox;
        ox.y = x2; ox.ldy = cols; ox.batch_y = count; ox.c = x; ox.alpha = 1.0f; ox.beta = coeff[0];
        if ((rc = launch_gemm(gx, ox, EBS_F32, EBS_F32, st))) return rc;
        float* t = x; x = x2; x2 = t;
    }
    const long long total = count * batch, blocks = (total + 255) / 256;
    const int grid = (int)(blocks < 148 * 16 ? blocks : 148 * 16);
    if (dtype == EBS_F32) scale_out_kernel<float><<<grid, 256, 0, st>>>(x, total, scale, static_cast<float*>(out));
    else if (dtype == EBS_F16) scale_out_kernel<__half><<<grid, 256, 0, st>>>(x, total, scale, static_cast<__half*>(out));
    else scale_out_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(x, total, scale, static_cast<__nv_bfloat16*>(out));
    return check_cuda(cudaGetLastError());
}

}  // extern "C"
