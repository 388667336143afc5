// Newton-Schulz orthogonalisation of update matrices.  See include/ebs.h.
#include <math.h>

#include "gemm_tile.cuh"

namespace ebs {

static size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }

// Matrices are kept as two fp16 planes hi + lo (22 bits) times a power of two: X by 2^-ex, its Gram matrix A by 2^-ea and
// B = b A + c A^2 by 2^-eb, chosen from bounds of the singular values so that no entry leaves fp16 (an entry is at most the
// largest singular value).
// Sums of squares in 64 bits, a part of each matrix a thread block (blockIdx.y: the matrix), in an order that depends on sizes alone.
template <typename T>
__global__ void __launch_bounds__(256) sum_squares_kernel(const T* __restrict__ g, long long count, double* __restrict__ part) {
    __shared__ double sums[8];
    g += blockIdx.y * count;
    double s = 0.0;
#pragma unroll 4
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < count; i += gridDim.x * 256LL) { const double v = to_f32(g[i]); s += v * v; }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) s += sums[i];
        part[blockIdx.y * gridDim.x + blockIdx.x] = s;
    }
}
// X = G / (|G|_F + eps), times `store`, as planes; parts: thread blocks of sum_squares_kernel a matrix.
template <typename T>
__global__ void __launch_bounds__(256) normalize_kernel(const T* __restrict__ g, int rows, int cols, float eps, float store, const double* __restrict__ part, int parts,
                                                        __half* __restrict__ x, long long ld, long long plane) {
    g += (long long)blockIdx.z * rows * cols;
    x += blockIdx.z * 2 * plane;
    double s = 0.0;
    for (int i = 0; i < parts; ++i) s += part[blockIdx.z * parts + i];
    const double inv = store / (sqrt(s) + (double)eps);
    for (int r = blockIdx.y; r < rows; r += gridDim.y)
        for (int c = blockIdx.x * 256 + threadIdx.x; c < cols; c += gridDim.x * 256) {
            const float v = (float)(to_f32(g[(long long)r * cols + c]) * inv);
            const __half hi = __float2half_rn(v);
            x[r * ld + c] = hi;
            x[plane + r * ld + c] = __float2half_rn(v - __half2float(hi));
        }
}
template <typename T>
static void launch_normalize(const void* g, int batch, int rows, int cols, float eps, float store, double* part, int parts, __half* x, long long ld, long long plane,
                             cudaStream_t st) {
    sum_squares_kernel<T><<<dim3(parts, batch), 256, 0, st>>>(static_cast<const T*>(g), (long long)rows * cols, part);
    const dim3 grid((cols + 255) / 256, rows < 1024 ? rows : 1024, batch);
    normalize_kernel<T><<<grid, 256, 0, st>>>(static_cast<const T*>(g), rows, cols, eps, store, part, parts, x, ld, plane);
}
template <typename T>
__global__ void __launch_bounds__(256) scale_out_kernel(const __half* x, long long ld, long long plane, int rows, int cols, int batch, float scale, T* out) {
    const long long count = (long long)rows * cols, total = count * batch;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < total; i += gridDim.x * 256LL) {
        const long long b = i / count, r = i % count, at = b * 2 * plane + r / cols * ld + r % cols;
        out[i] = from_f32<T>(scale * (__half2float(x[at]) + __half2float(x[plane + at])));
    }
}

// The largest singular value a step can give from singular values in 0 .. s, and the largest of |b v + c v^2|, v in 0 .. s^2 (b A + c A^2).
static void step_bounds(const float* c, double s, double* next, double* inner) {
    double top = 0.0, in = 0.0;
    for (int j = 1; j <= 4096; ++j) {
        const double v = s * j / 4096.0, v2 = v * v, q = fabs(v2 * (c[1] + v2 * (double)c[2])), p = fabs(v * (c[0] + v2 * (c[1] + v2 * (double)c[2])));
        top = p > top ? p : top;
        in = q > in ? q : in;
    }
    *next = top;
    *inner = in;
}
// The exponent e with v * 2^e in [2^13, 2^14): a factor of four below fp16's largest value for what roundings add to the bounds.
static int headroom(double v) { int e; frexp(v > 0.0 ? v : 1.0, &e); return 14 - e; }

struct OrthoBuffers {
    long long ld, plane, side_ld, side_plane;
    size_t x, a, part, total;
    int parts;                                                // sums of squares a matrix
};
static OrthoBuffers ortho_buffers(int batch, int rows, int cols) {
    const long long side = rows < cols ? rows : cols;
    OrthoBuffers b;
    b.ld = (cols + 7) & ~7LL;
    b.plane = b.ld * rows;
    b.side_ld = (side + 7) & ~7LL;
    b.side_plane = b.side_ld * side;
    b.x = round256((size_t)batch * 2 * b.plane * 2);
    b.a = round256((size_t)batch * 2 * b.side_plane * 2);
    const long long parts = ((long long)rows * cols + 8191) / 8192;
    b.parts = (int)(parts < 128 ? parts : 128);
    b.part = round256((size_t)batch * b.parts * 8);
    b.total = 2 * b.x + 2 * b.a + b.part;
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
    // singular values before each step, and the exponents of X, A and B
    double bound = 1.0;
    int ex[65], eb[64];
    for (int i = 0; i <= steps; ++i) {
        if (!(bound < 0x1p20 && bound > 0x1p-20)) return EBS_ERR_UNSUPPORTED;
        ex[i] = headroom(bound);
        if (i == steps) break;
        double next, inner;
        step_bounds(coeff, bound, &next, &inner);
        eb[i] = headroom(inner) < 60 ? headroom(inner) : 60;
        bound = next;
    }
    const OrthoBuffers b = ortho_buffers(batch, rows, cols);
    if (workspace_bytes < b.total) return EBS_ERR_INVALID_ARG;
    const size_t bytes = (size_t)batch * rows * cols * element_size(dtype);
    const uintptr_t pg = (uintptr_t)g, po = (uintptr_t)out, pw = (uintptr_t)workspace;
    if (pg != po && pg < po + bytes && po < pg + bytes) return EBS_ERR_INVALID_ARG;
    if ((pw < pg + bytes && pg < pw + b.total) || (pw < po + bytes && po < pw + b.total)) return EBS_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    __half* x = static_cast<__half*>(workspace);
    __half* x2 = reinterpret_cast<__half*>(static_cast<char*>(workspace) + b.x);
    __half* A = reinterpret_cast<__half*>(static_cast<char*>(workspace) + 2 * b.x);
    __half* B = reinterpret_cast<__half*>(static_cast<char*>(workspace) + 2 * b.x + b.a);
    const float first = ldexpf(1.0f, ex[0]);
    double* part = reinterpret_cast<double*>(static_cast<char*>(workspace) + 2 * b.x + 2 * b.a);
    if (dtype == EBS_F32) launch_normalize<float>(g, batch, rows, cols, eps, first, part, b.parts, x, b.ld, b.plane, st);
    else if (dtype == EBS_F16) launch_normalize<__half>(g, batch, rows, cols, eps, first, part, b.parts, x, b.ld, b.plane, st);
    else launch_normalize<__nv_bfloat16>(g, batch, rows, cols, eps, first, part, b.parts, x, b.ld, b.plane, st);
    if ((rc = check_cuda(cudaGetLastError()))) return rc;
    const bool tall = rows > cols;                            // then X X^T X is taken as X (X^T X): the smaller product
    const int m = tall ? cols : rows, n = tall ? rows : cols;
    for (int s = 0; s < steps; ++s) {
        // A 2^ea = X^T X or X X^T
        const GemmOperand xs{x, b.ld, tall, 2, b.plane, 2 * b.plane}, as{A, b.side_ld, false, 2, b.side_plane, 2 * b.side_plane}, bs{B, b.side_ld, false, 2, b.side_plane, 2 * b.side_plane};
        const int ea = 2 * ex[s] - 14;                          // entries of A are at most the square of X's bound: below 2^14
        PlanesOut oa{A, nullptr, b.side_ld, b.side_plane, 2 * b.side_plane, 0, 0, 0, ldexpf(1.0f, ea - 2 * ex[s]), 0.0f};
        if ((rc = launch_gemm(xs, xs, GemmShape{m, m, n, batch}, oa, st))) return rc;
        // B 2^eb = b A + c A^2  (A is symmetric: its rows are its columns)
        PlanesOut ob{B, A, b.side_ld, b.side_plane, 2 * b.side_plane, b.side_ld, b.side_plane, 2 * b.side_plane, coeff[2] * ldexpf(1.0f, eb[s] - 2 * ea), coeff[1] * ldexpf(1.0f, eb[s] - ea)};
        if ((rc = launch_gemm(as, as, GemmShape{m, m, m, batch}, ob, st))) return rc;
        // X 2^ex' = a X + B X or a X + X B
        PlanesOut ox{x2, x, b.ld, b.plane, 2 * b.plane, b.ld, b.plane, 2 * b.plane, ldexpf(1.0f, ex[s + 1] - eb[s] - ex[s]), coeff[0] * ldexpf(1.0f, ex[s + 1] - ex[s])};
        const GemmOperand xk{x, b.ld, false, 2, b.plane, 2 * b.plane}, xm{x, b.ld, true, 2, b.plane, 2 * b.plane};
        if ((rc = tall ? launch_gemm(xk, bs, GemmShape{rows, cols, m, batch}, ox, st) : launch_gemm(bs, xm, GemmShape{rows, cols, m, batch}, ox, st))) return rc;
        __half* t = x; x = x2; x2 = t;
    }
    const long long total = (long long)rows * cols * batch, blocks = (total + 255) / 256;
    const int grid = (int)(blocks < 148 * 16 ? blocks : 148 * 16);
    const float last = scale * ldexpf(1.0f, -ex[steps]);
    if (dtype == EBS_F32) scale_out_kernel<float><<<grid, 256, 0, st>>>(x, b.ld, b.plane, rows, cols, batch, last, static_cast<float*>(out));
    else if (dtype == EBS_F16) scale_out_kernel<__half><<<grid, 256, 0, st>>>(x, b.ld, b.plane, rows, cols, batch, last, static_cast<__half*>(out));
    else scale_out_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(x, b.ld, b.plane, rows, cols, batch, last, static_cast<__nv_bfloat16*>(out));
    return check_cuda(cudaGetLastError());
}

}  // extern "C"
