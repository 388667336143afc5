// Newton-Schulz orthogonalisation of update matrices.  See include/ebs.h.
#include <math.h>

#include "orthogonalize.cuh"

namespace ebs {

static size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }

// A step is three products: the Gram matrix A of X, Q = a I + A (b I + c A), and X <- Q X.  What is added to a product lies on its
// diagonal, so that no product reads anything beside its operands: A and b I + c A leave the first one together.  The first two are
// symmetric; half of each is summed.
// Matrices are kept as two fp16 planes hi + lo (22 bits) times a power of two each, chosen from bounds of the singular values so that
// no entry leaves fp16 (an entry is at most the largest singular value).
// Elements i .. i + N - 1 of a dense matrix of `count`, one 16-byte access where they all exist and it is aligned.
template <typename T>
__device__ __forceinline__ void load_elements(const T* p, long long left, bool vec, float (&v)[Pack<T>::N]) {
    if (vec && left >= Pack<T>::N) load_pack(p, v);
    else
#pragma unroll
        for (int e = 0; e < Pack<T>::N; ++e) v[e] = e < left ? to_f32(p[e]) : 0.0f;
}
// Sums of squares in 64 bits, a part of each matrix a thread block (blockIdx.y: the matrix), in an order that depends on sizes alone.
template <typename T>
__global__ void __launch_bounds__(256) sum_squares_kernel(const T* __restrict__ g, long long count, int vec, double* __restrict__ part) {
    __shared__ double sums[8];
    constexpr int N = Pack<T>::N;
    let_next_kernel_start();
    wait_for_previous_kernel();
    g += blockIdx.y * count;
    double s = 0.0;
    const long long step = gridDim.x * 256LL * N;
#pragma unroll 4
    for (long long i = (blockIdx.x * 256LL + threadIdx.x) * N; i < count; i += step) {
        float v[N];
        load_elements(g + i, count - i, vec, v);
#pragma unroll
        for (int e = 0; e < N; ++e) s = fma((double)v[e], (double)v[e], s);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) s += sums[i];
        part[blockIdx.y * gridDim.x + blockIdx.x] = s;
    }
}
// The sum of a matrix's parts, the same in every thread of a block.
__device__ __forceinline__ double total_of(const double* part, int parts) {
    __shared__ double total;
    if (threadIdx.x < 32) {
        double s = 0.0;
        for (int i = threadIdx.x; i < parts; i += 32) s += part[i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (threadIdx.x == 0) total = s;
    }
    __syncthreads();
    return total;
}
// X = G / (|G|_F + eps), times `store`, as planes; parts: thread blocks of sum_squares_kernel a matrix.
template <typename T>
__global__ void __launch_bounds__(256) normalize_kernel(const T* __restrict__ g, int rows, int cols, int vec, float eps, float store, const double* __restrict__ part, int parts,
                                                        __half* __restrict__ x, long long ld, long long plane) {
    constexpr int N = Pack<T>::N;
    let_next_kernel_start();
    wait_for_previous_kernel();
    g += (long long)blockIdx.y * rows * cols;
    x += blockIdx.y * 2 * plane;
    const double inv = store / (sqrt(total_of(part + (size_t)blockIdx.y * parts, parts)) + (double)eps);
    const int per_row = (cols + N - 1) / N;
    const long long items = (long long)per_row * rows, step = gridDim.x * 256LL;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < items; i += step) {
        const int r = (int)(i / per_row), c = (int)(i - (long long)r * per_row) * N;
        float v[N];
        load_elements(g + (long long)r * cols + c, cols - c, vec, v);
        __align__(16) uint32_t hi[N / 2], lo[N / 2];
#pragma unroll
        for (int e = 0; e < N; e += 2) split_pair((float)(v[e] * inv), (float)(v[e + 1] * inv), hi[e / 2], lo[e / 2]);
        __half* to = x + r * ld + c;                          // (rows of the planes are padded to whole groups of eight)
        if constexpr (N == 8) {
            *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(hi);
            *reinterpret_cast<uint4*>(to + plane) = *reinterpret_cast<const uint4*>(lo);
        } else {
            *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(hi);
            *reinterpret_cast<uint2*>(to + plane) = *reinterpret_cast<const uint2*>(lo);
        }
    }
}
static int blocks_for(long long items, int batch) {            // of 256 items, about eight an SM
    const long long b = (items + 255) / 256, most = (8LL * 148 + batch - 1) / batch;
    return (int)(b < most ? b : most);
}
template <typename T>
static int launch_normalize(const void* g, int batch, int rows, int cols, float eps, float store, double* part, int parts, __half* x, long long ld, long long plane,
                            cudaStream_t st) {
    constexpr int N = Pack<T>::N;
    const long long count = (long long)rows * cols;
    const int rc = launch_chained(sum_squares_kernel<T>, dim3(parts, batch), 256, 0, st, 1, static_cast<const T*>(g), count, (int)(count % N == 0), part);
    if (rc) return rc;
    const int vec = cols % N == 0;
    return launch_chained(normalize_kernel<T>, dim3(blocks_for((long long)rows * ((cols + N - 1) / N), batch), batch), 256, 0, st, 1, static_cast<const T*>(g), rows, cols, vec, eps,
                          store, (const double*)part, parts, x, ld, plane);
}
// out = scale * X, for no steps at all.
template <typename T>
__global__ void __launch_bounds__(256) scale_out_kernel(const __half* x, long long ld, long long plane, int rows, int cols, int batch, float scale, T* out) {
    let_next_kernel_start();
    wait_for_previous_kernel();
    const long long count = (long long)rows * cols, total = count * batch;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < total; i += gridDim.x * 256LL) {
        const long long b = i / count, r = i % count, at = b * 2 * plane + r / cols * ld + r % cols;
        out[i] = from_f32<T>(scale * (__half2float(x[at]) + __half2float(x[plane + at])));
    }
}

// For singular values in 0 .. s: the largest a step can give, and the largest entries of b + c v and a + b v + c v^2, v in 0 .. s^2.
struct StepBounds {
    double next, linear, square;
};
static StepBounds step_bounds(const float* coeff, double s) {
    const double a = coeff[0], b = coeff[1], c = coeff[2], top = s * s;
    StepBounds r = {0.0, fmax(fabs(b), fabs(b + c * top)), fmax(fabs(a), fabs(a + top * (b + c * top)))};
    auto inner = [&](double u) { return u > 0.0 && u < top; };
    auto step = [&](double u) { r.next = fmax(r.next, sqrt(u) * fabs(a + u * (b + c * u))); };      // u: a singular value squared
    if (c != 0.0 && inner(-b / (2.0 * c))) r.square = fmax(r.square, fabs(a - b * b / (4.0 * c)));
    step(top);                                                // the extremes: the end, and where a + 3 b u + 5 c u^2 = 0
    const double disc = 9.0 * b * b - 20.0 * a * c;
    if (c != 0.0 && disc >= 0.0)
        for (int sign = -1; sign <= 1; sign += 2) {
            const double u = (-3.0 * b + sign * sqrt(disc)) / (10.0 * c);
            if (inner(u)) step(u);
        }
    if (b != 0.0 && inner(-a / (3.0 * b))) step(-a / (3.0 * b));   // (c = 0, or next to it)
    return r;
}
// The exponent e with v * 2^e in [2^13, 2^14): a factor of four below fp16's largest value for what roundings add to the bounds.
// (At most 2^60: coefficients next to zero.)
static int headroom(double v) {
    int e;
    frexp(v > 0x1p-46 ? v : 0x1p-46, &e);
    return 14 - e;
}

struct OrthoBuffers {
    long long ld, plane, side_ld, side_plane;
    size_t x, a, part, scratch, total;
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
    const long long parts = ((long long)rows * cols + 4095) / 4096, most = (4LL * 148 + batch - 1) / batch;
    b.parts = (int)(parts < most ? parts : most);
    b.part = round256((size_t)batch * b.parts * 8);
    b.scratch = 0;                                            // of the products' partial sums; they run one after the other
    const int m = (int)side, n = rows < cols ? cols : rows;
    const GemmShape shapes[] = {{m, m, n, batch, true}, {m, m, m, batch, true}, {rows, cols, m, batch}};
    for (const GemmShape& s : shapes) { const size_t need = round256(gemm_route(s, 2).scratch); b.scratch = need > b.scratch ? need : b.scratch; }
    b.total = ortho_small_fits(rows, cols) ? 256 : 2 * b.x + 3 * b.a + b.part + b.scratch;      // (small matrices need none: any buffer will do)
    return b;
}
static int check_shape(int batch, int rows, int cols, int dtype, int steps) {
    if (batch < 1 || rows < 1 || cols < 1 || !real_dtype(dtype) || steps < 0 || steps > ORTHO_MAX_STEPS) return EBS_ERR_INVALID_ARG;
    // (a side of up to 2^30, as in a layer: tiles and stages are counted in 32 bits, rounded up)
    if (batch > 65535 || rows > (1 << 30) || cols > (1 << 30) || (long long)rows * cols > (1LL << 36) / batch) return EBS_ERR_OVERFLOW;
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
    // the singular values' bound before each step; from it the exponents of X, A, b I + c A and Q, and the products' factors
    OrthoFactors f = {};
    double bound = 1.0;
    int ex = headroom(bound);
    const float first = ldexpf(1.0f, ex);
    float last = scale / first;
    for (int i = 0; i < steps; ++i) {
        const StepBounds b = step_bounds(coeff, bound);
        if (!(b.next < 0x1p20 && b.next > 0x1p-20)) return EBS_ERR_UNSUPPORTED;
        const int ea = 2 * ex - 14, el = headroom(b.linear), eq = headroom(b.square), en = headroom(b.next);   // (an entry of A is at most the square of X's bound)
        f.gram[i] = ldexpf(1.0f, ea - 2 * ex);
        f.linear[i] = coeff[2] * ldexpf(1.0f, el - 2 * ex);
        f.linear_diag[i] = coeff[1] * ldexpf(1.0f, el);
        f.square[i] = ldexpf(1.0f, eq - ea - el);
        f.square_diag[i] = coeff[0] * ldexpf(1.0f, eq);
        f.next[i] = ldexpf(1.0f, en - eq - ex);
        // (Q's bound is that of a quadratic polynomial, whose terms are at most a few times it: neither product leaves fp32's range)
        f.quadratic[i] = (float)ldexp((double)coeff[2], eq - 2 * ea);
        f.direct[i] = (float)ldexp((double)coeff[1], eq - ea);
        last = scale * ldexpf(1.0f, -eq - ex);
        ex = en;
        bound = b.next;
    }
    const OrthoBuffers b = ortho_buffers(batch, rows, cols);
    if (workspace_bytes < b.total) return EBS_ERR_INVALID_ARG;
    const size_t bytes = (size_t)batch * rows * cols * element_size(dtype);
    const uintptr_t pg = (uintptr_t)g, po = (uintptr_t)out, pw = (uintptr_t)workspace;
    if (pg != po && pg < po + bytes && po < pg + bytes) return EBS_ERR_INVALID_ARG;
    if ((pw < pg + bytes && pg < pw + b.total) || (pw < po + bytes && po < pw + b.total)) return EBS_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (ortho_small_fits(rows, cols)) return launch_ortho_small(g, out, batch, rows, cols, dtype, steps, eps, first, last, f, st);
    __half* x = static_cast<__half*>(workspace);
    __half* x2 = reinterpret_cast<__half*>(static_cast<char*>(workspace) + b.x);
    __half* A = reinterpret_cast<__half*>(static_cast<char*>(workspace) + 2 * b.x);
    __half* L = reinterpret_cast<__half*>(static_cast<char*>(workspace) + 2 * b.x + b.a);
    __half* Q = reinterpret_cast<__half*>(static_cast<char*>(workspace) + 2 * b.x + 2 * b.a);
    float* scratch = reinterpret_cast<float*>(static_cast<char*>(workspace) + 2 * b.x + 3 * b.a + b.part);
    double* part = reinterpret_cast<double*>(static_cast<char*>(workspace) + 2 * b.x + 3 * b.a);
    if (dtype == EBS_F32) rc = launch_normalize<float>(g, batch, rows, cols, eps, first, part, b.parts, x, b.ld, b.plane, st);
    else if (dtype == EBS_F16) rc = launch_normalize<__half>(g, batch, rows, cols, eps, first, part, b.parts, x, b.ld, b.plane, st);
    else rc = launch_normalize<__nv_bfloat16>(g, batch, rows, cols, eps, first, part, b.parts, x, b.ld, b.plane, st);
    if (rc) return rc;
    const bool tall = rows > cols;                            // then X X^T X is taken as X (X^T X): the smaller product
    const int m = tall ? cols : rows, n = tall ? rows : cols;
    // What the tensor core truncates is, behind so many products, most of an fp32 result's error, and shorter sums have less of it.  Relative
    // error with sums of 4, 2 and 1 stages: 128 x 1152 2.6e-6, 2.7e-6, 1.7e-6 in 119, 119, 121 us; 2048^2 4.3e-6, 2.3e-6, 1.4e-6 in 709, 777,
    // 1029 us (products in fp32 throughout: 1.2e-6 and 2.9e-6).  A 16-bit result is rounded far above that.
    const int chunk = dtype != EBS_F32 ? GEMM_CHUNK : m <= 256 ? 1 : 2;
    for (int s = 0; s < steps; ++s) {
        const GemmOperand xs{x, b.ld, tall, 2, b.plane, 2 * b.plane}, as{A, b.side_ld, false, 2, b.side_plane, 2 * b.side_plane}, ls{L, b.side_ld, false, 2, b.side_plane, 2 * b.side_plane},
            qs{Q, b.side_ld, false, 2, b.side_plane, 2 * b.side_plane};
        PlanesOut oa{A, L, b.side_ld, b.side_plane, 2 * b.side_plane, f.gram[s], 0.0f, f.linear[s], f.linear_diag[s]};
        if ((rc = launch_gemm(xs, xs, GemmShape{m, m, n, batch, true, chunk}, scratch, oa, st))) return rc;
        PlanesOut oq{Q, nullptr, b.side_ld, b.side_plane, 2 * b.side_plane, f.square[s], f.square_diag[s], 0.0f, 0.0f};
        if ((rc = launch_gemm(as, ls, GemmShape{m, m, m, batch, true, chunk}, scratch, oq, st))) return rc;
        // X <- Q X or X Q; the last one is the result
        const GemmOperand xk{x, b.ld, false, 2, b.plane, 2 * b.plane}, xm{x, b.ld, true, 2, b.plane, 2 * b.plane};
        const GemmOperand &left = tall ? xk : qs, &right = tall ? qs : xm;
        const GemmShape shape{rows, cols, m, batch, false, chunk};
        if (s == steps - 1) return launch_gemm(left, right, shape, scratch, FinalOut{out, cols, (long long)rows * cols, last}, dtype, st);
        PlanesOut ox{x2, nullptr, b.ld, b.plane, 2 * b.plane, f.next[s], 0.0f, 0.0f, 0.0f};
        if ((rc = launch_gemm(left, right, shape, scratch, ox, st))) return rc;
        __half* t = x; x = x2; x2 = t;
    }
    if (steps > 0) return EBS_OK;
    const dim3 grid(blocks_for((long long)rows * cols * batch, 1));
    if (dtype == EBS_F32) return launch_chained(scale_out_kernel<float>, grid, 256, 0, st, 1, (const __half*)x, b.ld, b.plane, rows, cols, batch, last, static_cast<float*>(out));
    if (dtype == EBS_F16) return launch_chained(scale_out_kernel<__half>, grid, 256, 0, st, 1, (const __half*)x, b.ld, b.plane, rows, cols, batch, last, static_cast<__half*>(out));
    return launch_chained(scale_out_kernel<__nv_bfloat16>, grid, 256, 0, st, 1, (const __half*)x, b.ld, b.plane, rows, cols, batch, last, static_cast<__nv_bfloat16*>(out));
}

}  // extern "C"
