// Real-valued layers: y = act(x W^T + bias) + residual and its gradients.  See include/ebs.h.
#include "gemm_tile.cuh"

namespace ebs {

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
static size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }

// One tensor of a call: `rows` rows of `cols` elements, `ld` elements apart.
struct Rows {
    const void* p;
    long long rows, cols, ld;
    bool out;
};

// Whether two tensors share an element.  Rows of the same stride may interleave (column ranges of one buffer).
static bool overlap(const Rows& a, const Rows& b, size_t size) {
    if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0) return false;
    const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
    const uintptr_t ea = pa + ((a.rows - 1) * a.ld + a.cols) * size, eb = pb + ((b.rows - 1) * b.ld + b.cols) * size;
    if (pa >= eb || pb >= ea) return false;
    if (a.ld != b.ld) return true;
    const long long pitch = a.ld * (long long)size;
    long long d = ((long long)(pb - pa)) % pitch;
    if (d < 0) d += pitch;
    return !(d >= a.cols * (long long)size && pitch - d >= b.cols * (long long)size);
}

// The descriptor with its strides filled in, or an error.
static int complete(const ebs_linear_desc* in, ebs_linear_desc* d) {
    if (!in) return EBS_ERR_INVALID_ARG;
    *d = *in;
    if (d->m < 0 || d->n < 1 || d->k < 1 || !real_dtype(d->dtype) || d->act < EBS_ACT_NONE || d->act > EBS_ACT_SILU)
        return EBS_ERR_INVALID_ARG;
    const long long limit = 1LL << 40;
    long long* ld[5] = {&d->ldx, &d->ldw, &d->ldy, &d->ldr, &d->ldz};
    for (int i = 0; i < 5; ++i) {
        const long long dense = i < 2 ? d->k : d->n;
        if (*ld[i] == 0) *ld[i] = dense;
        if (*ld[i] < dense) return EBS_ERR_INVALID_ARG;
        if (*ld[i] > limit / (i == 1 ? d->n : (d->m > 0 ? d->m : 1))) return EBS_ERR_OVERFLOW;
    }
    return EBS_OK;
}

static int check_tensors(const Rows* t, int count, size_t size, const Rows* same_a, const Rows* same_b) {
    for (int i = 0; i < count; ++i) {
        if (!aligned16(t[i].p)) return EBS_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j) {
            if (!t[i].out && !t[j].out) continue;
            if (((&t[i] == same_a && &t[j] == same_b) || (&t[j] == same_a && &t[i] == same_b)) && t[i].p == t[j].p && t[i].ld == t[j].ld) continue;
            if (overlap(t[i], t[j], size)) return EBS_ERR_INVALID_ARG;
        }
    }
    return EBS_OK;
}

// ---------------------------------------------------------------------------------------------------- operands
// Takes buffers out of the workspace one behind the other; without a base it only counts.
struct Carver {
    char* base;
    size_t used = 0;
    template <typename T> T* take(size_t count) {
        char* p = base ? base + used : nullptr;
        used += round256(count * sizeof(T));
        return reinterpret_cast<T*>(p);
    }
};
static long long round8(long long v) { return (v + 7) & ~7LL; }

// A copy of 16-bit rows whose stride is a multiple of 16 bytes.
__global__ void __launch_bounds__(256) copy_rows_kernel(const uint16_t* __restrict__ src, long long ld, long long rows, int cols, uint16_t* __restrict__ dst, long long ldd) {
    for (long long r = blockIdx.y; r < rows; r += gridDim.y)
        for (int c = blockIdx.x * 256 + threadIdx.x; c < cols; c += gridDim.x * 256) dst[r * ldd + c] = src[r * ld + c];
}

// The power of two that brings values of magnitude up to the one with these bits below 2^15, and what is remembered of it: its
// negated exponent, or what kind of row this is.
__device__ __forceinline__ int split_exponent(unsigned top_bits) { return 141 - (int)(top_bits >> 23); }
__device__ __forceinline__ int split_record(unsigned top_bits) {
    if (top_bits > 0x7f800000u) return SCALE_NAN;
    if (top_bits == 0x7f800000u) return SCALE_INF;
    return top_bits == 0u ? 0 : -split_exponent(top_bits);
}
// x = (hi + lo) 2^-e: both halves rounded to nearest, 22 bits where hi is a normal number and lo has its 11 bits (values within 2^-17
// of the largest of the row), an absolute error of 2^-40 of the largest below.  Non-finite values are 0: their rows are flagged.
__device__ __forceinline__ void split_value(float x, int e, __half& hi, __half& lo) {
    const float v = (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? 0.0f : scale_pow2(x, e);
    hi = __float2half_rn(v);
    lo = __float2half_rn(v - __half2float(hi));
}

// Four neighbouring elements of a row, of which `left` exist: one 16-byte access where the rows allow it (VEC).
template <bool VEC>
__device__ __forceinline__ float4 load4(const float* p, int left) {
    if (VEC && left >= 4) return *reinterpret_cast<const float4*>(p);
    return make_float4(left > 0 ? p[0] : 0.0f, left > 1 ? p[1] : 0.0f, left > 2 ? p[2] : 0.0f, left > 3 ? p[3] : 0.0f);
}
__device__ __forceinline__ unsigned magnitude(const float4& v) {
    const unsigned a = max(__float_as_uint(v.x) & 0x7fffffffu, __float_as_uint(v.y) & 0x7fffffffu);
    return max(a, max(__float_as_uint(v.z) & 0x7fffffffu, __float_as_uint(v.w) & 0x7fffffffu));
}
// (the planes' rows are padded to whole groups of eight elements: what is written past the end of a row is padding)
__device__ __forceinline__ void store_split4(__half* hi_plane, __half* lo_plane, const float4& v, int e0, int e1, int e2, int e3) {
    __half hi[4], lo[4];
    split_value(v.x, e0, hi[0], lo[0]);
    split_value(v.y, e1, hi[1], lo[1]);
    split_value(v.z, e2, hi[2], lo[2]);
    split_value(v.w, e3, hi[3], lo[3]);
    *reinterpret_cast<uint2*>(hi_plane) = *reinterpret_cast<const uint2*>(hi);
    *reinterpret_cast<uint2*>(lo_plane) = *reinterpret_cast<const uint2*>(lo);
}

// Planes of a matrix whose reduction runs along its rows: one exponent a row.  A row is a warp's or (WIDE) a block's; its first
// 16 elements a thread stay in registers between the search for the largest and the split.
template <bool VEC, bool WIDE>
__global__ void __launch_bounds__(256) split_rows_kernel(const float* __restrict__ src, long long ld, long long rows, int cols, __half* __restrict__ dst,
                                                         long long ldd, int* __restrict__ exps) {
    __shared__ unsigned part[8];
    constexpr int T = WIDE ? 256 : 32;
    const int t = WIDE ? threadIdx.x : threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long step = WIDE ? gridDim.x : gridDim.x * 8LL;
    for (long long r = WIDE ? blockIdx.x : blockIdx.x * 8LL + warp; r < rows; r += step) {
        const float* x = src + r * ld;
        float4 held[4];
        unsigned top = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = (i * T + t) * 4;
            held[i] = load4<VEC>(x + c, cols - c);
            top = max(top, magnitude(held[i]));
        }
        for (int c = (4 * T + t) * 4; c < cols; c += 4 * T) top = max(top, magnitude(load4<VEC>(x + c, cols - c)));
        top = __reduce_max_sync(0xffffffffu, top);
        if (WIDE) {
            __syncthreads();                                  // (the previous row's reads are over)
            if ((threadIdx.x & 31) == 0) part[warp] = top;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, part[i]);
        }
        const int e = top < 0x7f800000u && top != 0u ? split_exponent(top) : 0;
        if (t == 0) exps[r] = split_record(top);
        __half *hi = dst + r * ldd, *lo = hi + rows * ldd;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = (i * T + t) * 4;
            if (c < cols) store_split4(hi + c, lo + c, held[i], e, e, e, e);
        }
        for (int c = (4 * T + t) * 4; c < cols; c += 4 * T) store_split4(hi + c, lo + c, load4<VEC>(x + c, cols - c), e, e, e, e);
    }
}
// The largest magnitudes of the columns (their bits, in `top`, which starts at zero): 128 columns a block.
template <bool VEC>
__global__ void __launch_bounds__(256) column_top_kernel(const float* __restrict__ src, long long ld, long long rows, int cols, unsigned* __restrict__ top) {
    __shared__ unsigned part[8][128];
    const int lane = threadIdx.x & 31, c = blockIdx.x * 128 + lane * 4, y = threadIdx.x >> 5;
    unsigned m[4] = {0u, 0u, 0u, 0u};
    if (c < cols)
#pragma unroll 4
        for (long long r = blockIdx.y * 8LL + y; r < rows; r += gridDim.y * 8LL) {
            const float4 v = load4<VEC>(src + r * ld + c, cols - c);
            m[0] = max(m[0], __float_as_uint(v.x) & 0x7fffffffu);
            m[1] = max(m[1], __float_as_uint(v.y) & 0x7fffffffu);
            m[2] = max(m[2], __float_as_uint(v.z) & 0x7fffffffu);
            m[3] = max(m[3], __float_as_uint(v.w) & 0x7fffffffu);
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) part[y][lane * 4 + i] = m[i];
    __syncthreads();
    if (threadIdx.x < 128 && blockIdx.x * 128 + threadIdx.x < cols) {
        unsigned v = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) v = max(v, part[i][threadIdx.x]);
        atomicMax(top + blockIdx.x * 128 + threadIdx.x, v);   // (a maximum does not depend on the order)
    }
}
// Planes of a matrix whose reduction runs across its rows: one exponent a column, from column_top_kernel.
template <bool VEC>
__global__ void __launch_bounds__(256) split_columns_kernel(const float* __restrict__ src, long long ld, long long rows, int cols, const unsigned* __restrict__ top,
                                                            __half* __restrict__ dst, long long ldd, int* __restrict__ exps) {
    const int lane = threadIdx.x & 31, c = blockIdx.x * 128 + lane * 4, y = threadIdx.x >> 5;
    if (c >= cols) return;
    int e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned t = c + i < cols ? top[c + i] : 0u;
        e[i] = t < 0x7f800000u && t != 0u ? split_exponent(t) : 0;
        if (blockIdx.y == 0 && y == 0 && c + i < cols) exps[c + i] = split_record(t);
    }
#pragma unroll 4
    for (long long r = blockIdx.y * 8LL + y; r < rows; r += gridDim.y * 8LL)
        store_split4(dst + r * ldd + c, dst + (rows + r) * ldd + c, load4<VEC>(src + r * ld + c, cols - c), e[0], e[1], e[2], e[3]);
}

// An operand of a product: 16-bit rows as they are, or copied where their starts are not on 16 bytes; fp32 rows split.
struct Prepared {
    GemmOperand op;
    const int* exps = nullptr;
};
struct Matrix {
    const void* p;
    long long rows, ld;
    int cols;
};
static unsigned row_blocks(long long rows, int per) { const long long b = (rows + per - 1) / per; return (unsigned)(b < 2048 ? b : 2048); }

// Row blocks (of at least 32 rows) for kernels that go down `across` blocks of columns: about eight blocks an SM.
static unsigned column_blocks(long long rows, int across) {
    long long b = (rows + 31) / 32, want = (8LL * gemm_sm_count() + across - 1) / across;
    if (b > want) b = want;
    return (unsigned)(b < 1 ? 1 : b > 65535 ? 65535 : b);
}

static int prepare_operand(const Matrix& m, int dtype, bool across, Carver& ws, bool run, cudaStream_t st, Prepared* out) {
    out->op = GemmOperand{m.p, m.ld, across};
    if (dtype != EBS_F32) {
        if ((m.ld & 7) == 0) return EBS_OK;
        const long long ldd = round8(m.cols);
        uint16_t* copy = ws.take<uint16_t>((size_t)m.rows * ldd);
        out->op.p = copy;
        out->op.ld = ldd;
        if (!run) return EBS_OK;
        copy_rows_kernel<<<dim3((m.cols + 255) / 256, row_blocks(m.rows, 1)), 256, 0, st>>>(static_cast<const uint16_t*>(m.p), m.ld, m.rows, m.cols, copy, ldd);
        return check_cuda(cudaGetLastError());
    }
    const long long ldd = round8(m.cols);
    __half* planes = ws.take<__half>(2 * (size_t)m.rows * ldd);
    int* exps = ws.take<int>(across ? m.cols : m.rows);
    unsigned* top = across ? ws.take<unsigned>(m.cols) : nullptr;
    out->op = GemmOperand{planes, ldd, across, 2, m.rows * ldd, 2 * m.rows * ldd};
    out->exps = exps;
    if (!run) return EBS_OK;
    const float* src = static_cast<const float*>(m.p);
    const bool vec = (m.ld & 3) == 0;
    if (!across) {
        const bool wide = m.cols > 512;
        const unsigned grid = row_blocks(m.rows, wide ? 1 : 8);
        auto kern = wide ? (vec ? split_rows_kernel<true, true> : split_rows_kernel<false, true>) : (vec ? split_rows_kernel<true, false> : split_rows_kernel<false, false>);
        kern<<<grid, 256, 0, st>>>(src, m.ld, m.rows, m.cols, planes, ldd, exps);
    } else {
        if (check_cuda(cudaMemsetAsync(top, 0, (size_t)m.cols * 4, st))) return EBS_ERR_CUDA;
        const dim3 grid((m.cols + 127) / 128, column_blocks(m.rows, (m.cols + 127) / 128));
        (vec ? column_top_kernel<true> : column_top_kernel<false>)<<<grid, 256, 0, st>>>(src, m.ld, m.rows, m.cols, top);
        (vec ? split_columns_kernel<true> : split_columns_kernel<false>)<<<grid, 256, 0, st>>>(src, m.ld, m.rows, m.cols, top, planes, ldd, exps);
    }
    return check_cuda(cudaGetLastError());
}

// One product with its operands prepared; a: its rows are the result's (across: its columns), likewise b for the result's columns.
static int product(const Prepared& a, const Matrix& am, const Prepared& b, const Matrix& bm, int red, GemmOut o, int dtype, cudaStream_t st) {
    GemmShape s{(int)(a.op.mn_major ? am.cols : am.rows), (int)(b.op.mn_major ? bm.cols : bm.rows), red, 1};
    if (dtype == EBS_F32) {
        o.row_exp = a.exps;
        o.col_exp = b.exps;
        o.fp32.a = static_cast<const float*>(am.p);
        o.fp32.b = static_cast<const float*>(bm.p);
        o.fp32.a_row = a.op.mn_major ? 1 : am.ld;
        o.fp32.a_red = a.op.mn_major ? am.ld : 1;
        o.fp32.b_col = b.op.mn_major ? 1 : bm.ld;
        o.fp32.b_red = b.op.mn_major ? bm.ld : 1;
        o.fp32.red = red;
    }
    return launch_gemm(a.op, b.op, s, o, dtype, st);
}

// ---------------------------------------------------------------------------------------------------- dz and dbias
// A half-precision dz is kept halved: the steepest slope (1.13) times the type's largest value would not fit.
static float dz_store_scale(const ebs_linear_desc& d) { return d.dtype == EBS_F16 && d.act ? 0.5f : 1.0f; }

// dz = dy * act'(z), stored times `store`, and the column sums of dz before its rounding.  A block takes 32 packs of N columns and
// the rows of one of gridDim.y chunks; the sums of a chunk go to `part`, or (one chunk) to dbias at once.
template <typename T, int N>
__global__ void __launch_bounds__(256) linear_dz_kernel(const T* __restrict__ dy, long long ldy, const T* __restrict__ z, long long ldz, int m, int n, int act, float store,
                                                        T* __restrict__ dz, long long lddz, T* __restrict__ dbias, float* __restrict__ part) {
    __shared__ float sums[8][32 * N + 4];
    const int lane = threadIdx.x & 31, y = threadIdx.x >> 5, col = (blockIdx.x * 32 + lane) * N;
    const long long r0 = (long long)m * blockIdx.y / gridDim.y, r1 = (long long)m * (blockIdx.y + 1) / gridDim.y;
    float sum[N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.0f;
    if (col < n) {
#pragma unroll 2
        for (long long r = r0 + y; r < r1; r += 8) {
            float v[N], zv[N];
            const bool whole = N > 1 && col + N <= n;
            if (whole) {
                if constexpr (N > 1) load_pack(dy + r * ldy + col, v);
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] = col + e < n ? to_f32(dy[r * ldy + col + e]) : 0.0f;
            }
            if (act) {
                if (whole) {
                    if constexpr (N > 1) load_pack(z + r * ldz + col, zv);
                } else {
#pragma unroll
                    for (int e = 0; e < N; ++e) zv[e] = col + e < n ? to_f32(z[r * ldz + col + e]) : 0.0f;
                }
                switch (act) {
#define EBS_SLOPE_CASE(A) case A: _Pragma("unroll") for (int e = 0; e < N; ++e) v[e] *= activation_slope(zv[e], A); break;
                    EBS_SLOPE_CASE(EBS_ACT_RELU) EBS_SLOPE_CASE(EBS_ACT_GELU) EBS_SLOPE_CASE(EBS_ACT_GELU_TANH) EBS_SLOPE_CASE(EBS_ACT_SILU)
#undef EBS_SLOPE_CASE
                    default: break;
                }
            }
#pragma unroll
            for (int e = 0; e < N; ++e) sum[e] += v[e];
            if (dz) {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] *= store;
                if (N > 1) {                                  // (rows of dz are padded to whole packs)
                    if constexpr (N > 1) store_pack(dz + r * lddz + col, v);
                } else {
                    dz[r * lddz + col] = from_f32<T>(v[0]);
                }
            }
        }
    }
    if (!dbias) return;
#pragma unroll
    for (int e = 0; e < N; ++e) sums[y][lane * N + e] = sum[e];
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * N; i += 256) {
        const int c = blockIdx.x * 32 * N + i;
        if (c >= n) break;
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < 8; ++q) s += sums[q][i];
        if (gridDim.y == 1) dbias[c] = from_f32<T>(s);
        else part[(size_t)blockIdx.y * n + c] = s;
    }
}
template <typename T>
__global__ void __launch_bounds__(256) linear_dbias_kernel(const float* __restrict__ part, int chunks, int n, T* __restrict__ dbias) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= n) return;
    float s = 0.0f;
#pragma unroll 8
    for (int i = 0; i < chunks; ++i) s += part[(size_t)i * n + c];
    dbias[c] = from_f32<T>(s);
}

// Chunks of rows the sums are taken in, from the sizes alone: about four blocks an SM, at least 32 rows each.
static int dz_chunks(const ebs_linear_desc& d) {
    const int packs = d.dtype == EBS_F32 ? 128 : 256, across = (d.n + packs - 1) / packs;
    long long c = (d.m + 31) / 32, want = (4LL * 148 + across - 1) / across;
    return (int)(c < want ? c : want);
}
template <typename T>
static int launch_dz(const void* dy, const void* z, const ebs_linear_desc& d, void* dz, long long lddz, void* dbias, float* part, cudaStream_t st) {
    constexpr int N = Pack<T>::N;
    const bool packs = d.ldy % N == 0 && (!d.act || d.ldz % N == 0);
    const int chunks = dz_chunks(d), per = packs ? 32 * N : 32;
    const dim3 grid((d.n + per - 1) / per, chunks);
    auto kern = packs ? linear_dz_kernel<T, N> : linear_dz_kernel<T, 1>;
    kern<<<grid, 256, 0, st>>>(static_cast<const T*>(dy), d.ldy, static_cast<const T*>(z), d.ldz, d.m, d.n, d.act, dz_store_scale(d), static_cast<T*>(dz), lddz, static_cast<T*>(dbias), part);
    if (dbias && chunks > 1) linear_dbias_kernel<T><<<(d.n + 255) / 256, 256, 0, st>>>(part, chunks, d.n, static_cast<T*>(dbias));
    return check_cuda(cudaGetLastError());
}

// ---------------------------------------------------------------------------------------------------- the calls
struct LinearTensors {
    const void *x, *w, *bias, *residual, *dy, *z;
    void *y, *keep, *dx, *dw, *dbias;
};
// Runs the call, or (run = false) counts its workspace.
static int forward(const ebs_linear_desc& d, const LinearTensors& t, Carver& ws, bool run, cudaStream_t st) {
    if (d.m == 0) return EBS_OK;
    const Matrix xm{t.x, d.m, d.ldx, d.k}, wm{t.w, d.n, d.ldw, d.k};
    Prepared x, w;
    int rc;
    if ((rc = prepare_operand(xm, d.dtype, false, ws, run, st, &x)) || (rc = prepare_operand(wm, d.dtype, false, ws, run, st, &w)) || !run) return rc;
    GemmOut o;
    o.bias = t.bias; o.residual = t.residual; o.z = t.keep; o.y = t.y; o.act = d.act;
    o.ldr = d.ldr; o.ldz = d.ldz; o.ldy = d.ldy;
    return product(x, xm, w, wm, d.k, o, d.dtype, st);
}
static int backward(const ebs_linear_desc& d, const LinearTensors& t, Carver& ws, bool run, cudaStream_t st) {
    int rc;
    if (d.m == 0) {
        if (!run) return EBS_OK;
        const size_t size = element_size(d.dtype);
        if (t.dw && check_cuda(cudaMemset2DAsync(t.dw, d.ldw * size, 0, d.k * size, d.n, st))) return EBS_ERR_CUDA;
        if (t.dbias && check_cuda(cudaMemsetAsync(t.dbias, 0, d.n * size, st))) return EBS_ERR_CUDA;
        return EBS_OK;
    }
    Matrix dm{t.dy, d.m, d.ldy, d.n};
    if (d.act || t.dbias || !run) {
        void* dz = nullptr;
        if (d.act) {
            const long long ld = round8(d.n);
            dz = d.dtype == EBS_F32 ? (void*)ws.take<float>((size_t)d.m * ld) : (void*)ws.take<uint16_t>((size_t)d.m * ld);
            dm.p = dz;
            dm.ld = ld;
        }
        float* part = dz_chunks(d) > 1 ? ws.take<float>((size_t)dz_chunks(d) * d.n) : nullptr;
        if (run) {
            if (d.dtype == EBS_F32) rc = launch_dz<float>(t.dy, t.z, d, dz, dm.ld, t.dbias, part, st);
            else if (d.dtype == EBS_F16) rc = launch_dz<__half>(t.dy, t.z, d, dz, dm.ld, t.dbias, part, st);
            else rc = launch_dz<__nv_bfloat16>(t.dy, t.z, d, dz, dm.ld, t.dbias, part, st);
            if (rc) return rc;
        }
    }
    GemmOut o;
    o.alpha = 1.0f / dz_store_scale(d);
    Prepared g, other;
    const bool shared = d.dtype != EBS_F32;                  // one 16-bit copy serves both products
    if (shared && (rc = prepare_operand(dm, d.dtype, false, ws, run && (t.dx || t.dw), st, &g))) return rc;
    if (t.dx || !run) {
        const Matrix wm{t.w, d.n, d.ldw, d.k};
        if (!shared && (rc = prepare_operand(dm, d.dtype, false, ws, run, st, &g))) return rc;
        if ((rc = prepare_operand(wm, d.dtype, true, ws, run, st, &other))) return rc;
        o.y = t.dx; o.ldy = d.ldx;
        if (run && (rc = product(g, dm, other, wm, d.n, o, d.dtype, st))) return rc;
    }
    if (t.dw || !run) {
        const Matrix xm{t.x, d.m, d.ldx, d.k};
        if (!shared) { if ((rc = prepare_operand(dm, d.dtype, true, ws, run, st, &g))) return rc; }
        else g.op.mn_major = true;
        if ((rc = prepare_operand(xm, d.dtype, true, ws, run, st, &other))) return rc;
        o.y = t.dw; o.ldy = d.ldw;
        if (run && (rc = product(g, dm, other, xm, d.m, o, d.dtype, st))) return rc;
    }
    return EBS_OK;
}
static size_t linear_workspace(const ebs_linear_desc& d, bool back) {
    Carver count{nullptr};
    const LinearTensors none{};
    if (back) backward(d, none, count, false, nullptr);
    else forward(d, none, count, false, nullptr);
    return count.used;
}

}  // namespace ebs

using namespace ebs;

extern "C" {

size_t ebs_linear_workspace_bytes(const ebs_linear_desc* desc, int backward) {
    ebs_linear_desc d;
    if (complete(desc, &d)) return 0;
    return linear_workspace(d, backward != 0);
}

int ebs_linear_forward(const void* x, const void* w, const void* bias, const void* residual, const ebs_linear_desc* desc, void* y, void* z,
                       void* workspace, size_t workspace_bytes, void* stream) {
    ebs_linear_desc d;
    const int rc = complete(desc, &d);
    if (rc) return rc;
    if (!w || (d.m > 0 && (!x || !y))) return EBS_ERR_INVALID_ARG;
    const size_t size = element_size(d.dtype), need = linear_workspace(d, false);
    if (need && (!workspace || workspace_bytes < need)) return EBS_ERR_INVALID_ARG;
    const Rows t[] = {{x, d.m, d.k, d.ldx, false}, {w, d.n, d.k, d.ldw, false}, {bias, 1, d.n, d.n, false}, {residual, d.m, d.n, d.ldr, false},
                      {y, d.m, d.n, d.ldy, true}, {z, d.m, d.n, d.ldz, true}, {need ? workspace : nullptr, 1, (long long)(need / size), (long long)(need / size), true}};
    if (check_tensors(t, 7, size, &t[3], &t[4])) return EBS_ERR_INVALID_ARG;
    Carver ws{static_cast<char*>(workspace)};
    return forward(d, LinearTensors{x, w, bias, residual, nullptr, nullptr, y, z, nullptr, nullptr, nullptr}, ws, true, static_cast<cudaStream_t>(stream));
}

int ebs_linear_backward(const void* dy, const void* x, const void* w, const void* z, const ebs_linear_desc* desc, void* dx, void* dw, void* dbias,
                        void* workspace, size_t workspace_bytes, void* stream) {
    ebs_linear_desc d;
    const int rc = complete(desc, &d);
    if (rc) return rc;
    if (!dx && !dw && !dbias && d.m > 0) return EBS_ERR_INVALID_ARG;
    if (d.m > 0 && (!dy || (dx && !w) || (dw && !x) || (d.act && !z))) return EBS_ERR_INVALID_ARG;
    const size_t size = element_size(d.dtype), need = linear_workspace(d, true);
    if (need && (!workspace || workspace_bytes < need)) return EBS_ERR_INVALID_ARG;
    const Rows t[] = {{dy, d.m, d.n, d.ldy, false}, {x, d.m, d.k, d.ldx, false}, {w, d.n, d.k, d.ldw, false}, {d.act ? z : nullptr, d.m, d.n, d.ldz, false},
                      {dx, d.m, d.k, d.ldx, true}, {dw, d.n, d.k, d.ldw, true}, {dbias, 1, d.n, d.n, true},
                      {need ? workspace : nullptr, 1, (long long)(need / size), (long long)(need / size), true}};
    if (check_tensors(t, 8, size, nullptr, nullptr)) return EBS_ERR_INVALID_ARG;
    Carver ws{static_cast<char*>(workspace)};
    return backward(d, LinearTensors{x, w, nullptr, nullptr, dy, z, nullptr, nullptr, dx, dw, dbias}, ws, true, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
