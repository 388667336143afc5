// Real-valued layers: y = act(x W^T + bias) + residual and its gradients.  See include/ebs.h.
#include <type_traits>

#include "gemm_tile.cuh"
#include "tensors.cuh"

namespace ebs {

// The descriptor with its strides filled in, or an error.
int complete_linear(const ebs_linear_desc* in, ebs_linear_desc* d) {
    if (!in) return EBS_ERR_INVALID_ARG;
    *d = *in;
    if (d->m < 0 || d->n < 1 || d->k < 1 || !real_dtype(d->dtype) || d->act < EBS_ACT_NONE || d->act > EBS_ACT_SILU)
        return EBS_ERR_INVALID_ARG;
    if (d->m > (1 << 30) || d->n > (1 << 30) || d->k > (1 << 30)) return EBS_ERR_OVERFLOW;
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

// ---------------------------------------------------------------------------------------------------- operands
// Copies of 16-bit rows: 256 elements of a row a warp, all on their way at once.
__global__ void __launch_bounds__(256) copy_rows_kernel(const __grid_constant__ CopyJobs j) {
    let_next_kernel_start();
    wait_for_previous_kernel();
    const int lane = threadIdx.x & 31;
    for (long long p = blockIdx.x * 8LL + (threadIdx.x >> 5); p < j.pieces; p += gridDim.x * 8LL) {
        int i = 0;
        while (i + 1 < j.count && p >= j.first[i + 1]) ++i;
        const long long q = p - j.first[i], r = q / j.across[i];
        const int c0 = (int)(q - r * j.across[i]) * 256 + lane;
        const uint16_t* src = j.src[i] + r * j.ld[i];
        uint16_t *dst = j.dst[i] + r * j.ldd[i], v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c0 + 32 * e < j.cols[i] ? src[c0 + 32 * e] : (uint16_t)0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c0 + 32 * e < j.cols[i]) dst[c0 + 32 * e] = v[e];
    }
}

// The power of two that brings values of magnitude up to the one with these bits below 2^15, and what is remembered of it: its
// negated exponent, or what kind of row this is.
__device__ __forceinline__ int split_exponent(unsigned top_bits) { return top_bits < 0x7f800000u && top_bits != 0u ? 141 - (int)(top_bits >> 23) : 0; }
__device__ __forceinline__ int split_record(unsigned top_bits) {
    if (top_bits > 0x7f800000u) return SCALE_NAN;
    if (top_bits == 0x7f800000u) return SCALE_INF;
    return -split_exponent(top_bits);
}
// x = (hi + lo) 2^-e: both halves rounded to nearest, 22 bits where hi is a normal number and lo has its 11 bits (values within 2^-17
// of the largest of the row), an absolute error of 2^-40 of the largest below.  Non-finite values are 0: their rows are flagged.
__device__ __forceinline__ float scaled_finite(float x, int e) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u ? 0.0f : scale_pow2(x, e); }
// Four neighbouring elements of a row, of which `left` exist: one 16-byte access where the rows allow it.
__device__ __forceinline__ float4 load4(const float* p, int left, bool vec) {
    if (vec && left >= 4) return *reinterpret_cast<const float4*>(p);
    return make_float4(left > 0 ? p[0] : 0.0f, left > 1 ? p[1] : 0.0f, left > 2 ? p[2] : 0.0f, left > 3 ? p[3] : 0.0f);
}
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// (the planes' rows are padded to whole groups of eight elements: what is written past the end of a row is padding)
__device__ __forceinline__ void store_split4(__half* hi_plane, __half* lo_plane, const float4& v, const int (&e)[4]) {
    uint2 hi, lo;
    split_pair(scaled_finite(v.x, e[0]), scaled_finite(v.y, e[1]), hi.x, lo.x);
    split_pair(scaled_finite(v.z, e[2]), scaled_finite(v.w, e[3]), hi.y, lo.y);
    *reinterpret_cast<uint2*>(hi_plane) = hi;
    *reinterpret_cast<uint2*>(lo_plane) = lo;
}

// A matrix to split into planes.  across = 0: its reduction runs along a row, one exponent a row.  across = 1: down the rows, one
// exponent a column; the largest magnitudes of the columns then come from column_tops for each of `chunks` chunks of rows, and where they are
// many over the chunks from linear_chunks_kernel (first row of `tops`).
struct SplitJob {
    const float* src;
    long long ld, rows;
    int cols, across;
    __half* dst;
    long long ldd;
    int* exps;
    unsigned* tops;                        // [chunks][cols]
    int chunks, joined, vec;               // joined: chunks that are left when the matrix is split
    unsigned blocks, first;                // thread blocks, and the first of them in the launch
};
constexpr int MAX_SPLIT_JOBS = 4;
constexpr int FEW_CHUNKS = 8;              // so many a split joins by itself: less than a launch costs
constexpr int SPLIT_WIDE = 1280;           // columns from which on a block shares a row
struct SplitJobs {
    SplitJob job[MAX_SPLIT_JOBS];
    int count;
};

// A row is a warp's or (WIDE) a block's; its first 4 * H elements a thread stay in registers between the search for the largest and the
// split, all of them on their way at once.
template <bool WIDE, int H>
__device__ __forceinline__ void split_rows(const SplitJob& j, unsigned block, unsigned* part) {
    constexpr int T = WIDE ? 256 : 32;
    const int t = WIDE ? threadIdx.x : threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long step = WIDE ? j.blocks : j.blocks * 8LL;
    for (long long r = WIDE ? block : block * 8LL + warp; r < j.rows; r += step) {
        const float* x = j.src + r * j.ld;
        float4 held[H];
        unsigned top = 0u;
#pragma unroll
        for (int i = 0; i < H; ++i) {
            const int c = (i * T + t) * 4;
            held[i] = load4(x + c, j.cols - c, j.vec);
        }
#pragma unroll
        for (int i = 0; i < H; ++i) top = max(max(top, max(magnitude(held[i].x), magnitude(held[i].y))), max(magnitude(held[i].z), magnitude(held[i].w)));
        for (int c = (H * T + t) * 4; c < j.cols; c += 4 * T) {
            const float4 v = load4(x + c, j.cols - c, j.vec);
            top = max(max(top, max(magnitude(v.x), magnitude(v.y))), max(magnitude(v.z), magnitude(v.w)));
        }
        top = __reduce_max_sync(0xffffffffu, top);
        if (WIDE) {
            __syncthreads();                                  // (the previous row's reads are over)
            if ((threadIdx.x & 31) == 0) part[warp] = top;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, part[i]);
        }
        const int e = split_exponent(top), es[4] = {e, e, e, e};
        if (t == 0) j.exps[r] = split_record(top);
        __half *hi = j.dst + r * j.ldd, *lo = hi + j.rows * j.ldd;
#pragma unroll
        for (int i = 0; i < H; ++i) {
            const int c = (i * T + t) * 4;
            if (c < j.cols) store_split4(hi + c, lo + c, held[i], es);
        }
        for (int c = (H * T + t) * 4; c < j.cols; c += 4 * T) store_split4(hi + c, lo + c, load4(x + c, j.cols - c, j.vec), es);
    }
}
__device__ __forceinline__ void tops_of_block(unsigned (&m)[4], unsigned (*part)[128], unsigned* out, int col0, int cols) {
    const int lane = threadIdx.x & 31, y = threadIdx.x >> 5;
#pragma unroll
    for (int i = 0; i < 4; ++i) part[y][lane * 4 + i] = m[i];
    __syncthreads();
    if (threadIdx.x < 128 && col0 + (int)threadIdx.x < cols) {
        unsigned v = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) v = max(v, part[i][threadIdx.x]);
        out[threadIdx.x] = v;
    }
}
// The largest magnitudes of 128 columns over one chunk of rows.
__device__ __forceinline__ void column_tops(const SplitJob& j, unsigned block, unsigned (*part)[128]) {
    const int across = (j.cols + 127) / 128, bx = (int)(block % across), by = (int)(block / across);
    const int lane = threadIdx.x & 31, y = threadIdx.x >> 5, c = bx * 128 + lane * 4;
    const long long r0 = j.rows * by / j.chunks, r1 = j.rows * (by + 1) / j.chunks;
    unsigned m[4] = {0u, 0u, 0u, 0u};
    if (c < j.cols)
#pragma unroll 8
        for (long long r = r0 + y; r < r1; r += 8) {
            const float4 v = load4(j.src + r * j.ld + c, j.cols - c, j.vec);
            m[0] = max(m[0], magnitude(v.x));
            m[1] = max(m[1], magnitude(v.y));
            m[2] = max(m[2], magnitude(v.z));
            m[3] = max(m[3], magnitude(v.w));
        }
    tops_of_block(m, part, j.tops + (size_t)by * j.cols + bx * 128, bx * 128, j.cols);
}
__device__ __forceinline__ void split_columns(const SplitJob& j, unsigned block) {
    const int across = (j.cols + 127) / 128, bx = (int)(block % across), by = (int)(block / across), down = (int)(j.blocks / across);
    const int lane = threadIdx.x & 31, y = threadIdx.x >> 5, c = bx * 128 + lane * 4;
    int e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned t = 0u;
        if (c + i < j.cols)
#pragma unroll 4
            for (int q = 0; q < j.joined; ++q) t = max(t, j.tops[(size_t)q * j.cols + c + i]);
        e[i] = split_exponent(t);
        if (by == 0 && y == 0 && c + i < j.cols) j.exps[c + i] = split_record(t);
    }
    if (c >= j.cols) return;
    const long long r0 = j.rows * by / down, r1 = j.rows * (by + 1) / down;
#pragma unroll 8
    for (long long r = r0 + y; r < r1; r += 8)
        store_split4(j.dst + r * j.ldd + c, j.dst + (j.rows + r) * j.ldd + c, load4(j.src + r * j.ld + c, j.cols - c, j.vec), e);
}

__device__ __forceinline__ int job_of(const SplitJobs& s, unsigned block) {
    int i = 0;
    while (i + 1 < s.count && block >= s.job[i + 1].first) ++i;
    return i;
}
// Splits of a call: all in one launch, or (large matrices) those by rows and those by columns in one each -- the rows' registers
// would cost the columns half their threads.
template <bool ROWS, bool COLUMNS>
__global__ void __launch_bounds__(256) split_kernel(const __grid_constant__ SplitJobs jobs) {
    __shared__ unsigned part[8];
    let_next_kernel_start();
    wait_for_previous_kernel();
    const SplitJob& j = jobs.job[job_of(jobs, blockIdx.x)];
    const unsigned block = blockIdx.x - j.first;
    if (COLUMNS && (!ROWS || j.across)) split_columns(j, block);
    if (ROWS && (!COLUMNS || !j.across)) {
        if (j.cols > SPLIT_WIDE) split_rows<true, 4>(j, block, part);
        else if (j.cols > 512) split_rows<false, 10>(j, block, part);
        else split_rows<false, 4>(j, block, part);
    }
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
// Chunks (of at least 32 rows) for work that goes down `across` blocks of columns: about eight blocks an SM; from the sizes alone.
static int row_chunks(long long rows, int across) {
    const long long c = (rows + 31) / 32, want = (8LL * 148 + across - 1) / across;
    return (int)(c < want ? c : want);
}
// Describes the operand and takes its buffers; fp32: adds its split to the jobs.
static Prepared plan_operand(const Matrix& m, int dtype, bool across, Carver& ws, SplitJobs* jobs) {
    Prepared out;
    out.op = GemmOperand{m.p, m.ld, across};
    const long long ldd = round8(m.cols);
    if (dtype != EBS_F32) {
        if ((m.ld & 7) == 0) return out;
        out.op.p = ws.take<uint16_t>((size_t)m.rows * ldd);
        out.op.ld = ldd;
        return out;
    }
    SplitJob j{static_cast<const float*>(m.p), m.ld, m.rows, m.cols, across, ws.take<__half>(2 * (size_t)m.rows * ldd), ldd, ws.take<int>(across ? m.cols : m.rows), nullptr, 0, 0, (m.ld & 3) == 0, 0, 0};
    if (across) {
        const int blocks = (m.cols + 127) / 128;
        j.chunks = row_chunks(m.rows, blocks);
        j.joined = j.chunks > FEW_CHUNKS ? 1 : j.chunks;
        j.tops = ws.take<unsigned>((size_t)j.chunks * m.cols);
        j.blocks = (unsigned)(blocks * j.chunks);
    } else {
        const long long b = m.cols > SPLIT_WIDE ? m.rows : (m.rows + 7) / 8;
        j.blocks = (unsigned)(b < 4096 ? b : 4096);
    }
    out.op = GemmOperand{j.dst, ldd, across, 2, m.rows * ldd, 2 * m.rows * ldd};
    out.exps = j.exps;
    jobs->job[jobs->count++] = j;
    return out;
}
void add_copy_rows(CopyJobs* j, const void* src, void* dst, long long rows, int cols, long long ld, long long ldd) {
    const int i = j->count++;
    j->src[i] = static_cast<const uint16_t*>(src);
    j->dst[i] = static_cast<uint16_t*>(dst);
    j->ld[i] = ld;
    j->ldd[i] = ldd;
    j->cols[i] = cols;
    j->across[i] = (cols + 255) / 256;
    j->first[i] = j->pieces;
    j->pieces += rows * j->across[i];
}
static void add_copy(CopyJobs* j, const Matrix& m, const Prepared& p) {
    if (!p.op.p || p.op.planes == 2 || p.op.p == m.p) return;
    add_copy_rows(j, m.p, const_cast<void*>(p.op.p), m.rows, m.cols, m.ld, p.op.ld);
}
int launch_copies(const CopyJobs& j, cudaStream_t st) {
    const long long blocks = (j.pieces + 7) / 8;
    return j.count ? launch_chained(copy_rows_kernel, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), 256, 0, st, 1, j) : EBS_OK;
}
static int launch_splits(const SplitJobs& all, cudaStream_t st) {
    long long elements = 0;
    for (int i = 0; i < all.count; ++i) elements += all.job[i].rows * all.job[i].cols;
    const bool together = elements < (1LL << 22);
    for (int pass = 0; pass < (together ? 1 : 2); ++pass) {
        SplitJobs jobs = {};
        unsigned blocks = 0;
        bool rows = false, columns = false;
        for (int i = 0; i < all.count; ++i) {
            if (!together && all.job[i].across != pass) continue;
            (all.job[i].across ? columns : rows) = true;
            jobs.job[jobs.count] = all.job[i];
            jobs.job[jobs.count++].first = blocks;
            blocks += all.job[i].blocks;
        }
        if (!blocks) continue;
        const int rc = launch_chained(rows && columns ? split_kernel<true, true> : rows ? split_kernel<true, false> : split_kernel<false, true>, dim3(blocks), 256, 0, st, 1, jobs);
        if (rc) return rc;
    }
    return EBS_OK;
}

// A product of prepared operands; a: its rows are the result's (across: its columns), likewise b for the result's columns.
static GemmShape product_shape(const Prepared& a, const Matrix& am, const Prepared& b, const Matrix& bm, int red) {
    return GemmShape{(int)(a.op.mn_major ? am.cols : am.rows), (int)(b.op.mn_major ? bm.cols : bm.rows), red, 1};
}
static GemmOut product_out(const Prepared& a, const Matrix& am, const Prepared& b, const Matrix& bm, int red, GemmOut o, int dtype) {
    if (dtype != EBS_F32) return o;
    o.row_exp = a.exps;
    o.col_exp = b.exps;
    o.fp32.a = static_cast<const float*>(am.p);
    o.fp32.b = static_cast<const float*>(bm.p);
    o.fp32.a_row = a.op.mn_major ? 1 : am.ld;
    o.fp32.a_red = a.op.mn_major ? am.ld : 1;
    o.fp32.b_col = b.op.mn_major ? 1 : bm.ld;
    o.fp32.b_red = b.op.mn_major ? bm.ld : 1;
    o.fp32.red = red;
    return o;
}

// ---------------------------------------------------------------------------------------------------- dz and dbias
struct DzArgs {
    const void *dy, *z;
    long long ldy, ldz, lddz;
    int m, n, act;
    float store;
    void *dz, *dbias;
    float* part;                           // [chunks][n]: column sums of dz
    unsigned* tops;                        // [chunks][n]: largest magnitudes of dz (fp32, for the split)
    int chunks;
    unsigned blocks;                       // of this part of the launch; the column tops of `jobs` follow
};

// dz = dy * act'(z), stored times `store`, and the column sums of dz before its rounding.  A block takes 32 * N columns and the rows of one
// chunk; a lane has N neighbouring columns (VEC: 16 bytes an access) or, where the rows start anywhere, every 32nd.  fp32: the column
// tops of dz here, those of other matrices (jobs with chunks) in further blocks.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256, 4) linear_dz_kernel(const __grid_constant__ DzArgs g, const __grid_constant__ SplitJobs jobs) {
    constexpr int N = Pack<T>::N, U = 2;                      // U rows under way: enough bytes in flight to cover the memory's latency
    __shared__ float sums[8][32 * N + 4];
    __shared__ unsigned part[8][128];
    let_next_kernel_start();
    wait_for_previous_kernel();
    if (blockIdx.x >= g.blocks) {
        const SplitJob& j = jobs.job[job_of(jobs, blockIdx.x)];
        column_tops(j, blockIdx.x - j.first, part);
        return;
    }
    const int across = (g.n + 32 * N - 1) / (32 * N), bx = (int)(blockIdx.x % across), by = (int)(blockIdx.x / across);
    const int lane = threadIdx.x & 31, y = threadIdx.x >> 5, col0 = bx * 32 * N;
    auto local = [&](int e) { return VEC ? lane * N + e : lane + 32 * e; };              // column of element e in this block's
    const long long r0 = (long long)g.m * by / g.chunks, r1 = (long long)g.m * (by + 1) / g.chunks;
    const T *dy = static_cast<const T*>(g.dy) + col0, *z = static_cast<const T*>(g.z) + col0;
    T* dz = static_cast<T*>(g.dz) + col0;
    const int left = g.n - col0;
    float sum[N];
    unsigned top[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.0f;
    const bool whole = VEC && local(N - 1) < left;
    auto load = [&](const T* row) {
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        if (whole) return *reinterpret_cast<const uint4*>(row + local(0));
        T* t = reinterpret_cast<T*>(&u);
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (local(e) < left) t[e] = row[local(e)];
        return u;
    };
    if (local(0) < left)
        for (long long r = r0 + y; r < r1; r += 8 * U) {
            uint4 a[U], b[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (r + 8 * u < r1) {
                    a[u] = load(dy + (r + 8 * u) * g.ldy);
                    if (g.act) b[u] = load(z + (r + 8 * u) * g.ldz);
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (r + 8 * u >= r1) break;
                float v[N], zv[N];
                unpack<T>(a[u], v);
                if (g.act) unpack<T>(b[u], zv);
                switch (g.act) {
#define EBS_SLOPE_CASE(A) case A: _Pragma("unroll") for (int e = 0; e < N; ++e) v[e] *= activation_slope<sizeof(T) == 2>(zv[e], A); break;
                    EBS_SLOPE_CASE(EBS_ACT_RELU) EBS_SLOPE_CASE(EBS_ACT_GELU) EBS_SLOPE_CASE(EBS_ACT_GELU_TANH) EBS_SLOPE_CASE(EBS_ACT_SILU)
#undef EBS_SLOPE_CASE
                    default: break;
                }
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    sum[e] += v[e];
                    if (sizeof(T) == 4) top[e] = max(top[e], magnitude(v[e]));
                    if (std::is_same<T, __half>::value) v[e] *= g.store;
                }
                if (!g.dz) continue;
                T* to = dz + (r + 8 * u) * g.lddz;
                if (VEC) store_pack(to + local(0), v);        // (rows of dz are padded to whole packs)
                else
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        if (local(e) < left) to[local(e)] = from_f32<T>(v[e]);
            }
        }
    if (sizeof(T) == 4 && g.tops) {
#pragma unroll
        for (int e = 0; e < 4; ++e) part[y][local(e) & 127] = top[e];
        __syncthreads();
        if (threadIdx.x < 128 && (int)threadIdx.x < left) {
            unsigned t = 0u;
#pragma unroll
            for (int q = 0; q < 8; ++q) t = max(t, part[q][threadIdx.x]);
            g.tops[(size_t)by * g.n + col0 + threadIdx.x] = t;
        }
    }
    if (!g.dbias) return;
#pragma unroll
    for (int e = 0; e < N; ++e) sums[y][local(e)] = sum[e];
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * N && i < left; i += 256) {
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < 8; ++q) s += sums[q][i];
        if (g.chunks == 1) static_cast<T*>(g.dbias)[col0 + i] = from_f32<T>(s);
        else g.part[(size_t)by * g.n + col0 + i] = s;
    }
}
// dbias from the chunks' sums, 32 columns a block, its eight warps take every eighth chunk; behind those blocks the column tops of the jobs,
// over their chunks likewise (into the first chunk's place).
template <typename T>
__global__ void __launch_bounds__(256) linear_chunks_kernel(const float* __restrict__ part, int chunks, int n, T* __restrict__ dbias, unsigned blocks, const __grid_constant__ SplitJobs jobs) {
    __shared__ unsigned words[8][33];
    let_next_kernel_start();
    wait_for_previous_kernel();
    const int lane = threadIdx.x & 31, y = threadIdx.x >> 5;
    if (blockIdx.x < blocks) {
        const int c = blockIdx.x * 32 + lane;
        float s = 0.0f;
        if (c < n)
#pragma unroll 8
            for (int i = y; i < chunks; i += 8) s += part[(size_t)i * n + c];
        words[y][lane] = __float_as_uint(s);
        __syncthreads();
        if (y == 0 && c < n) {
            for (int q = 1; q < 8; ++q) s += __uint_as_float(words[q][lane]);
            dbias[c] = from_f32<T>(s);
        }
        return;
    }
    const SplitJob& j = jobs.job[job_of(jobs, blockIdx.x)];
    const int c = (int)(blockIdx.x - j.first) * 32 + lane;
    unsigned t = 0u;
    if (c < j.cols)
#pragma unroll 8
        for (int i = y; i < j.chunks; i += 8) t = max(t, j.tops[(size_t)i * j.cols + c]);
    words[y][lane] = t;
    __syncthreads();                                          // (every chunk of these columns is read)
    if (y == 0 && c < j.cols) {
        for (int q = 1; q < 8; ++q) t = max(t, words[q][lane]);
        j.tops[c] = t;
    }
}
template <typename T>
static int launch_dz(DzArgs& g, SplitJobs& jobs, cudaStream_t st) {
    constexpr int N = Pack<T>::N;
    const bool vec = g.ldy % N == 0 && (!g.act || g.ldz % N == 0);
    g.blocks = g.dz || g.dbias || g.tops ? (unsigned)((g.n + 32 * N - 1) / (32 * N) * g.chunks) : 0u;
    SplitJobs tops = {};
    unsigned blocks = g.blocks;
    for (int i = 0; i < jobs.count; ++i) {
        if (!jobs.job[i].across || jobs.job[i].tops == g.tops) continue;
        tops.job[tops.count] = jobs.job[i];
        tops.job[tops.count++].first = blocks;
        blocks += jobs.job[i].blocks;
    }
    int rc = EBS_OK;
    if (blocks) rc = launch_chained(vec ? linear_dz_kernel<T, true> : linear_dz_kernel<T, false>, dim3(blocks), 256, 0, st, 1, g, tops);
    if (rc) return rc;
    const unsigned sums = g.dbias && g.chunks > 1 ? (unsigned)((g.n + 31) / 32) : 0u;
    SplitJobs chunked = {};
    blocks = sums;
    for (int i = 0; i < jobs.count; ++i) {
        if (!jobs.job[i].across || jobs.job[i].joined == jobs.job[i].chunks) continue;
        chunked.job[chunked.count] = jobs.job[i];
        chunked.job[chunked.count++].first = blocks;
        blocks += (unsigned)((jobs.job[i].cols + 31) / 32);
    }
    if (blocks) rc = launch_chained(linear_chunks_kernel<T>, dim3(blocks), 256, 0, st, 1, (const float*)g.part, g.chunks, g.n, static_cast<T*>(g.dbias), sums, chunked);
    return rc;
}

// ---------------------------------------------------------------------------------------------------- the calls
struct LinearTensors {
    const void *x, *w, *bias, *residual, *dy, *z;
    void *y, *keep, *dx, *dw, *dbias;
};
// Runs the call, or (run = false) counts its workspace.
static int forward(const ebs_linear_desc& d, const LinearTensors& t, Carver& ws, bool run, cudaStream_t st) {
    if (d.m == 0) return EBS_OK;
    GemmOut o;
    o.bias = t.bias; o.residual = t.residual; o.z = t.keep; o.y = t.y; o.act = d.act;
    o.ldr = d.ldr; o.ldz = d.ldz; o.ldy = d.ldy;
    if (d.m <= (d.dtype == EBS_F32 ? 4 : 1)) return run ? launch_gemm_rows(t.x, d.ldx, t.w, d.ldw, d.m, d.n, d.k, o, d.dtype, st) : EBS_OK;
    const Matrix xm{t.x, d.m, d.ldx, d.k}, wm{t.w, d.n, d.ldw, d.k};
    SplitJobs jobs = {};
    const Prepared x = plan_operand(xm, d.dtype, false, ws, &jobs), w = plan_operand(wm, d.dtype, false, ws, &jobs);
    const int planes = d.dtype == EBS_F32 ? 2 : 1;
    float* scratch = ws.take<float>(gemm_route(GemmShape{d.m, d.n, d.k, 1}, planes).scratch / 4);
    if (!run) return EBS_OK;
    int rc;
    CopyJobs copies = {};
    add_copy(&copies, xm, x);
    add_copy(&copies, wm, w);
    if ((rc = launch_splits(jobs, st)) || (rc = launch_copies(copies, st))) return rc;
    return launch_gemm(x.op, w.op, product_shape(x, xm, w, wm, d.k), scratch, product_out(x, xm, w, wm, d.k, o, d.dtype), d.dtype, st);
}
static int backward(const ebs_linear_desc& d, const LinearTensors& t, Carver& ws, bool run, cudaStream_t st) {
    int rc = EBS_OK;
    if (d.m == 0) {
        if (!run) return EBS_OK;
        const size_t size = element_size(d.dtype);
        if (t.dw && check_cuda(cudaMemset2DAsync(t.dw, d.ldw * size, 0, d.k * size, d.n, st))) return EBS_ERR_CUDA;
        if (t.dbias && check_cuda(cudaMemsetAsync(t.dbias, 0, d.n * size, st))) return EBS_ERR_CUDA;
        return EBS_OK;
    }
    const bool fp32 = d.dtype == EBS_F32, want_dx = t.dx || !run, want_dw = t.dw || !run;
    const Matrix wm{t.w, d.n, d.ldw, d.k}, xm{t.x, d.m, d.ldx, d.k};
    Matrix dm{t.dy, d.m, d.ldy, d.n};
    DzArgs g = {t.dy, t.z, d.ldy, d.ldz, 0, d.m, d.n, d.act, dz_store_scale(d), nullptr, t.dbias, nullptr, nullptr, 0, 0};
    // 16-bit columns come 256 a block, fp32 columns 128: the chunks of the sums follow the sizes, not the strides
    g.chunks = row_chunks(d.m, (d.n + (fp32 ? 127 : 255)) / (fp32 ? 128 : 256));
    if (d.act) {
        g.lddz = round8(d.n);
        g.dz = fp32 ? (void*)ws.take<float>((size_t)d.m * g.lddz) : (void*)ws.take<uint16_t>((size_t)d.m * g.lddz);
        dm.p = g.dz;
        dm.ld = g.lddz;
        if (!want_dx && !want_dw) g.dz = nullptr;
    }
    if (g.chunks > 1) g.part = ws.take<float>((size_t)g.chunks * d.n);
    SplitJobs jobs = {};
    Prepared rows, columns, w, x;                            // dz for dx and for dW, W, x
    if (fp32) {
        if (want_dw) {
            columns = plan_operand(dm, d.dtype, true, ws, &jobs);
            g.tops = jobs.job[0].tops;
            g.chunks = jobs.job[0].chunks;                   // (the same number)
        }
        if (want_dx) rows = plan_operand(dm, d.dtype, false, ws, &jobs);
    } else {
        rows = columns = plan_operand(dm, d.dtype, false, ws, &jobs);
        columns.op.mn_major = true;                          // one matrix, or one copy of it, serves both products
    }
    if (want_dx) w = plan_operand(wm, d.dtype, true, ws, &jobs);
    if (want_dw) x = plan_operand(xm, d.dtype, true, ws, &jobs);
    size_t need = 0;                                          // the products run one after the other
    const int planes = fp32 ? 2 : 1;
    if (want_dx) need = gemm_route(GemmShape{d.m, d.k, d.n, 1}, planes).scratch;
    if (want_dw) { const size_t b = gemm_route(GemmShape{d.n, d.k, d.m, 1}, planes).scratch; need = b > need ? b : need; }
    float* scratch = ws.take<float>(need / 4);
    if (!run) return EBS_OK;
    if (fp32) rc = launch_dz<float>(g, jobs, st);
    else if (d.act || t.dbias) rc = d.dtype == EBS_F16 ? launch_dz<__half>(g, jobs, st) : launch_dz<__nv_bfloat16>(g, jobs, st);
    if (rc || (rc = launch_splits(jobs, st))) return rc;
    CopyJobs copies = {};
    if (t.dx || t.dw) add_copy(&copies, dm, rows);
    if (t.dx) add_copy(&copies, wm, w);
    if (t.dw) add_copy(&copies, xm, x);
    if ((rc = launch_copies(copies, st))) return rc;
    GemmOut ox, ow;
    ox.alpha = ow.alpha = 1.0f / dz_store_scale(d);
    ox.y = t.dx; ox.ldy = d.ldx;
    ow.y = t.dw; ow.ldy = d.ldw;
    if (t.dx) ox = product_out(rows, dm, w, wm, d.n, ox, d.dtype);
    if (t.dw) ow = product_out(columns, dm, x, xm, d.m, ow, d.dtype);
    const GemmShape sx{d.m, d.k, d.n, 1}, sw{d.n, d.k, d.m, 1};
    if (t.dx && t.dw && !gemm_route(sx, planes).pair && !gemm_route(sw, planes).pair)
        return launch_gemm_tiles({{rows.op, w.op, sx}, {columns.op, x.op, sw}}, {ox, ow}, d.dtype, st);
    if (t.dx && (rc = launch_gemm(rows.op, w.op, sx, scratch, ox, d.dtype, st))) return rc;
    if (t.dw && (rc = launch_gemm(columns.op, x.op, sw, scratch, ow, d.dtype, st))) return rc;
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
    if (complete_linear(desc, &d)) return 0;
    return linear_workspace(d, backward != 0);
}

int ebs_linear_forward(const void* x, const void* w, const void* bias, const void* residual, const ebs_linear_desc* desc, void* y, void* z,
                       void* workspace, size_t workspace_bytes, void* stream) {
    ebs_linear_desc d;
    const int rc = complete_linear(desc, &d);
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
    const int rc = complete_linear(desc, &d);
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
