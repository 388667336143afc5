// Norm of all gradients of a network and their clipping.  See include/ebs.h.
//
// Bound by the bytes: one pass reads every gradient for the sum of squares, one reads it again and writes it (537 million bf16: 154 us, 7.0 TB/s, and 333 us, 6.4 TB/s).  The work list ("plan") cuts all
// tensors into chunks, a record each, so that a block learns from one 48-byte load what to do next, however many tensors there are and whatever their
// sizes; the next record is on its way while a chunk is read.  The second pass takes the chunks from the last to the first, so that it begins with what the
// second-level cache has (from the first to the last: 73 MB of padded fp16 rows, again and again, 42.5 us instead of 37.4, 134 MB 75.0 and 68.8, 268 MB 142.8 and 138.3, 1.07 GB the same).
//
// The sum is taken in 64 bits.  A pack of 16 bytes is squared and added in fp32 first (relative error 2^-22 of the pack at most), unless that sum
// leaves the range where neither an overflow nor a lost small square matters; then each square is taken in 64 bits.  Partial sums are added in
// an order that goes by the plan alone.
#include <algorithm>
#include <cstring>
#include <new>

#include "tensors.cuh"

namespace ebs {

constexpr int CLIP_BLOCKS = 148 * 4;        // at most: a wave of blocks of 256 threads
constexpr int CLIP_THREADS = 256;
constexpr int CLIP_UNROLL = 8;              // packs of a thread under way: 32 KB a block (four, and records loaded when they are needed: 1.07 GB read at 3.4 TB/s)
constexpr int CLIP_NARROW = 512;            // bytes of a row that a warp's lanes would not fill
// Bytes of a chunk of pieces of one row or of narrow rows: as many as the block has under way; a network of a few MB is cut finer, so that every SM has some.
constexpr long long CLIP_CHUNK = CLIP_THREADS * 16 * CLIP_UNROLL, CLIP_CHUNK_SMALL = CLIP_THREADS * 16, CLIP_SMALL = 8 << 20;

// rows = 1: the block's threads share the row; more: a warp takes a row, or, of narrow rows, the threads their pieces of 16 bytes.
struct alignas(16) ClipChunk {
    const void* in;
    void* out;
    long long ld_in, ld_out;
    int rows, cols, dtype, pad;
};
static_assert(sizeof(ClipChunk) == EBS_CLIP_CHUNK_BYTES, "chunk record");

__device__ __forceinline__ ClipChunk load_chunk(const ClipChunk* p) {
    const uint4* q = reinterpret_cast<const uint4*>(p);
    const uint4 a = q[0], b = q[1], d = q[2];
    auto wide = [](uint32_t low, uint32_t high) { return (long long)((unsigned long long)high << 32 | low); };
    ClipChunk c;
    c.in = reinterpret_cast<const void*>(wide(a.x, a.y));
    c.out = reinterpret_cast<void*>(wide(a.z, a.w));
    c.ld_in = wide(b.x, b.y);
    c.ld_out = wide(b.z, b.w);
    c.rows = (int)d.x;
    c.cols = (int)d.y;
    c.dtype = (int)d.z;
    return c;
}

// The sum of the squares of one pack.
template <typename T>
__device__ __noinline__ double squares_of(const uint4 u) {
    double sum = 0.0;
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = __uint_as_float(w[i]), b = 0.0f;
        if (sizeof(T) == 2) {
            a = to_f32(reinterpret_cast<const T*>(&w[i])[0]);
            b = to_f32(reinterpret_cast<const T*>(&w[i])[1]);
        }
        sum += (double)a * (double)a + (double)b * (double)b;
    }
    return sum;
}
// In fp32; false: it is left out, for squares_of (below 1e-28 a square of the pack may be lost that matters, above 1e37 one may be infinite that is not).
template <typename T>
__device__ __forceinline__ bool add_squares(const uint4& u, double& sum) {
    constexpr int N = Pack<T>::N;
    float v[N], s = 0.0f;
    unpack<T>(u, v);
#pragma unroll
    for (int i = 0; i < N; ++i) s = fmaf(v[i], v[i], s);
    const bool fits = s >= 1e-28f && s <= 1e37f;
    sum += (double)(fits ? s : 0.0f);
    return fits || ((u.x | u.y | u.z | u.w) & (sizeof(T) == 2 ? 0x7fff7fffu : 0x7fffffffu)) == 0u;
}
template <typename T>
__device__ __forceinline__ void add_square(T x, double& sum) {
    const double d = (double)to_f32(x);
    sum += d * d;
}
// Elements before the first 16-byte boundary of a row (its elements lie on multiples of their size).
template <typename T>
__device__ __forceinline__ int head_of(const T* p, int cols) {
    const int h = (int)((16u - ((unsigned)(uintptr_t)p & 15u)) & 15u) / (int)sizeof(T);
    return h < cols ? h : cols;
}
template <typename T>
__device__ __forceinline__ void row_squares(const T* p, int cols, int t, int step, double& sum) {
    constexpr int N = Pack<T>::N;
    const int head = head_of(p, cols), packs = (cols - head) / N, tail = head + packs * N;
    // (a head and a tail have fewer elements than a warp has lanes)
    const T first = t < head ? p[t] : from_f32<T>(0.0f), last = tail + t < cols ? p[tail + t] : from_f32<T>(0.0f);
    const uint4* q = reinterpret_cast<const uint4*>(p + head);
    for (int i = t; i < packs; i += CLIP_UNROLL * step) {
        uint4 u[CLIP_UNROLL];
#pragma unroll
        for (int j = 0; j < CLIP_UNROLL; ++j) u[j] = i + j * step < packs ? q[i + j * step] : make_uint4(0u, 0u, 0u, 0u);
        unsigned left_out = 0u;
#pragma unroll
        for (int j = 0; j < CLIP_UNROLL; ++j) left_out |= (add_squares<T>(u[j], sum) ? 0u : 1u) << j;
        if (left_out)                                             // (rare: read again, so that nothing is kept for it)
#pragma unroll 1
            for (int j = 0; j < CLIP_UNROLL; ++j)
                if (left_out >> j & 1u) sum += squares_of<T>(q[i + j * step]);
    }
    if (t < N) {
        add_square(first, sum);
        add_square(last, sum);
    }
}
// Several rows that start anywhere, as the 16-byte pieces of memory that they lie in: piece `at` of all is one of a row's `pieces` (as many as its elements can touch); its
// first element is element `start` of the row, which may lie before the row's first one.  (23 layers of 1792 x 64 and 64 x 1792 bf16, rows of 65 and 1793: an element a thread 44 us, so 31.  Wide rows
// not: pieces at their ends cost more than lanes without work, 73 MB of padded fp16 rows 85 us instead of 46.)
template <typename T>
struct Piece {
    const T* row;
    int r, start;
};
template <typename T> __device__ __forceinline__ unsigned pieces_of(int cols) { return (unsigned)(cols + 2 * Pack<T>::N - 2) / (unsigned)Pack<T>::N; }
template <typename T>
__device__ __forceinline__ Piece<T> piece_at(const ClipChunk& c, unsigned pieces, unsigned at) {
    Piece<T> q;
    q.r = (int)(at / pieces);
    q.row = static_cast<const T*>(c.in) + q.r * c.ld_in;
    q.start = (int)(at - (unsigned)q.r * pieces) * Pack<T>::N - (int)((unsigned)(uintptr_t)q.row & 15u) / (int)sizeof(T);
    return q;
}
// Zero where there is no element of the row.
template <typename T>
__device__ __forceinline__ uint4 load_piece(const Piece<T>& q, int cols) {
    constexpr int N = Pack<T>::N;
    if (q.start >= 0 && q.start + N <= cols) return *reinterpret_cast<const uint4*>(q.row + q.start);
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (q.start + e >= 0 && q.start + e < cols) reinterpret_cast<T*>(&u)[e] = q.row[q.start + e];
    return u;
}
template <typename T>
__device__ __forceinline__ void rows_squares(const ClipChunk& c, double& sum) {
    const unsigned pieces = pieces_of<T>(c.cols), all = (unsigned)c.rows * pieces;
    for (unsigned i = threadIdx.x; i < all; i += CLIP_UNROLL * CLIP_THREADS) {
        uint4 u[CLIP_UNROLL];
#pragma unroll
        for (unsigned j = 0; j < CLIP_UNROLL; ++j) u[j] = i + j * CLIP_THREADS < all ? load_piece(piece_at<T>(c, pieces, i + j * CLIP_THREADS), c.cols) : make_uint4(0u, 0u, 0u, 0u);
        unsigned left_out = 0u;
#pragma unroll
        for (int j = 0; j < CLIP_UNROLL; ++j) left_out |= (add_squares<T>(u[j], sum) ? 0u : 1u) << j;
        if (left_out)
#pragma unroll 1
            for (unsigned j = 0; j < CLIP_UNROLL; ++j)
                if (left_out >> j & 1u) sum += squares_of<T>(load_piece(piece_at<T>(c, pieces, i + j * CLIP_THREADS), c.cols));
    }
}
template <typename T>
__device__ __forceinline__ void chunk_squares(const ClipChunk& c, double& sum) {
    if (c.rows == 1) row_squares(static_cast<const T*>(c.in), c.cols, threadIdx.x, CLIP_THREADS, sum);
    else if (c.cols * (int)sizeof(T) < CLIP_NARROW) rows_squares<T>(c, sum);
    else
        for (int r = threadIdx.x >> 5; r < c.rows; r += CLIP_THREADS / 32) row_squares(static_cast<const T*>(c.in) + r * c.ld_in, c.cols, threadIdx.x & 31, 32, sum);
}
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double part[CLIP_THREADS / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int i = 0; i < CLIP_THREADS / 32; ++i) v += part[i];
    return v;
}

__global__ void __launch_bounds__(CLIP_THREADS, 4) clip_norm_kernel(const ClipChunk* __restrict__ chunks, long long count, double* __restrict__ partial) {
    let_next_kernel_start();
    wait_for_previous_kernel();
    double sum = 0.0;
    ClipChunk next = load_chunk(chunks + blockIdx.x);             // (no more blocks than chunks)
    for (long long i = blockIdx.x; i < count; i += gridDim.x) {
        const ClipChunk c = next;
        if (i + gridDim.x < count) next = load_chunk(chunks + i + gridDim.x);
        if (c.dtype == EBS_F32) chunk_squares<float>(c, sum);
        else if (c.dtype == EBS_F16) chunk_squares<__half>(c, sum);
        else chunk_squares<__nv_bfloat16>(c, sum);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

template <typename T>
__device__ __forceinline__ void scale_pack(uint4& u, float f) {
    float v[Pack<T>::N];
    unpack<T>(u, v);
#pragma unroll
    for (int i = 0; i < Pack<T>::N; ++i) v[i] *= f;
    store_pack(reinterpret_cast<T*>(&u), v);
}
template <typename T>
__device__ __forceinline__ void row_scale(const T* p, T* to, int cols, int t, int step, float f) {
    constexpr int N = Pack<T>::N;
    if ((((uintptr_t)p ^ (uintptr_t)to) & 15u) != 0) {        // in and out never on a boundary together
        for (int i = t; i < cols; i += step) to[i] = from_f32<T>(to_f32(p[i]) * f);
        return;
    }
    const int head = head_of(p, cols), packs = (cols - head) / N, tail = head + packs * N;
    const uint4* q = reinterpret_cast<const uint4*>(p + head);
    uint4* r = reinterpret_cast<uint4*>(to + head);
    constexpr int U = CLIP_UNROLL / 2;                        // (with the bytes written as many are under way)
    int i = t;
    for (; i + (U - 1) * step < packs; i += U * step) {
        uint4 u[U];
#pragma unroll
        for (int j = 0; j < U; ++j) u[j] = q[i + j * step];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            scale_pack<T>(u[j], f);
            r[i + j * step] = u[j];
        }
    }
    for (; i < packs; i += step) {
        uint4 u = q[i];
        scale_pack<T>(u, f);
        r[i] = u;
    }
    if (t < head) to[t] = from_f32<T>(to_f32(p[t]) * f);
    if (tail + t < cols) to[tail + t] = from_f32<T>(to_f32(p[tail + t]) * f);
}
template <typename T>
__device__ __forceinline__ void rows_scale(const ClipChunk& c, float f) {
    constexpr int N = Pack<T>::N, U = CLIP_UNROLL / 2;
    const unsigned pieces = pieces_of<T>(c.cols), all = (unsigned)c.rows * pieces;
    for (unsigned i = threadIdx.x; i < all; i += U * CLIP_THREADS) {
        uint4 u[U];
#pragma unroll
        for (unsigned j = 0; j < U; ++j)
            if (i + j * CLIP_THREADS < all) u[j] = load_piece(piece_at<T>(c, pieces, i + j * CLIP_THREADS), c.cols);
#pragma unroll
        for (unsigned j = 0; j < U; ++j) {
            if (i + j * CLIP_THREADS >= all) break;
            const Piece<T> q = piece_at<T>(c, pieces, i + j * CLIP_THREADS);
            T* to = static_cast<T*>(c.out) + q.r * c.ld_out;
            scale_pack<T>(u[j], f);
            if (q.start >= 0 && q.start + N <= c.cols && (((uintptr_t)(to + q.start)) & 15u) == 0) *reinterpret_cast<uint4*>(to + q.start) = u[j];
            else
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (q.start + e >= 0 && q.start + e < c.cols) to[q.start + e] = reinterpret_cast<const T*>(&u[j])[e];
        }
    }
}
template <typename T>
__device__ __forceinline__ void chunk_scale(const ClipChunk& c, float f) {
    if (c.rows == 1) row_scale(static_cast<const T*>(c.in), static_cast<T*>(c.out), c.cols, threadIdx.x, CLIP_THREADS, f);
    else if (c.cols * (int)sizeof(T) < CLIP_NARROW) rows_scale<T>(c, f);
    else
        for (int r = threadIdx.x >> 5; r < c.rows; r += CLIP_THREADS / 32)
            row_scale(static_cast<const T*>(c.in) + r * c.ld_in, static_cast<T*>(c.out) + r * c.ld_out, c.cols, threadIdx.x & 31, 32, f);
}

__global__ void __launch_bounds__(CLIP_THREADS, 4) clip_scale_kernel(const ClipChunk* __restrict__ chunks, long long count, const double* __restrict__ partial, int parts,
                                                                  float max_norm, float* __restrict__ norm_out) {
    let_next_kernel_start();
    wait_for_previous_kernel();
    ClipChunk next = {};
    if (blockIdx.x < count) next = load_chunk(chunks + count - 1 - blockIdx.x);
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += CLIP_THREADS) sum += partial[i];
    const double norm = sqrt(block_sum(sum));
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const float f = norm <= (double)max_norm ? 1.0f : (float)((double)max_norm / norm);      // (a NaN norm: NaN)
    for (long long i = (long long)count - 1 - blockIdx.x; i >= 0; i -= gridDim.x) {
        const ClipChunk c = next;
        if (i >= gridDim.x) next = load_chunk(chunks + i - gridDim.x);
        if (f == 1.0f && c.in == c.out) continue;
        if (c.dtype == EBS_F32) chunk_scale<float>(c, f);
        else if (c.dtype == EBS_F16) chunk_scale<__half>(c, f);
        else chunk_scale<__nv_bfloat16>(c, f);
    }
}

// ---------------------------------------------------------------------------------------------------- the plan
// A tensor with its strides filled in; rows that lie one behind the other are one row.
static int complete_tensor(const ebs_clip_tensor& in, ebs_clip_tensor* t) {
    *t = in;
    if (t->rows < 0 || t->cols < 0 || !real_dtype(t->dtype)) return EBS_ERR_INVALID_ARG;
    if (t->ld_in == 0) t->ld_in = t->cols;
    if (t->ld_out == 0) t->ld_out = t->cols;
    if (t->ld_in < t->cols || t->ld_out < t->cols) return EBS_ERR_INVALID_ARG;
    const long long limit = 1LL << 40;
    if (t->cols > limit || t->rows > limit) return EBS_ERR_OVERFLOW;
    if (t->rows == 0 || t->cols == 0) {
        t->rows = t->cols = 0;
        return EBS_OK;
    }
    if (t->ld_in > limit / t->rows || t->ld_out > limit / t->rows) return EBS_ERR_OVERFLOW;
    const uintptr_t size = element_size(t->dtype);
    if (!t->in_dev || !t->out_dev || (uintptr_t)t->in_dev % size || (uintptr_t)t->out_dev % size) return EBS_ERR_INVALID_ARG;
    if (t->in_dev == t->out_dev && t->ld_in != t->ld_out) return EBS_ERR_INVALID_ARG;
    if (t->rows > 1 && t->ld_in == t->cols && t->ld_out == t->cols) {
        t->cols *= t->rows;
        t->ld_in = t->ld_out = t->cols;
        t->rows = 1;
    }
    return EBS_OK;
}
// How a tensor of a network of `bytes` is cut: whole rows, eights of them where a warp takes one, or pieces of one.  Strided rows of 6 to 16 KB go one by one where the network has no
// eight of them for every SM: 512 rows of 16 KB 10.0 us in eights, 8.2 one by one, 1024 of 8 KB 12.8 and 9.6, 1024 of 16 KB 20.2 and 11.7; 4096 of 8 KB 14.8 and 23.5, 1900 of 4.4 KB 10.1 and 12.4.
struct Cut {
    long long rows, cols;
};
static Cut cut_of(const ebs_clip_tensor& t, long long bytes) {
    const long long size = (long long)element_size(t.dtype), chunk = (bytes <= CLIP_SMALL ? CLIP_CHUNK_SMALL : CLIP_CHUNK) / size, row = t.cols * size;
    if (t.rows == 1 || row > 16384) return {1, chunk};
    if (row > 6144 && bytes < 148 * 8 * row) return {1, t.cols};
    const long long r = chunk / t.cols & ~7LL;
    return {r < 8 ? 8 : r, t.cols};
}
static long long tensor_chunks(const ebs_clip_tensor& t, long long bytes) {
    if (t.rows == 0) return 0;
    const Cut c = cut_of(t, bytes);
    return (t.rows + c.rows - 1) / c.rows * ((t.cols + c.cols - 1) / c.cols);
}
// What a tensor reads or writes, in bytes; pitch: 0 for one row.
struct Extent {
    uintptr_t begin, end, pitch, width;
    int tensor;
    bool out;
};
static bool share(const Extent& a, const Extent& b) {
    // (their extents meet, b begins behind a: the caller knows; matrices of different strides are not looked at further)
    if (a.pitch == 0 || (b.pitch != 0 && a.pitch != b.pitch)) return true;
    const uintptr_t d = (b.begin - a.begin) % a.pitch;
    return !(d >= a.width && a.pitch - d >= b.width);
}

}  // namespace ebs

using namespace ebs;

extern "C" {

int ebs_clip_plan(const ebs_clip_tensor* tensors, int count, void* plan_host, long long* chunks) {
    if (!chunks || count < 0 || (count && !tensors)) return EBS_ERR_INVALID_ARG;
    long long total = 0, bytes = 0;
    for (int i = 0; i < count; ++i) {
        ebs_clip_tensor t;
        const int rc = complete_tensor(tensors[i], &t);
        if (rc) return rc;
        bytes += t.rows * t.cols * (long long)element_size(t.dtype);
        if (bytes > (1LL << 42)) return EBS_ERR_OVERFLOW;
    }
    for (int i = 0; i < count; ++i) {
        ebs_clip_tensor t;
        complete_tensor(tensors[i], &t);
        total += tensor_chunks(t, bytes);
        if (total > (1LL << 31)) return EBS_ERR_OVERFLOW;
    }
    // no output may share an element with another tensor: extents in the order of their addresses
    Extent* e = new (std::nothrow) Extent[2 * (size_t)count + 1];
    if (!e) return EBS_ERR_OVERFLOW;
    int n = 0;
    for (int i = 0; i < count; ++i) {
        ebs_clip_tensor t;
        complete_tensor(tensors[i], &t);
        if (t.rows == 0) continue;
        const uintptr_t size = element_size(t.dtype);
        for (int out = 0; out < 2; ++out) {
            const uintptr_t p = (uintptr_t)(out ? t.out_dev : t.in_dev), ld = (uintptr_t)(out ? t.ld_out : t.ld_in);
            e[n++] = Extent{p, p + ((uintptr_t)(t.rows - 1) * ld + (uintptr_t)t.cols) * size, t.rows > 1 ? ld * size : 0, (uintptr_t)t.cols * size, i, out == 1};
        }
    }
    std::sort(e, e + n, [](const Extent& a, const Extent& b) { return a.begin < b.begin; });
    bool apart = true;
    for (int i = 0; i < n && apart; ++i)
        for (int j = i + 1; j < n && e[j].begin < e[i].end && apart; ++j) {
            if (!e[i].out && !e[j].out) continue;
            if (e[i].tensor == e[j].tensor && e[i].begin == e[j].begin) continue;             // (in place)
            apart = !share(e[i], e[j]);
        }
    delete[] e;
    if (!apart) return EBS_ERR_INVALID_ARG;
    if (plan_host) {
        if (*chunks < total) return EBS_ERR_INVALID_ARG;
        char* to = static_cast<char*>(plan_host);
        for (int i = 0; i < count; ++i) {
            ebs_clip_tensor t;
            complete_tensor(tensors[i], &t);
            if (t.rows == 0) continue;
            const long long size = (long long)element_size(t.dtype);
            const Cut cut = cut_of(t, bytes);
            for (long long r = 0; r < t.rows; r += cut.rows)
                for (long long c = 0; c < t.cols; c += cut.cols) {
                    ClipChunk k = {};
                    k.in = static_cast<const char*>(t.in_dev) + (r * t.ld_in + c) * size;
                    k.out = static_cast<char*>(t.out_dev) + (r * t.ld_out + c) * size;
                    k.ld_in = t.ld_in;
                    k.ld_out = t.ld_out;
                    k.rows = (int)(t.rows - r < cut.rows ? t.rows - r : cut.rows);
                    k.cols = (int)(t.cols - c < cut.cols ? t.cols - c : cut.cols);
                    k.dtype = t.dtype;
                    memcpy(to, &k, sizeof(k));
                    to += sizeof(k);
                }
        }
    }
    *chunks = total;
    return EBS_OK;
}

size_t ebs_clip_workspace_bytes(long long chunks) {
    if (chunks < 0 || chunks > (1LL << 31)) return 0;
    return round256((size_t)(chunks < 1 ? 1 : chunks < CLIP_BLOCKS ? chunks : CLIP_BLOCKS) * sizeof(double));
}

int ebs_clip_gradients(const void* plan_dev, long long chunks, float max_norm, float* norm_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
    if (chunks < 0 || chunks > (1LL << 31) || (chunks && !plan_dev) || !norm_dev || !workspace_dev || !(max_norm >= 0.0f)) return EBS_ERR_INVALID_ARG;
    if (!aligned16(plan_dev) || ((uintptr_t)norm_dev & 3u) || !aligned16(workspace_dev) || workspace_bytes < ebs_clip_workspace_bytes(chunks)) return EBS_ERR_INVALID_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const ClipChunk* plan = static_cast<const ClipChunk*>(plan_dev);
    double* partial = static_cast<double*>(workspace_dev);
    const int blocks = (int)(chunks < CLIP_BLOCKS ? chunks : CLIP_BLOCKS);
    if (blocks) {
        const int rc = launch_chained(clip_norm_kernel, dim3((unsigned)blocks), CLIP_THREADS, 0, st, 1, plan, chunks, partial);
        if (rc) return rc;
    }
    return launch_chained(clip_scale_kernel, dim3((unsigned)(blocks ? blocks : 1)), CLIP_THREADS, 0, st, 1, plan, chunks, (const double*)partial, blocks, max_norm, norm_dev);
}

}  // extern "C"
