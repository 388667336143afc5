// Persistent kernel of the large real-valued products: a pair of thread blocks on two SMs works on 256 x 256 results at a time.
//
// The MMAs are M = 256, N = 256 over both blocks' shared and tensor memory (cta_group::2): each block fetches its 128 rows of A and half
// of the 256 columns of B, so that an operand element crosses shared memory half as often as in a single block's 128 x 128 tile
// (that one reads 128 bytes a clock, all there are).  Warp 16 of each block fetches by TMA, warp 17 of the even block issues, warps 0-15
// of both take the sums of their 128 rows out of tensor memory (lanes 32 (w % 4), columns 64 (w / 4)) and write the results
// through a patch of shared memory, so that neighbouring lanes write neighbouring bytes.  Two accumulators of 256 columns: the
// MMAs of the next tile (split products: of the next few stages, see gemm_tile.cu) run while one is taken out.
#include "gemm_tile.cuh"

namespace ebs {

static __device__ unsigned long long g_gemm_pair_timeouts = 0ull;

// ---------------------------------------------------------------------------------------------------- results by rows
// Where the results' rows start on 16 bytes they leave by TMA: a thread has one row of the tile (its lane of tensor memory), finishes
// CW neighbouring columns in registers and puts them, 64 bytes, into its warp's buffer (64-byte swizzle: no bank conflicts), which one
// instruction stores, clipped at the edges.  Against lanes that share rows through a patch this leaves out nearly all address
// arithmetic; 8192 x 4096 with a reduction of 64 measured 46.8 us that way.
// Chunk byte 16 * c of row `row` of a buffer (base a multiple of 512 bytes).
constexpr int PAIR_BUFFER = 32 * 64;
__device__ __forceinline__ uint4* row_chunk(uint8_t* buffer, int row, int c) { return reinterpret_cast<uint4*>(buffer + row * 64 + ((c ^ ((row >> 1) & 3)) << 4)); }
// CW values -> this thread's 64 bytes.
template <typename T, int CW>
__device__ __forceinline__ void put_row(uint8_t* buffer, int lane, const float (&v)[CW]) {
    constexpr int N = Pack<T>::N;
    static_assert(CW == 4 * N, "64 bytes");
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        float t[N];
#pragma unroll
        for (int e = 0; e < N; ++e) t[e] = v[c * N + e];
        store_pack(reinterpret_cast<T*>(row_chunk(buffer, lane, c)), t);
    }
}
// A warp's ring of R buffers: a buffer is written again when the store that reads it, R stores back, is done with it.
template <int R>
struct RowRing {
    uint8_t* base;
    int lane, at = 0;
    __device__ __forceinline__ uint8_t* next() {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;\n" ::"n"(R - 1) : "memory");
        __syncwarp();
        uint8_t* p = base + at * PAIR_BUFFER;
        at = at + 1 == R ? 0 : at + 1;
        return p;
    }
    // after every lane has written its row; one store is one group
    __device__ __forceinline__ void store(const CUtensorMap* map, const uint8_t* buffer, int x, int y, int z, bool exists) {
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            if (exists) tma_store_3d(map, buffer, x, y, z);
            tma_store_commit();
        }
    }
};

// CW: columns at a time; begin: the columns' terms of a tile; ahead: what a row needs from memory; finish: the values into buffers.
template <class EPI> struct RowOut;

template <typename T>
struct RowOut<LinearOut<T>> {
    static constexpr bool HOLES = LinearOut<T>::HOLES;
    static constexpr int CW = 64 / sizeof(T), N = Pack<T>::N;
    struct Ahead { uint4 residual[4]; };
    static __device__ __forceinline__ void begin(const LinearOut<T>& e, float* terms, int columns, int at, int col, int cols) {
        terms[at] = e.o.bias && col < cols ? to_f32(static_cast<const T*>(e.o.bias)[col]) : 0.0f;
        if (sizeof(T) == 4) {                                 // (a factor of zero: an exponent that is not an ordinary one)
            const int x = col < cols ? e.o.col_exp[col] : 0;
            terms[columns + at] = abs(x) <= SCALE_PLAIN ? power_of_two(x) * e.o.alpha : 0.0f;
        }
    }
    static __device__ __forceinline__ int row_term(const LinearOut<T>& e, long long row, bool exists) { return sizeof(T) == 4 && exists ? e.o.row_exp[row] : 0; }
    static __device__ __forceinline__ void ahead(const LinearOut<T>& e, int, long long row, int col, int left, Ahead& a) {
        if (!e.o.residual || left <= 0) return;
        const T* p = static_cast<const T*>(e.o.residual) + row * e.o.ldr + col;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (c * N < left) a.residual[c] = load_raw(p + c * N, left - c * N, left >= (c + 1) * N);
    }
    static __device__ __forceinline__ void scale(const LinearOut<T>& e, float (&v)[CW], const float* terms, int columns, int col, int left, int row_term, uint8_t* buffer, int lane, bool exists, volatile int* holes) {
        if constexpr (sizeof(T) == 4) {
            float t[CW];
            bool plain = abs(row_term) <= SCALE_PLAIN;
#pragma unroll
            for (int i = 0; i < CW; i += 4) {
                *reinterpret_cast<float4*>(t + i) = *reinterpret_cast<const float4*>(terms + columns + i);
                plain = plain && t[i] != 0.0f && t[i + 1] != 0.0f && t[i + 2] != 0.0f && t[i + 3] != 0.0f;
            }
            if (plain) {
                const float f = power_of_two(row_term);
#pragma unroll
                for (int i = 0; i < CW; i += 4) {
                    const float4 b = *reinterpret_cast<const float4*>(terms + i);
                    v[i] = fmaf(v[i], f * t[i], b.x); v[i + 1] = fmaf(v[i + 1], f * t[i + 1], b.y);
                    v[i + 2] = fmaf(v[i + 2], f * t[i + 2], b.z); v[i + 3] = fmaf(v[i + 3], f * t[i + 3], b.w);
                }
                return;
            }
            // rare: through this thread's row of the buffer, an element at a time.  A hole becomes zero without the bias: act(0) is zero, so that y
            // gets the residual, which may be y itself and is read again by finish_infinite.
            put_row<float>(buffer, lane, v);
#pragma unroll 1
            for (int i = 0; i < CW && i < left; ++i) {
                float* at = reinterpret_cast<float*>(row_chunk(buffer, lane, i >> 2)) + (i & 3);
                bool hole = false;
                const float s = exists ? unscale(*at, row_term, e.o.col_exp[col + i], hole) : 0.0f;
                *at = hole ? 0.0f : fmaf(s, e.o.alpha, terms[i]);
                if (hole) *holes = 1;
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float4 q = *reinterpret_cast<const float4*>(row_chunk(buffer, lane, c));
                v[4 * c] = q.x; v[4 * c + 1] = q.y; v[4 * c + 2] = q.z; v[4 * c + 3] = q.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < CW; i += 4) {
                const float4 b = *reinterpret_cast<const float4*>(terms + i);
                v[i] = fmaf(v[i], e.o.alpha, b.x); v[i + 1] = fmaf(v[i + 1], e.o.alpha, b.y);
                v[i + 2] = fmaf(v[i + 2], e.o.alpha, b.z); v[i + 3] = fmaf(v[i + 3], e.o.alpha, b.w);
            }
        }
    }
    static __device__ __forceinline__ void activate(const LinearOut<T>& e, float (&v)[CW], const Ahead& a) {
        switch (e.o.act) {
#define EBS_ACT_CASE(A) case A: _Pragma("unroll") for (int i = 0; i < CW; ++i) v[i] = activation<sizeof(T) == 2>(v[i], A); break;
            EBS_ACT_CASE(EBS_ACT_RELU) EBS_ACT_CASE(EBS_ACT_GELU) EBS_ACT_CASE(EBS_ACT_GELU_TANH) EBS_ACT_CASE(EBS_ACT_SILU)
#undef EBS_ACT_CASE
            default: break;
        }
        if (e.o.residual) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float t[N];
                unpack<T>(a.residual[c], t);
#pragma unroll
                for (int i = 0; i < N; ++i) v[c * N + i] += t[i];
            }
        }
    }
    template <int R>
    static __device__ __forceinline__ void finish(const LinearOut<T>& e, const CUtensorMap* y, const CUtensorMap* z, RowRing<R>& ring, float (&v)[CW], const float* terms, int columns, int, int rows, int batch, int row0,
                                                  int col, int left, int row_term, const Ahead& a, bool exists, volatile int* holes) {
        uint8_t* to = ring.next();
        scale(e, v, terms, columns, col, left, row_term, to, ring.lane, row0 + ring.lane < rows, holes);
        if (e.o.z) {
            put_row<T>(to, ring.lane, v);
            ring.store(z, to, col, row0, batch, exists);
            to = ring.next();
        }
        activate(e, v, a);
        put_row<T>(to, ring.lane, v);
        ring.store(y, to, col, row0, batch, exists);
    }
};

// Rows of planes: a buffer for hi, one for lo.
template <>
struct RowOut<PlanesOut> {
    static constexpr bool HOLES = false;
    static constexpr int CW = 32;
    struct Ahead {};
    static __device__ __forceinline__ void begin(const PlanesOut&, float*, int, int, int, int) {}
    static __device__ __forceinline__ int row_term(const PlanesOut&, long long, bool) { return 0; }
    static __device__ __forceinline__ void ahead(const PlanesOut&, int, long long, int, int, Ahead&) {}
    template <int R>
    static __device__ __forceinline__ void matrix(__half* to, const PlanesOut& e, const CUtensorMap* y, RowRing<R>& ring, const float (&v)[CW], float factor, float on_diag, int mirror, int rows,
                                                  int batch, int row0, int col, int left, bool exists) {
        const int lane = ring.lane, diagonal = row0 + lane - col;             // the column of this row that lies on the diagonal
        __half* image = to + batch * e.batch + (long long)col * e.ld + row0 + lane;
        uint8_t* buffer = ring.next();
        uint32_t lo[CW / 2];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            uint32_t hi[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = c * 8 + 2 * i;
                split_pair(v[at] * factor + (at == diagonal ? on_diag : 0.0f), v[at + 1] * factor + (at + 1 == diagonal ? on_diag : 0.0f), hi[i], lo[c * 4 + i]);
            }
            *row_chunk(buffer, lane, c) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            if (mirror && row0 + lane < rows) {                   // the image across the diagonal: 32 lanes write 64 bytes of a row
                const __half *h = reinterpret_cast<const __half*>(hi), *l = reinterpret_cast<const __half*>(lo + c * 4);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c * 8 + i < left) {
                        image[(c * 8 + i) * e.ld] = h[i];
                        image[(c * 8 + i) * e.ld + e.plane] = l[i];
                    }
            }
        }
        ring.store(y, buffer, col, row0, 2 * batch, exists);
        buffer = ring.next();
#pragma unroll
        for (int c = 0; c < 4; ++c) *row_chunk(buffer, lane, c) = make_uint4(lo[4 * c], lo[4 * c + 1], lo[4 * c + 2], lo[4 * c + 3]);
        ring.store(y, buffer, col, row0, 2 * batch + 1, exists);
    }
    template <int R>
    static __device__ __forceinline__ void finish(const PlanesOut& e, const CUtensorMap* y, const CUtensorMap* y2, RowRing<R>& ring, float (&v)[CW], const float*, int, int mirror, int rows, int batch,
                                                  int row0, int col, int left, int, const Ahead&, bool exists, volatile int*) {
        matrix(e.y, e, y, ring, v, e.alpha, e.diag, mirror, rows, batch, row0, col, left, exists);
        if (e.y2) matrix(e.y2, e, y2, ring, v, e.alpha2, e.diag2, mirror, rows, batch, row0, col, left, exists);
    }
};

template <typename T>
struct RowOut<TypedFinal<T>> {
    static constexpr bool HOLES = false;
    static constexpr int CW = 64 / sizeof(T);
    struct Ahead {};
    static __device__ __forceinline__ void begin(const TypedFinal<T>&, float*, int, int, int, int) {}
    static __device__ __forceinline__ int row_term(const TypedFinal<T>&, long long, bool) { return 0; }
    static __device__ __forceinline__ void ahead(const TypedFinal<T>&, int, long long, int, int, Ahead&) {}
    template <int R>
    static __device__ __forceinline__ void finish(const TypedFinal<T>& e, const CUtensorMap* y, const CUtensorMap*, RowRing<R>& ring, float (&v)[CW], const float*, int, int, int rows, int batch, int row0, int col,
                                                  int, int, const Ahead&, bool exists, volatile int*) {
#pragma unroll
        for (int i = 0; i < CW; ++i) v[i] *= e.o.alpha;
        uint8_t* to = ring.next();
        put_row<T>(to, ring.lane, v);
        ring.store(y, to, col, row0, batch, exists);
    }
};

template <>
struct RowOut<PartialOut> {
    static constexpr bool HOLES = false;
    static constexpr int CW = 16;
    struct Ahead {};
    static __device__ __forceinline__ void begin(const PartialOut&, float*, int, int, int, int) {}
    static __device__ __forceinline__ int row_term(const PartialOut&, long long, bool) { return 0; }
    static __device__ __forceinline__ void ahead(const PartialOut&, int, long long, int, int, Ahead&) {}
    template <int R>
    static __device__ __forceinline__ void finish(const PartialOut&, const CUtensorMap* y, const CUtensorMap*, RowRing<R>& ring, float (&v)[CW], const float*, int, int, int, int slice, int row0, int col, int,
                                                  int, const Ahead&, bool exists, volatile int*) {
        uint8_t* to = ring.next();
        put_row<float>(to, ring.lane, v);
        ring.store(y, to, col, row0, slice, exists);
    }
};

constexpr int PAIR_EPI_WARPS = 16;                               // a quarter of the columns each four: fewer leave the memory and barrier latencies of small reductions in the open
constexpr int PAIR_THREADS = (PAIR_EPI_WARPS + 4) * 32;          // and a warpgroup that fetches and issues (two of its warps idle)
constexpr int PAIR_A = 128 * GEMM_ROW_BYTES;                     // a block's 128 rows of A: 64 elements each
template <int TN> __host__ __device__ constexpr int pair_b() { return TN / 2 * GEMM_ROW_BYTES; }             // and its half of B
template <int PL, int TN> __host__ __device__ constexpr int pair_stage_bytes() { return PL * (PAIR_A + pair_b<TN>()); }
template <int PL, int TN> __host__ __device__ constexpr int pair_stages() { return 192 * 1024 / pair_stage_bytes<PL, TN>(); }      // 6 or 8, 3 or 4
// Per warp, behind the stages: a ring of buffers of 64-byte rows of results on their way out.
constexpr int PAIR_RING = 1;
constexpr int PAIR_TERMS = 4 * 2 * 64 * 4;                       // per column quarter: bias and factor of up to 64 columns
constexpr int PAIR_BARRIERS = 256;
template <int PL, int TN> __host__ __device__ constexpr int pair_smem_bytes() {
    return pair_stages<PL, TN>() * pair_stage_bytes<PL, TN>() + PAIR_EPI_WARPS * PAIR_RING * PAIR_BUFFER + PAIR_TERMS + PAIR_BARRIERS;
}

// Tiles in bands of eight tile rows, column by column within a band: the tiles under way at a time share few rows and columns.
// A symmetric result: only the tiles of the 256 x 256 squares on and below the diagonal, row by row.
// Parts of the reduction of one tile follow one another.
template <int TN>
__host__ __device__ __forceinline__ int symmetric_tiles(int tiles_m, int tiles_n) {
    constexpr int Q = 256 / TN;
    return tiles_m * (tiles_m + 1) / 2 * Q - (tiles_m * Q - tiles_n);      // (the last square's second half need not exist)
}
template <int TN>
__device__ __forceinline__ void pair_tile(int t, int tiles_m, int tiles_n, int symmetric, int split, int blocks, int& batch, int& tm, int& tn, int& part, int& kb0, int& kb1) {
    part = 0;
    if (split > 1) {
        part = t % split;
        t /= split;
    }
    kb0 = (int)((long long)blocks * part / split);
    kb1 = (int)((long long)blocks * (part + 1) / split);
    const int per = symmetric ? symmetric_tiles<TN>(tiles_m, tiles_n) : tiles_m * tiles_n;
    batch = t / per;
    t -= batch * per;
    if (symmetric) {
        constexpr int Q = 256 / TN;
        const int square = t / Q;
        tm = (int)((sqrtf(8.0f * square + 1.0f) - 1.0f) * 0.5f);
        while (tm * (tm + 1) / 2 > square) --tm;
        while ((tm + 1) * (tm + 2) / 2 <= square) ++tm;
        tn = (square - tm * (tm + 1) / 2) * Q + t % Q;
        return;
    }
    const int band = t / (8 * tiles_n), first = band * 8, height = tiles_m - first < 8 ? tiles_m - first : 8;
    t -= band * 8 * tiles_n;
    tn = t / height;
    tm = first + t - tn * height;
}

// CHUNKS: sums leave tensor memory every g.chunk stages and go on in registers.
template <class EPI, int PL, int TN, bool CHUNKS>
__global__ void __launch_bounds__(PAIR_THREADS, 1) gemm_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                           const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_z, const TileArgs g,
                                                           const EPI epi) {
    extern __shared__ __align__(1024) uint8_t tiles[];            // (nothing static: the stages take all but a few hundred bytes)
    constexpr int S = pair_stages<PL, TN>(), STAGE = pair_stage_bytes<PL, TN>(), R = PAIR_RING;
    constexpr int B_HALF = pair_b<TN>(), CQ = TN / 4;             // CQ: columns of a warp
    uint8_t* behind = tiles + S * STAGE;
    float* all_terms = reinterpret_cast<float*>(behind + PAIR_EPI_WARPS * R * PAIR_BUFFER);
    uint64_t* full = reinterpret_cast<uint64_t*>(behind + PAIR_EPI_WARPS * R * PAIR_BUFFER + PAIR_TERMS);
    uint64_t *empty = full + S, *acc_full = empty + S, *acc_empty = acc_full + 2, *terms_there = acc_empty + 2, *terms_read = terms_there + 4;
    uint32_t& tmem_slot = *reinterpret_cast<uint32_t*>(terms_read + 4);
    volatile int& abort_flag = *reinterpret_cast<volatile int*>(terms_read + 5);
    volatile int* holes = &abort_flag + 1;                        // results were left to finish_infinite
    static_assert((2 * S + 12 + 2) * 8 <= PAIR_BARRIERS, "barriers");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)(blockIdx.x & 1), pairs = (int)(gridDim.x >> 1);
    const int blocks = (g.red + GEMM_BK - 1) / GEMM_BK, chunk = CHUNKS ? g.chunk : blocks;
    const int tiles_m = (g.out_rows + 255) / 256, tiles_n = (g.out_cols + TN - 1) / TN, count = (g.symmetric ? symmetric_tiles<TN>(tiles_m, tiles_n) : tiles_m * tiles_n) * g.batch * g.split;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 2 * PAIR_EPI_WARPS); }
        for (int q = 0; q < 4; ++q) { mbar_init(&terms_there[q], 4); mbar_init(&terms_read[q], 4); }
        abort_flag = *holes = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == PAIR_EPI_WARPS + 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_slot)), "r"(2u * TN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    __syncthreads();
    cluster_sync_all();                                           // the partner's barriers are ready too
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    const uint32_t tmem = uni(tmem_slot);
    let_next_kernel_start();
    wait_for_previous_kernel();

    // Sums taken in chunks are 64 a thread.  Registers are dealt anew among the warpgroups: 4 * 128 * 104 + 128 * 56 = 60416 of the
    // 640 * 96 = 61440 the block was launched with.  (Each at the head of its warpgroup's own code: the compiler counts registers by
    // what it can reach.)
    if (warp >= PAIR_EPI_WARPS) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 56;\n");
      if (warp == PAIR_EPI_WARPS) {
        const bool leader = elect_one();
        int i = 0;                                                // stages filled so far
        bool ok = true;
        for (int t = (int)(blockIdx.x >> 1); t < count && ok; t += pairs) {
            int batch, tm, tn, part, kb0, kb1;
            pair_tile<TN>(t, tiles_m, tiles_n, g.symmetric, g.split, blocks, batch, tm, tn, part, kb0, kb1);
            const int a0 = tm * 256 + rank * 128, b0 = tn * TN + rank * (TN / 2);
            for (int kb = kb0; kb < kb1; ++kb, ++i) {
                const int s = i % S, k = kb * GEMM_BK;
                ok = mbar_wait_warp(&empty[s], ((i / S) & 1) ^ 1, &abort_flag, g.wait_limit);
                if (!ok) break;
                if (leader) {
                    const uint32_t base = smem_u32(tiles) + s * STAGE, bar = cluster_addr(&full[s], 0);
                    if (rank == 0) mbar_expect_tx(&full[s], 2 * STAGE);
#pragma unroll
                    for (int p = 0; p < PL; ++p) {
                        const uint32_t at = base + p * PAIR_A, bt = base + PL * PAIR_A + p * B_HALF;
                        const int z = batch * PL + p;
                        if (!g.a_mn) tma_load_3d_pair(at, &map_a, k, a0, z, bar);
                        else { tma_load_3d_pair(at, &map_a, a0, k, z, bar); tma_load_3d_pair(at + 8192, &map_a, a0 + 64, k, z, bar); }
                        if (!g.b_mn) tma_load_3d_pair(bt, &map_b, k, b0, z, bar);
                        else
#pragma unroll
                            for (int h = 0; h < TN / 128; ++h) tma_load_3d_pair(bt + h * 8192, &map_b, b0 + h * 64, k, z, bar);
                    }
                }
                __syncwarp();
            }
        }
      } else if (warp == PAIR_EPI_WARPS + 1 && rank == 0) {
            const uint32_t leader = elect_one() ? 1u : 0u;
            const uint32_t idesc = gemm_idesc(256, TN, g.bf16, g.a_mn, g.b_mn);
            const uint32_t a_step = g.a_mn ? 2048 >> 4 : 32 >> 4, b_step = g.b_mn ? 2048 >> 4 : 32 >> 4;
            int i = 0, c = 0;                                     // stages and accumulators used so far
            bool ok = true;
            for (int t = (int)(blockIdx.x >> 1); t < count && ok; t += pairs) {
                int batch, tm, tn, part, kb0, kb1;
                pair_tile<TN>(t, tiles_m, tiles_n, g.symmetric, g.split, blocks, batch, tm, tn, part, kb0, kb1);
                for (int kb = kb0; kb < kb1 && ok; ++kb, ++i) {
                    const int s = i % S, in_chunk = (kb - kb0) % chunk;
                    if (in_chunk == 0 && c >= 2) ok = mbar_wait_cluster_warp(&acc_empty[c & 1], ((c >> 1) & 1) ^ 1, &abort_flag, g.wait_limit);
                    ok = ok && mbar_wait_warp(&full[s], (i / S) & 1, &abort_flag, g.wait_limit);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                    const bool last = in_chunk == chunk - 1 || kb == kb1 - 1;
                    if ((g.test_flags & 1) == 0) {                // (give-up test: nothing is ever issued)
                        const uint32_t d = tmem + (uint32_t)((c & 1) * TN), base = smem_u32(tiles) + s * STAGE;
                        const uint32_t ah = tile_desc_lo(base, g.a_mn), bh = tile_desc_lo(base + PL * PAIR_A, g.b_mn);
                        if (PL == 2)                              // (the small products first: each MMA truncates at the size of what is there)
#pragma unroll
                            for (int k = 0; k < GEMM_BK / 16; ++k) {
                                const uint32_t a = ah + k * a_step, b = bh + k * b_step;
                                umma_f16_pair(leader, d, a, b + (B_HALF >> 4), idesc, (in_chunk | k) != 0);
                                umma_f16_pair(leader, d, a + (PAIR_A >> 4), b, idesc, 1u);
                            }
#pragma unroll
                        for (int k = 0; k < GEMM_BK / 16; ++k) umma_f16_pair(leader, d, ah + k * a_step, bh + k * b_step, idesc, PL == 2 || (in_chunk | k) != 0);
                        umma_commit_both(leader, cluster_addr(&empty[s], 0), cluster_addr(&empty[s], 1));
                        if (last) umma_commit_both(leader, cluster_addr(&acc_full[c & 1], 0), cluster_addr(&acc_full[c & 1], 1));
                    }
                    c += last;
                }
            }
      }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;\n");
        using Rows = RowOut<EPI>;
        constexpr bool ELEMENTS = !std::is_same<EPI, PlanesOut>::value && !std::is_same<EPI, PartialOut>::value;      // (those always have whole rows)
        constexpr int CW = Rows::CW;
        RowRing<R> ring{behind + warp * R * PAIR_BUFFER, lane};
        float* terms = all_terms + (warp >> 2) * 2 * CQ;             // shared by the four warps of a column quarter
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (warp >> 2) * CQ;
        int c = 0, done = 0;                                      // accumulators and tiles so far
        bool ok = true;
        for (int t = (int)(blockIdx.x >> 1); t < count && ok; t += pairs, ++done) {
            int batch, tm, tn, part, kb0, kb1;
            pair_tile<TN>(t, tiles_m, tiles_n, g.symmetric, g.split, blocks, batch, tm, tn, part, kb0, kb1);
            const int row0 = tm * 256 + rank * 128 + (warp & 3) * 32, col0 = tn * TN + (warp >> 2) * CQ;
            const int slice = part * g.batch + batch;             // (parts: a matrix each)
            // rows by TMA
            int row_term = 0;
            if (g.packs) {
                const int at = (warp & 3) * (CQ / 4) + lane;
                // (mbarriers, not a block barrier: a warp that gave up is not waited for without end)
                if (done > 0) ok = mbar_wait_bounded(&terms_read[warp >> 2], (done - 1) & 1, &abort_flag, g.wait_limit);
                if (!ok) break;
                if (lane < CQ / 4) Rows::begin(epi, terms, CQ, at, col0 + at, g.out_cols);
                row_term = Rows::row_term(epi, row0 + lane, row0 + lane < g.out_rows);
                __syncwarp();
                if (lane == 0) mbar_arrive(&terms_there[warp >> 2]);
                ok = mbar_wait_bounded(&terms_there[warp >> 2], done & 1, &abort_flag, g.wait_limit);
                if (!ok) break;
            }
            typename Rows::Ahead row_ahead;
            auto rows_ahead = [&](int column) {
                if (row0 + lane < g.out_rows) Rows::ahead(epi, slice, row0 + lane, col0 + column, g.out_cols - col0 - column, row_ahead);
            };
            auto rows_out = [&](int column, float (&v)[CW]) {
                const int col = col0 + column;
                Rows::finish(epi, &map_y, &map_z, ring, v, terms + column, CQ, g.symmetric && tn / (256 / TN) != tm, g.out_rows, slice, row0, col, g.out_cols - col, row_term, row_ahead,
                             col < g.out_cols && row0 < g.out_rows, holes);
            };
            // Outputs whose rows start anywhere, 16 columns at a time: through the warp's buffer, then two rows an access, neighbouring lanes
            // at neighbouring elements, eight accesses' loads under way.
            auto elements_out = [&](int column, const float (&f)[16]) {
                if constexpr (ELEMENTS) {
                    __syncwarp();
#pragma unroll
                    for (int q = 0; q < 4; ++q) *reinterpret_cast<float4*>(row_chunk(ring.base, lane, q)) = make_float4(f[4 * q], f[4 * q + 1], f[4 * q + 2], f[4 * q + 3]);
                    __syncwarp();
                    const int cc = lane & 15, col = col0 + column + cc;
                    if (col < g.out_cols) {
                        typename EPI::Column terms_of;
                        epi.column(col, terms_of);
#pragma unroll 1
                        for (int r0 = lane >> 4; r0 < 32; r0 += 16) {
                            typename EPI::Place place[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (row0 + r0 + 2 * i < g.out_rows) epi.place(row0 + r0 + 2 * i, col, place[i]);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const int r = r0 + 2 * i;
                                const float v = reinterpret_cast<const float*>(row_chunk(ring.base, r, cc >> 2))[cc & 3];
                                if (row0 + r < g.out_rows && epi.one(batch, row0 + r, col, v, terms_of, place[i])) *holes = 1;
                            }
                        }
                    }
                }
            };
            if constexpr (CHUNKS) {
                float acc[CQ];
#pragma unroll
                for (int j = 0; j < CQ; ++j) acc[j] = 0.0f;
                for (int kb = kb0; kb < kb1 && ok; kb += chunk, ++c) {
                    ok = mbar_wait_bounded(&acc_full[c & 1], (c >> 1) & 1, &abort_flag, g.wait_limit);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#pragma unroll
                    for (int j = 0; j < CQ; j += 32) {
                        uint32_t v[32];
                        tmem_ld32_issue(lanes + (c & 1) * TN + j, v);
                        tmem_ld32_wait(v);
#pragma unroll
                        for (int e = 0; e < 32; ++e) acc[j + e] += __uint_as_float(v[e]);
                    }
                    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
                    if (lane == 0) mbar_arrive_cluster(cluster_addr(&acc_empty[c & 1], 0));
                }
                if (!ok) break;
                if (g.packs) {
#pragma unroll
                    for (int j = 0; j < CQ; j += CW) {
                        rows_ahead(j);
                        float v[CW];
#pragma unroll
                        for (int e = 0; e < CW; ++e) v[e] = acc[j + e];
                        rows_out(j, v);
                    }
                } else {
#pragma unroll 1
                    for (int j = 0; j < CQ; j += 16) {            // (registers have no index: one copy of the moves a position)
                        float v[16];
#pragma unroll
                        for (int q = 0; q < CQ; q += 16)
                            if (q == j) {
#pragma unroll
                                for (int e = 0; e < 16; ++e) v[e] = acc[q + e];
                            }
                        elements_out(j, v);
                    }
                }
            } else {
                if (g.packs) rows_ahead(0);
                ok = mbar_wait_bounded(&acc_full[c & 1], (c >> 1) & 1, &abort_flag, g.wait_limit);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#pragma unroll 1
                for (int j = 0; j < CQ; j += 32) {
                    uint32_t raw[32];
                    tmem_ld32_issue(lanes + (c & 1) * TN + j, raw);
                    if (g.packs && j > 0) rows_ahead(j);
                    tmem_ld32_wait(raw);
                    if (j == CQ - 32) {
                        asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
                        if (lane == 0) mbar_arrive_cluster(cluster_addr(&acc_empty[c & 1], 0));
                    }
#pragma unroll
                    for (int h = 0; h < 32; h += CW) {
                        if (!g.packs) break;
                        float v[CW];
#pragma unroll
                        for (int e = 0; e < CW; ++e) v[e] = __uint_as_float(raw[h + e]);
                        rows_out(j + h, v);
                    }
                    if (!g.packs)
#pragma unroll
                        for (int h = 0; h < 32; h += 16) {
                            float v[16];
#pragma unroll
                            for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(raw[h + e]);
                            elements_out(j + h, v);
                        }
                }
                ++c;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&terms_read[warp >> 2]);
        }
        if (lane == 0) tma_store_wait_all();
    }
    __syncthreads();
    if (abort_flag) {
        giveup_drain();
        if (threadIdx.x == 0) atomicAdd(&g_gemm_pair_timeouts, 1ull);
    }
    if constexpr (RowOut<EPI>::HOLES) {                           // (behind all waits, by the warps that have the registers)
        if (*holes && !abort_flag && warp < PAIR_EPI_WARPS)
            for (int t = (int)(blockIdx.x >> 1); t < count; t += pairs) {
                int batch, tm, tn, part, kb0, kb1;
                pair_tile<TN>(t, tiles_m, tiles_n, g.symmetric, g.split, blocks, batch, tm, tn, part, kb0, kb1);
                const int row0 = tm * 256 + rank * 128, col0 = tn * TN;
                finish_infinite<PAIR_EPI_WARPS, 1>(epi.o, row0, min(128, g.out_rows - row0), col0, min(TN, g.out_cols - col0), reinterpret_cast<unsigned*>(behind));
            }
    }
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    cluster_sync_all();                                           // no block leaves while the other's MMAs or arrivals reach it
    if (warp == PAIR_EPI_WARPS + 1)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(2u * TN) : "memory");
}

unsigned long long gemm_pair_timeouts() {
    unsigned long long n = 0;
    return cudaMemcpyFromSymbol(&n, g_gemm_pair_timeouts, sizeof(n)) == cudaSuccess ? n : 0;
}

template <typename T>
static bool result_maps(const LinearOut<T>& e, const GemmShape& s, CUtensorMap* y, CUtensorMap* z) {
    const auto whole = [](const void* p, long long ld) { return !p || (((uintptr_t)p & 15) == 0 && (ld * sizeof(T)) % 16 == 0); };
    return whole(e.o.residual, e.o.ldr) && result_map<T>(e.o.y, s.rows, s.cols, e.o.ldy, 1, 0, y) && result_map<T>(e.o.z, s.rows, s.cols, e.o.ldz, 1, 0, z);
}
static bool result_maps(const PlanesOut& e, const GemmShape& s, CUtensorMap* y, CUtensorMap* y2) {
    return result_map<__half>(e.y, s.rows, s.cols, e.ld, 2LL * s.batch, e.plane, y, true) && result_map<__half>(e.y2, s.rows, s.cols, e.ld, 2LL * s.batch, e.plane, y2, true);
}
template <typename T>
static bool result_maps(const TypedFinal<T>& e, const GemmShape& s, CUtensorMap* y, CUtensorMap*) {
    return result_map<T>(e.o.y, s.rows, s.cols, e.o.ld, s.batch, e.o.batch, y);
}
static bool result_maps(const PartialOut& e, const GemmShape& s, CUtensorMap* y, CUtensorMap*) {
    return result_map<float>(e.y, s.rows, s.cols, e.ld, (long long)s.batch * e.parts, e.batch, y, true);
}

template <class EPI, int PL, int TN, bool CHUNKS>
static int launch_pair(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const EPI& epi, bool bf16, int split, cudaStream_t st) {
    const bool symmetric = s.symmetric && std::is_same<EPI, PlanesOut>::value;
    TileArgs g = {};
    g.red = s.red;
    g.out_rows = s.rows;
    g.out_cols = s.cols;
    g.batch = s.batch;
    g.split = split;
    g.symmetric = symmetric;
    g.a_mn = A.mn_major;
    g.b_mn = B.mn_major;
    g.bf16 = bf16;
    g.chunk = PL == 2 ? s.chunk : GEMM_LONG;
    g.wait_limit = device_wait_limit();
    g.test_flags = device_test_flags();
    const long long side = (s.rows + 255) / 256, across = (s.cols + TN - 1) / TN, tiles = (symmetric ? side * (side + 1) / 2 * (256 / TN) - (side * (256 / TN) - across) : side * across) * s.batch * split;
    if (tiles >= (1LL << 30)) return EBS_ERR_OVERFLOW;
    CUtensorMap a, b, y{}, z{};
    if (!gemm_operand_map(A, s.rows, s.red, s.batch, 128, bf16, &a) || !gemm_operand_map(B, s.cols, s.red, s.batch, TN / 2, bf16, &b)) return EBS_ERR_CUDA;
    g.packs = result_maps(epi, s, &y, &z);
    if (symmetric && !g.packs) return EBS_ERR_CUDA;               // (kept planes always have whole rows)
    auto kern = gemm_pair_kernel<EPI, PL, TN, CHUNKS>;
    constexpr int bytes = pair_smem_bytes<PL, TN>();
    static_assert(bytes <= 227 * 1024, "shared memory of a block");
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        if (check_cuda(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes))) return EBS_ERR_CUDA;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    const int pairs = gemm_sm_count() / 2;
    return launch_chained(kern, dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs))), PAIR_THREADS, (size_t)bytes, st, 2, a, b, y, z, g, epi);
}

// Adds the parts of a product split over its reduction, in their order, and finishes the results: a thread a pack.  Where there may be holes a block
// takes 32 x 32 results at a time, what finish_infinite does, and its registers (a called function's count too) are bounded so that four blocks run.
template <class EPI>
__global__ void __launch_bounds__(256, EPI::HOLES ? 4 : 0) reduce_parts_kernel(const PartialOut in, const int parts, const int rows, const int cols, const int packs, const EPI epi) {
    constexpr int N = EPI::N;
    let_next_kernel_start();
    wait_for_previous_kernel();
    const int per_row = EPI::HOLES ? (cols + 31) / 32 : (cols + N - 1) / N, batch = (int)blockIdx.y;      // squares, or packs
    const long long items = EPI::HOLES ? (long long)per_row * ((rows + 31) / 32) * 256 : (long long)per_row * rows;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < items; i += gridDim.x * 256LL) {
        int row, col;
        if constexpr (EPI::HOLES) {
            static_assert(N == 4, "eight packs of 32 columns");
            const int square = (int)(i >> 8);
            row = square / per_row * 32 + (int)threadIdx.x / 8;
            col = square % per_row * 32 + (int)threadIdx.x % 8 * N;
        } else {
            row = (int)(i / per_row);
            col = (int)(i - (long long)row * per_row) * N;
        }
        bool holes = false;
        if (!EPI::HOLES || (row < rows && col < cols)) {
            const int left = cols - col;
            const bool vec = packs && left >= N;
            typename EPI::Columns columns;
            typename EPI::Ahead ahead;
            epi.columns(col, left, vec, columns);
            epi.ahead(batch, row, col, left, vec, ahead);
            float v[N];
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] = 0.0f;
            const float* p = in.y + batch * in.batch + row * in.ld + col;
#pragma unroll 4
            for (int q = 0; q < parts; ++q) {
#pragma unroll
                for (int e = 0; e < N; e += 4) {
                    const float4 t = *reinterpret_cast<const float4*>(p + q * in.part + e);
                    v[e] += t.x; v[e + 1] += t.y; v[e + 2] += t.z; v[e + 3] += t.w;
                }
            }
            holes = epi.pack(batch, row, col, left, vec, v, columns, ahead);
        }
        if constexpr (EPI::HOLES) {
            __shared__ unsigned masks[64];
            const int row0 = row & ~31, col0 = col & ~31;
            if (__syncthreads_or(holes)) finish_infinite<8, 0>(epi.o, row0, min(32, rows - row0), col0, min(32, cols - col0), masks);
        }
    }
}
// (16-bit operands, and parts: tiles of 256 columns)
template <class EPI, int PL>
static int launch_pair_form(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const EPI& epi, bool bf16, int tn, int split, cudaStream_t st) {
    if constexpr (PL == 2) {
        if constexpr (!std::is_same<EPI, PartialOut>::value)
            if (tn == 128) return launch_pair<EPI, PL, 128, true>(A, B, s, epi, bf16, split, st);
        return launch_pair<EPI, PL, 256, true>(A, B, s, epi, bf16, split, st);
    } else {
        const int stages = ((s.red + GEMM_BK - 1) / GEMM_BK + split - 1) / split;
        return stages > GEMM_LONG ? launch_pair<EPI, PL, 256, true>(A, B, s, epi, bf16, split, st) : launch_pair<EPI, PL, 256, false>(A, B, s, epi, bf16, split, st);
    }
}
template <class EPI, int PL>
static int launch_pair_or_parts(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const EPI& epi, bool bf16, bool packs, const GemmRoute& route, float* scratch, cudaStream_t st) {
    if (route.split == 1) return launch_pair_form<EPI, PL>(A, B, s, epi, bf16, route.tn, 1, st);
    PartialOut p;
    p.y = scratch;
    p.ld = (s.cols + 7) & ~7LL;
    p.batch = p.ld * s.rows;
    p.part = p.batch * s.batch;
    p.parts = route.split;
    const int rc = launch_pair_form<PartialOut, PL>(A, B, s, p, bf16, 256, route.split, st);
    if (rc) return rc;
    const long long items = (long long)((s.cols + EPI::N - 1) / EPI::N) * s.rows, blocks = EPI::HOLES ? (s.rows + 31LL) / 32 * ((s.cols + 31) / 32) : (items + 255) / 256;
    return launch_chained(reduce_parts_kernel<EPI>, dim3((unsigned)(blocks < 4096 ? blocks : 4096), s.batch), 256, 0, st, 1, p, route.split, s.rows, s.cols, (int)packs, epi);
}

int launch_gemm_pair(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const GemmRoute& r, float* scratch, const GemmOut& out, int dtype, cudaStream_t st) {
    const bool packs = packs_ok(out, element_size(dtype));
    if (dtype == EBS_F32) return launch_pair_or_parts<LinearOut<float>, 2>(A, B, s, {out}, false, packs, r, scratch, st);
    if (dtype == EBS_F16) return launch_pair_or_parts<LinearOut<__half>, 1>(A, B, s, {out}, false, packs, r, scratch, st);
    return launch_pair_or_parts<LinearOut<__nv_bfloat16>, 1>(A, B, s, {out}, true, packs, r, scratch, st);
}
int launch_gemm_pair(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const GemmRoute& r, float* scratch, const PlanesOut& out, cudaStream_t st) {
    return launch_pair_or_parts<PlanesOut, 2>(A, B, s, out, false, true, r, scratch, st);
}
int launch_gemm_pair(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const GemmRoute& r, float* scratch, const FinalOut& out, int dtype, cudaStream_t st) {
    const bool packs = out.ld * (long long)element_size(dtype) % 16 == 0 && (out.batch * (long long)element_size(dtype)) % 16 == 0;
    if (dtype == EBS_F32) return launch_pair_or_parts<TypedFinal<float>, 2>(A, B, s, {out}, false, packs, r, scratch, st);
    if (dtype == EBS_F16) return launch_pair_or_parts<TypedFinal<__half>, 2>(A, B, s, {out}, false, packs, r, scratch, st);
    return launch_pair_or_parts<TypedFinal<__nv_bfloat16>, 2>(A, B, s, {out}, false, packs, r, scratch, st);
}

// The kernel for a product, from its sizes alone (and so the same for the workspace's count and for the call).
GemmRoute gemm_route(const GemmShape& s, int planes) {
    GemmRoute r;
    const long long side = (s.rows + 255) / 256, wide = (s.symmetric ? side * (side + 1) / 2 : side * ((s.cols + 255) / 256)) * s.batch;
    const long long narrow = side * ((s.cols + 127) / 128) * s.batch;
    const int blocks = (s.red + GEMM_BK - 1) / GEMM_BK;
    // (a symmetric result by half pays from fewer tiles on, where the tile kernel's whole one is more than a round)
    const long long whole = (long long)((s.rows + 127) / 128) * ((s.cols + 127) / 128) * s.batch;
    r.pair = s.rows > 128 && s.cols > 128 && (wide >= 32 || (s.symmetric && wide >= 20 && whole > 148));
    if (r.pair) {
        // Split products on tiles of 128 columns where 256 leave pairs idle (us with 256 and 128: 512 x 4608 over 512 23.3 and 13.9, 12544 x 256 over
        // 1152 33.5 and 30.2, 2048 x 2048 over 2048 48.0 and 43.4) or the reduction is short and the last round fuller (12544 x 1152 over 256
        // 37.1 and 33.2; 4096 x 4096 over 1024 78.4 and 81.4).  16-bit operands never: half the work per byte fetched (8192 x 4096 over 512 36.7
        // and 55.4).
        const long long w = (wide + 73) / 74 * 2, n = (narrow + 73) / 74;
        // Symmetric ones where 256 leave half the pairs idle (an orthogonalisation of 2048 x 2048 739 and 480 us; three rounds of 128 instead of two of
        // 256 do not pay: 3300 x 3300 2348 and 2467 us).
        if (planes == 2 && s.symmetric && wide <= 37) r.tn = 128;
        if (planes == 2 && !s.symmetric && (wide <= 74 || (blocks <= 8 && n < w))) r.tn = 128;
    } else if (s.rows > 128 && s.cols > 128 && blocks >= 64) {
        const long long all = side * ((s.cols + 255) / 256) * s.batch;
        r.split = (int)(74 / all);
        if (r.split > blocks / 8) r.split = blocks / 8;
        r.pair = r.split > 1;
        if (r.split < 1) r.split = 1;
    }
    if (r.pair && r.split > 1) r.scratch = (size_t)r.split * s.batch * s.rows * ((s.cols + 7) & ~7LL) * 4;
    return r;
}

}  // namespace ebs
