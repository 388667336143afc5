// Persistent kernel of the large real-valued products: a pair of thread blocks on two SMs works on 256 x 256 results at a time.
//
// The MMAs are M = 256, N = 256 over both blocks' shared and tensor memory (cta_group::2): each block fetches its 128 rows of A and half
// of the 256 columns of B, so that an operand element crosses shared memory half as often as in a single block's 128 x 128 tile
// (that one reads 128 bytes a clock, all there are).  Warp 8 of each block fetches by TMA, warp 9 of the even block issues, warps 0-7
// of both take the sums of their 128 rows out of tensor memory (lanes 32 (w % 4), columns 128 (w / 4)) and write the results
// through a patch of shared memory, so that neighbouring lanes write neighbouring bytes.  Two accumulators of 256 columns: the
// MMAs of the next tile (split products: of the next GEMM_CHUNK stages, see gemm_tile.cu) run while one is taken out.
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
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, const void* src, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];\n" ::"l"(map), "r"(smem_u32(src)), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_store_commit() { asm volatile("cp.async.bulk.commit_group;\n" ::: "memory"); }
__device__ __forceinline__ void tma_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory"); }
__device__ __forceinline__ void tma_store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory"); }

// CW, BUFFERS; TERMS: fp32 values a column; begin: the columns' terms of a tile; ahead: what a row needs from memory; finish: the values
// into the buffer(s); planes: stores a buffer leads to.
template <class EPI> struct RowOut;

template <typename T>
struct RowOut<LinearOut<T>> {
    static constexpr int CW = 64 / sizeof(T), BUFFERS = sizeof(T) == 2 ? 2 : 1, TERMS = sizeof(T) == 2 ? 1 : 2, N = Pack<T>::N;
    struct Ahead { uint4 residual[4]; };
    // returns whether every column's exponent is an ordinary one
    static __device__ __forceinline__ bool begin(const LinearOut<T>& e, float* terms, int col0, int cols, int lane) {
        bool plain = true;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = i * 32 + lane, col = col0 + at;
            terms[at] = e.o.bias && col < cols ? to_f32(static_cast<const T*>(e.o.bias)[col]) : 0.0f;
            if (sizeof(T) == 4) {
                const int x = col < cols ? e.o.col_exp[col] : 0;
                plain = plain && abs(x) <= SCALE_PLAIN;
                terms[128 + at] = power_of_two(abs(x) <= SCALE_PLAIN ? x : 0) * e.o.alpha;
            }
        }
        return __all_sync(0xffffffffu, plain);
    }
    static __device__ __forceinline__ int row_term(const LinearOut<T>& e, long long row, bool exists) { return sizeof(T) == 4 && exists ? e.o.row_exp[row] : 0; }
    static __device__ __forceinline__ void ahead(const LinearOut<T>& e, int, long long row, int col, int left, Ahead& a) {
        if (!e.o.residual || left <= 0) return;
        const T* p = static_cast<const T*>(e.o.residual) + row * e.o.ldr + col;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (c * N < left) a.residual[c] = load_raw(p + c * N, left - c * N, left >= (c + 1) * N);
    }
    // first: the pre-activations (if wanted) in buffer 0 (T of two bytes: 1), then the result in buffer 0
    static __device__ __forceinline__ void scale(const LinearOut<T>& e, float (&v)[CW], const float* terms, long long row, int col, int left, int row_term, bool plain) {
        if constexpr (sizeof(T) == 4) {
            if (plain && abs(row_term) <= SCALE_PLAIN) {
                const float f = power_of_two(row_term);
#pragma unroll
                for (int i = 0; i < CW; i += 4) {
                    const float4 t = *reinterpret_cast<const float4*>(terms + 128 + i), b = *reinterpret_cast<const float4*>(terms + i);
                    v[i] = fmaf(v[i], f * t.x, b.x); v[i + 1] = fmaf(v[i + 1], f * t.y, b.y);
                    v[i + 2] = fmaf(v[i + 2], f * t.z, b.z); v[i + 3] = fmaf(v[i + 3], f * t.w, b.w);
                }
                return;
            }
            const GemmFp32& g = e.o.fp32;
#pragma unroll 1
            for (int i = 0; i < CW && i < left; ++i) {
                float s = 0.0f;
#pragma unroll
                for (int q = 0; q < CW; ++q) s = q == i ? v[q] : s;                      // (registers have no index)
                s = gemm_unscale(g.a + row * g.a_row, g.a_red, g.b + (col + i) * g.b_col, g.b_red, g.red, row_term, e.o.col_exp[col + i], s);
                s = fmaf(s, e.o.alpha, terms[i]);
#pragma unroll
                for (int q = 0; q < CW; ++q) v[q] = q == i ? s : v[q];
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
    // the buffer is free of earlier stores' reads when this is called
    static __device__ __forceinline__ void finish(const LinearOut<T>& e, const CUtensorMap* y, const CUtensorMap* z, uint8_t* buffer, float (&v)[CW], const float* terms, int, int batch, int row0,
                                                  int col, int left, int lane, int row_term, bool plain, const Ahead& a, bool store) {
        scale(e, v, terms, row0 + lane, col, left, row_term, plain);
        if (e.o.z) {
            uint8_t* to = buffer + (BUFFERS - 1) * PAIR_BUFFER;
            put_row<T>(to, lane, v);
            asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
            __syncwarp();
            if (lane == 0 && store) { tma_store_3d(z, to, col, row0, batch); tma_store_commit(); }
            if (BUFFERS == 1) {
                if (lane == 0) tma_store_wait_read();
                __syncwarp();
            }
        }
        activate(e, v, a);
        put_row<T>(buffer, lane, v);
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        __syncwarp();
        if (lane == 0 && store) { tma_store_3d(y, buffer, col, row0, batch); tma_store_commit(); }
    }
};

// Rows of planes: hi in buffer 0, lo in buffer 1.
template <>
struct RowOut<PlanesOut> {
    static constexpr int CW = 32, BUFFERS = 2, TERMS = 0;
    struct Ahead { uint4 hi[4], lo[4]; };
    static __device__ __forceinline__ bool begin(const PlanesOut&, float*, int, int, int) { return true; }
    static __device__ __forceinline__ int row_term(const PlanesOut&, long long, bool) { return 0; }
    static __device__ __forceinline__ void ahead(const PlanesOut& e, int batch, long long row, int col, int left, Ahead& a) {
        if (!e.c) return;
        const __half* p = e.c + batch * e.c_batch + row * e.c_ld + col;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (c * 8 < left) {
                a.hi[c] = *reinterpret_cast<const uint4*>(p + c * 8);
                a.lo[c] = *reinterpret_cast<const uint4*>(p + e.c_plane + c * 8);
            }
    }
    static __device__ __forceinline__ void finish(const PlanesOut& e, const CUtensorMap* y, const CUtensorMap*, uint8_t* buffer, float (&v)[CW], const float*, int mirror, int batch, int row0, int col,
                                                  int left, int lane, int, bool, const Ahead& a, bool store) {
        __half* image = e.y + batch * e.batch + (long long)col * e.ld + row0 + lane;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            __align__(16) __half hi[8], lo[8];
            float ch[8], cl[8];
            if (e.c) { unpack<__half>(a.hi[c], ch); unpack<__half>(a.lo[c], cl); }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float t = v[c * 8 + i] * e.alpha;
                if (e.c) t = fmaf(e.beta, ch[i] + cl[i], t);
                hi[i] = __float2half_rn(t);
                lo[i] = __float2half_rn(t - __half2float(hi[i]));
            }
            *row_chunk(buffer, lane, c) = *reinterpret_cast<const uint4*>(hi);
            *row_chunk(buffer + PAIR_BUFFER, lane, c) = *reinterpret_cast<const uint4*>(lo);
            if (mirror && row0 + lane < mirror) {                 // the image across the diagonal: 32 lanes write 64 bytes of a row
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c * 8 + i < left) {
                        image[(c * 8 + i) * e.ld] = hi[i];
                        image[(c * 8 + i) * e.ld + e.plane] = lo[i];
                    }
            }
        }
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        __syncwarp();
        if (lane == 0 && store) {
            tma_store_3d(y, buffer, col, row0, 2 * batch);
            tma_store_3d(y, buffer + PAIR_BUFFER, col, row0, 2 * batch + 1);
            tma_store_commit();
        }
    }
};

template <typename T>
struct RowOut<TypedFinal<T>> {
    static constexpr int CW = 64 / sizeof(T), BUFFERS = 1, TERMS = 0, G = CW / 8;
    struct Ahead { uint4 hi[G], lo[G]; };
    static __device__ __forceinline__ bool begin(const TypedFinal<T>&, float*, int, int, int) { return true; }
    static __device__ __forceinline__ int row_term(const TypedFinal<T>&, long long, bool) { return 0; }
    static __device__ __forceinline__ void ahead(const TypedFinal<T>& e, int batch, long long row, int col, int left, Ahead& a) {
        const __half* p = e.o.c + batch * e.o.c_batch + row * e.o.c_ld + col;
#pragma unroll
        for (int c = 0; c < G; ++c)
            if (c * 8 < left) {
                a.hi[c] = *reinterpret_cast<const uint4*>(p + c * 8);
                a.lo[c] = *reinterpret_cast<const uint4*>(p + e.o.c_plane + c * 8);
            }
    }
    static __device__ __forceinline__ void finish(const TypedFinal<T>& e, const CUtensorMap* y, const CUtensorMap*, uint8_t* buffer, float (&v)[CW], const float*, int, int batch, int row0, int col,
                                                  int, int lane, int, bool, const Ahead& a, bool store) {
#pragma unroll
        for (int c = 0; c < G; ++c) {
            float ch[8], cl[8];
            unpack<__half>(a.hi[c], ch);
            unpack<__half>(a.lo[c], cl);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c * 8 + i] = fmaf(e.o.beta, ch[i] + cl[i], v[c * 8 + i] * e.o.alpha);
        }
        put_row<T>(buffer, lane, v);
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        __syncwarp();
        if (lane == 0 && store) { tma_store_3d(y, buffer, col, row0, batch); tma_store_commit(); }
    }
};

template <>
struct RowOut<PartialOut> {
    static constexpr int CW = 16, BUFFERS = 1, TERMS = 0;
    struct Ahead {};
    static __device__ __forceinline__ bool begin(const PartialOut&, float*, int, int, int) { return true; }
    static __device__ __forceinline__ int row_term(const PartialOut&, long long, bool) { return 0; }
    static __device__ __forceinline__ void ahead(const PartialOut&, int, long long, int, int, Ahead&) {}
    static __device__ __forceinline__ void finish(const PartialOut&, const CUtensorMap* y, const CUtensorMap*, uint8_t* buffer, float (&v)[CW], const float*, int, int slice, int row0, int col, int,
                                                  int lane, int, bool, const Ahead&, bool store) {
        put_row<float>(buffer, lane, v);
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        __syncwarp();
        if (lane == 0 && store) { tma_store_3d(y, buffer, col, row0, slice); tma_store_commit(); }
    }
};

constexpr int PAIR_THREADS = 384;                                // three warpgroups: two that take sums out, one that fetches and issues (two of its warps idle)
constexpr int PAIR_HALF = 128 * GEMM_ROW_BYTES;                  // 128 rows of 64 elements
template <int PL> __host__ __device__ constexpr int pair_stage_bytes() { return 2 * PL * PAIR_HALF; }
template <int PL> __host__ __device__ constexpr int pair_stages() { return PL == 1 ? 5 : 3; }
// Per warp, behind the stages: 64-byte rows of results on their way out (one buffer, or two), the columns' terms as fp32.
constexpr int PAIR_PATCH_COLUMNS = 16, PAIR_PATCH_PITCH = PAIR_PATCH_COLUMNS + 4;
template <class EPI> __host__ __device__ constexpr int pair_warp_bytes() {
    const int buffers = RowOut<EPI>::BUFFERS * PAIR_BUFFER, patch = 32 * PAIR_PATCH_PITCH * 4;
    return (buffers > patch ? buffers : patch) + RowOut<EPI>::TERMS * 128 * 4;
}
template <class EPI, int PL> __host__ __device__ constexpr int pair_smem_bytes() {
    return 1024 + pair_stages<PL>() * pair_stage_bytes<PL>() + 8 * pair_warp_bytes<EPI>();
}

// A load into this block's shared memory that signals a barrier of either block of the pair.
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(dst), "l"(map),
                 "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void umma_f16_pair(uint32_t leader, uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %3};\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "setp.ne.b32 q, %6, 0;\n\t"
        "@q tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, p;\n\t}\n"
        :: "r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(TILE_DESC_HI), "r"(idesc), "r"(accumulate), "r"(leader)
        : "memory");
}
// Completion of the pair's MMAs issued so far, on the barrier at this place in both blocks.
__device__ __forceinline__ void umma_commit_both(uint32_t leader, uint32_t bar0, uint32_t bar1) {
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %2, 0;\n\t"
        "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t"
        "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%1];\n\t}\n"
        ::"r"(bar0), "r"(bar1), "r"(leader) : "memory");
}
__device__ __forceinline__ void tmem_ld32_issue(uint32_t taddr, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
          "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]),
          "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld32_wait(uint32_t (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;\n"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]),
                   "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]),
                   "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])
                 :: "memory");
}

// Tiles in bands of eight tile rows, column by column within a band: the tiles under way at a time share few rows and columns.
// A symmetric result: only the tiles on and below the diagonal, row by row.
// Parts of the reduction of one tile follow one another.
__device__ __forceinline__ void pair_tile(int t, int tiles_m, int tiles_n, int symmetric, int split, int blocks, int& batch, int& tm, int& tn, int& part, int& kb0, int& kb1) {
    part = 0;
    if (split > 1) {
        part = t % split;
        t /= split;
    }
    kb0 = (int)((long long)blocks * part / split);
    kb1 = (int)((long long)blocks * (part + 1) / split);
    const int per = symmetric ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n;
    batch = t / per;
    t -= batch * per;
    if (symmetric) {
        tm = (int)((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
        while (tm * (tm + 1) / 2 > t) --tm;
        while ((tm + 1) * (tm + 2) / 2 <= t) ++tm;
        tn = t - tm * (tm + 1) / 2;
        return;
    }
    const int band = t / (8 * tiles_n), first = band * 8, height = tiles_m - first < 8 ? tiles_m - first : 8;
    t -= band * 8 * tiles_n;
    tn = t / height;
    tm = first + t - tn * height;
}

template <class EPI, int PL>
__global__ void __launch_bounds__(PAIR_THREADS, 1) gemm_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                           const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_z, const TileArgs g,
                                                           const EPI epi) {
    extern __shared__ uint8_t smem_raw[];
    constexpr int S = pair_stages<PL>(), STAGE = pair_stage_bytes<PL>(), PC = PAIR_PATCH_COLUMNS, PITCH = PAIR_PATCH_PITCH;
    __shared__ uint64_t full[S], empty[S], acc_full[2], acc_empty[2];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)(blockIdx.x & 1), pairs = (int)(gridDim.x >> 1);
    const int blocks = (g.red + GEMM_BK - 1) / GEMM_BK, chunk = PL == 2 ? GEMM_CHUNK : blocks;
    const int tiles_m = (g.out_rows + 255) / 256, tiles_n = (g.out_cols + 255) / 256, count = (g.symmetric ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n) * g.batch * g.split;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 16); }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    __syncthreads();
    cluster_sync_all();                                           // the partner's barriers are ready too
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    const uint32_t tmem = uni(tmem_slot);
    let_next_kernel_start();
    wait_for_previous_kernel();

    // Split products keep 128 sums a thread.  Registers are dealt anew among the warpgroups: 2 * 128 * 208 + 128 * 80 = 63488 of the
    // 384 * 168 = 64512 the block was launched with.  (Each at the head of its warpgroup's own code: the compiler counts registers by
    // what it can reach.)
    if (warp >= 8) {
      if (PL == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 80;\n");
      if (warp == 8) {
        const bool leader = elect_one();
        int i = 0;                                                // stages filled so far
        bool ok = true;
        for (int t = (int)(blockIdx.x >> 1); t < count && ok; t += pairs) {
            int batch, tm, tn, part, kb0, kb1;
            pair_tile(t, tiles_m, tiles_n, g.symmetric, g.split, blocks, batch, tm, tn, part, kb0, kb1);
            const int a0 = tm * 256 + rank * 128, b0 = tn * 256 + rank * 128;
            for (int kb = kb0; kb < kb1; ++kb, ++i) {
                const int s = i % S, k = kb * GEMM_BK;
                ok = mbar_wait_warp(&empty[s], ((i / S) & 1) ^ 1, &abort_flag, g.wait_limit);
                if (!ok) break;
                if (leader) {
                    const uint32_t base = smem_u32(tiles) + s * STAGE, bar = cluster_addr(&full[s], 0);
                    if (rank == 0) mbar_expect_tx(&full[s], 2 * STAGE);
#pragma unroll
                    for (int p = 0; p < PL; ++p) {
                        const uint32_t at = base + p * PAIR_HALF, bt = base + (PL + p) * PAIR_HALF;
                        const int z = batch * PL + p;
                        if (!g.a_mn) tma_load_3d_pair(at, &map_a, k, a0, z, bar);
                        else { tma_load_3d_pair(at, &map_a, a0, k, z, bar); tma_load_3d_pair(at + 8192, &map_a, a0 + 64, k, z, bar); }
                        if (!g.b_mn) tma_load_3d_pair(bt, &map_b, k, b0, z, bar);
                        else { tma_load_3d_pair(bt, &map_b, b0, k, z, bar); tma_load_3d_pair(bt + 8192, &map_b, b0 + 64, k, z, bar); }
                    }
                }
                __syncwarp();
            }
        }
      } else if (warp == 9 && rank == 0) {
            const uint32_t leader = elect_one() ? 1u : 0u;
            const uint32_t idesc = gemm_idesc(256, 256, g.bf16, g.a_mn, g.b_mn);
            const uint32_t a_step = g.a_mn ? 2048 >> 4 : 32 >> 4, b_step = g.b_mn ? 2048 >> 4 : 32 >> 4;
            int i = 0, c = 0;                                     // stages and accumulators used so far
            bool ok = true;
            for (int t = (int)(blockIdx.x >> 1); t < count && ok; t += pairs) {
                int batch, tm, tn, part, kb0, kb1;
                pair_tile(t, tiles_m, tiles_n, g.symmetric, g.split, blocks, batch, tm, tn, part, kb0, kb1);
                for (int kb = kb0; kb < kb1 && ok; ++kb, ++i) {
                    const int s = i % S, in_chunk = (kb - kb0) % chunk;
                    if (in_chunk == 0 && c >= 2) ok = mbar_wait_cluster_warp(&acc_empty[c & 1], ((c >> 1) & 1) ^ 1, &abort_flag, g.wait_limit);
                    ok = ok && mbar_wait_warp(&full[s], (i / S) & 1, &abort_flag, g.wait_limit);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                    const bool last = in_chunk == chunk - 1 || kb == kb1 - 1;
                    if ((g.test_flags & 1) == 0) {                // (give-up test: nothing is ever issued)
                        const uint32_t d = tmem + (uint32_t)((c & 1) * 256), base = smem_u32(tiles) + s * STAGE;
                        const uint32_t ah = tile_desc_lo(base, g.a_mn), bh = tile_desc_lo(base + PL * PAIR_HALF, g.b_mn);
#pragma unroll
                        for (int k = 0; k < GEMM_BK / 16; ++k) {
                            const uint32_t a = ah + k * a_step, b = bh + k * b_step;
                            umma_f16_pair(leader, d, a, b, idesc, (in_chunk | k) != 0);
                            if (PL == 2) {
                                umma_f16_pair(leader, d, a, b + (PAIR_HALF >> 4), idesc, 1u);
                                umma_f16_pair(leader, d, a + (PAIR_HALF >> 4), b, idesc, 1u);
                            }
                        }
                        umma_commit_both(leader, cluster_addr(&empty[s], 0), cluster_addr(&empty[s], 1));
                        if (last) umma_commit_both(leader, cluster_addr(&acc_full[c & 1], 0), cluster_addr(&acc_full[c & 1], 1));
                    }
                    c += last;
                }
            }
      }
    } else {
        if (PL == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;\n");
        using Rows = RowOut<EPI>;
        constexpr int CW = Rows::CW, WARP_BYTES = pair_warp_bytes<EPI>();
        uint8_t* mine = tiles + S * STAGE + warp * (WARP_BYTES - Rows::TERMS * 512);
        float* terms = reinterpret_cast<float*>(tiles + S * STAGE + 8 * (WARP_BYTES - Rows::TERMS * 512)) + warp * Rows::TERMS * 128;
        float* patch = reinterpret_cast<float*>(mine);
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (warp >> 2) * 128;
        constexpr int N = EPI::N, PER_ROW = PC / N, ROWS = 32 / PER_ROW, STEPS = 32 / ROWS;
        int c = 0;
        bool ok = true;
        for (int t = (int)(blockIdx.x >> 1); t < count && ok; t += pairs) {
            int batch, tm, tn, part, kb0, kb1;
            pair_tile(t, tiles_m, tiles_n, g.symmetric, g.split, blocks, batch, tm, tn, part, kb0, kb1);
            const int row0 = tm * 256 + rank * 128 + (warp & 3) * 32, col0 = tn * 256 + (warp >> 2) * 128;
            const int slice = part * g.batch + batch;             // (parts: a matrix each)
            // rows by TMA
            bool plain = false;
            int row_term = 0;
            if (g.packs) {
                __syncwarp();                                     // (the terms of the tile before are read)
                plain = Rows::begin(epi, terms, col0, g.out_cols, lane);
                row_term = Rows::row_term(epi, row0 + lane, row0 + lane < g.out_rows);
                __syncwarp();
            }
            typename Rows::Ahead row_ahead;
            auto rows_ahead = [&](int column) {
                if (row0 + lane < g.out_rows) Rows::ahead(epi, slice, row0 + lane, col0 + column, g.out_cols - col0 - column, row_ahead);
            };
            auto rows_out = [&](int column, float (&v)[CW]) {
                if (lane == 0) tma_store_wait_read();             // the buffers' last stores have read them
                __syncwarp();
                const int col = col0 + column;
                Rows::finish(epi, &map_y, &map_z, mine, v, terms + column, g.symmetric && tm != tn ? g.out_rows : 0, slice, row0, col, g.out_cols - col, lane, row_term, plain, row_ahead,
                             col < g.out_cols && row0 < g.out_rows);
            };
            // lanes that share rows, through a patch: outputs whose rows start anywhere
            auto patch_out = [&](int column) {
                __syncwarp();
                const int pack_col = (lane % PER_ROW) * N, col = col0 + column + pack_col, left = g.out_cols - col;
                typename EPI::Columns columns;
                typename EPI::Ahead ahead[STEPS];
                if (left > 0) {
                    epi.columns(col, left, false, columns);
#pragma unroll
                    for (int i = 0; i < STEPS; ++i)
                        if (row0 + lane / PER_ROW + i * ROWS < g.out_rows) epi.ahead(slice, row0 + lane / PER_ROW + i * ROWS, col, left, false, ahead[i]);
#pragma unroll
                    for (int i = 0; i < STEPS; ++i) {
                        const int r = lane / PER_ROW + i * ROWS;
                        float v[N];
                        const float* p = patch + r * PITCH + pack_col;
#pragma unroll
                        for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(v + e) = *reinterpret_cast<const float4*>(p + e);
                        if (row0 + r < g.out_rows) epi.pack(slice, row0 + r, col, left, false, v, columns, ahead[i]);
                    }
                }
                __syncwarp();
            };
            auto put_patch = [&](const float* f) {
#pragma unroll
                for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4*>(patch + lane * PITCH + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
            };
            if constexpr (PL == 2) {
                float acc[128];
#pragma unroll
                for (int j = 0; j < 128; ++j) acc[j] = 0.0f;
                for (int kb = kb0; kb < kb1 && ok; kb += chunk, ++c) {
                    ok = mbar_wait_bounded(&acc_full[c & 1], (c >> 1) & 1, &abort_flag, g.wait_limit);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#pragma unroll
                    for (int j = 0; j < 128; j += 32) {
                        uint32_t v[32];
                        tmem_ld32_issue(lanes + (c & 1) * 256 + j, v);
                        tmem_ld32_wait(v);
#pragma unroll
                        for (int e = 0; e < 32; ++e) acc[j + e] += __uint_as_float(v[e]);
                    }
                    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
                    if (lane == 0) mbar_arrive_cluster(cluster_addr(&acc_empty[c & 1], 0));
                }
                if (!ok) break;
#pragma unroll 1
                for (int j = 0; j < 128 / CW; ++j) {              // (registers have no index: one copy of the moves a position)
                    if (g.packs) rows_ahead(j * CW);
                    float v[CW];
#pragma unroll
                    for (int q = 0; q < 128 / CW; ++q)
                        if (q == j) {
#pragma unroll
                            for (int e = 0; e < CW; ++e) v[e] = acc[q * CW + e];
                        }
                    if (g.packs) rows_out(j * CW, v);
                    else
#pragma unroll
                        for (int h = 0; h < CW; h += 16) {
                            put_patch(v + h);
                            patch_out(j * CW + h);
                        }
                }
            } else {
                if (g.packs) rows_ahead(0);
                ok = mbar_wait_bounded(&acc_full[c & 1], (c >> 1) & 1, &abort_flag, g.wait_limit);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#pragma unroll 1
                for (int j = 0; j < 128; j += 32) {
                    uint32_t raw[32];
                    tmem_ld32_issue(lanes + (c & 1) * 256 + j, raw);
                    if (g.packs && j > 0) rows_ahead(j);
                    tmem_ld32_wait(raw);
                    if (j == 96) {
                        asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
                        if (lane == 0) mbar_arrive_cluster(cluster_addr(&acc_empty[c & 1], 0));
                    }
#pragma unroll
                    for (int h = 0; h < 32; h += CW) {
                        float v[CW];
#pragma unroll
                        for (int e = 0; e < CW; ++e) v[e] = __uint_as_float(raw[h + e]);
                        if (g.packs) rows_out(j + h, v);
                        else
#pragma unroll
                            for (int q = 0; q < CW; q += 16) {
                                put_patch(v + q);
                                patch_out(j + h + q);
                            }
                    }
                }
                ++c;
            }
        }
        if (lane == 0) tma_store_wait_all();
    }
    __syncthreads();
    if (abort_flag) {
        giveup_drain();
        if (threadIdx.x == 0) atomicAdd(&g_gemm_pair_timeouts, 1ull);
    }
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    cluster_sync_all();                                           // no block leaves while the other's MMAs or arrivals reach it
    if (warp == 9)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(512u) : "memory");
}

unsigned long long gemm_pair_timeouts() {
    unsigned long long n = 0;
    return cudaMemcpyFromSymbol(&n, g_gemm_pair_timeouts, sizeof(n)) == cudaSuccess ? n : 0;
}

// Tensor map of outputs: matrices [rows][cols] of `slices`, 64 bytes by 32 rows a store.  False: rows that do not start on 16 bytes.
template <typename T>
static bool result_map(const void* p, long long rows, long long cols, long long ld, long long slices, long long slice, CUtensorMap* map) {
    if (!p) return true;
    if (((uintptr_t)p & 15) != 0 || (ld * sizeof(T)) % 16 != 0 || (slice * sizeof(T)) % 16 != 0) return false;
    const CUtensorMapDataType type = std::is_same<T, float>::value ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : std::is_same<T, __half>::value ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)slices};
    const cuuint64_t strides[2] = {(cuuint64_t)ld * sizeof(T), (cuuint64_t)(slices > 1 ? slice : ld * rows) * sizeof(T)};
    const cuuint32_t box[3] = {(cuuint32_t)(64 / sizeof(T)), 32, 1};
    return encode_map(map, type, p, dims, strides, box, true);
}
template <typename T>
static bool result_maps(const LinearOut<T>& e, const GemmShape& s, CUtensorMap* y, CUtensorMap* z) {
    const auto whole = [](const void* p, long long ld) { return !p || (((uintptr_t)p & 15) == 0 && (ld * sizeof(T)) % 16 == 0); };
    return whole(e.o.residual, e.o.ldr) && result_map<T>(e.o.y, s.rows, s.cols, e.o.ldy, 1, 0, y) && result_map<T>(e.o.z, s.rows, s.cols, e.o.ldz, 1, 0, z);
}
static bool result_maps(const PlanesOut& e, const GemmShape& s, CUtensorMap* y, CUtensorMap*) { return result_map<__half>(e.y, s.rows, s.cols, e.ld, 2LL * s.batch, e.plane, y); }
template <typename T>
static bool result_maps(const TypedFinal<T>& e, const GemmShape& s, CUtensorMap* y, CUtensorMap*) {
    return result_map<T>(e.o.y, s.rows, s.cols, e.o.ld, s.batch, e.o.batch, y);
}
static bool result_maps(const PartialOut& e, const GemmShape& s, CUtensorMap* y, CUtensorMap*) {
    return result_map<float>(e.y, s.rows, s.cols, e.ld, (long long)s.batch * e.parts, e.batch, y);
}

template <class EPI, int PL>
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
    g.wait_limit = device_wait_limit();
    g.test_flags = device_test_flags();
    const long long side = (s.rows + 255) / 256, tiles = (symmetric ? side * (side + 1) / 2 : side * ((s.cols + 255) / 256)) * s.batch * split;
    if (tiles >= (1LL << 30)) return EBS_ERR_OVERFLOW;
    CUtensorMap a, b, y{}, z{};
    if (!gemm_operand_map(A, s.rows, s.red, s.batch, 128, bf16, &a) || !gemm_operand_map(B, s.cols, s.red, s.batch, 128, bf16, &b)) return EBS_ERR_CUDA;
    g.packs = result_maps(epi, s, &y, &z);
    if (symmetric && !g.packs) return EBS_ERR_CUDA;               // (kept planes always have whole rows)
    auto kern = gemm_pair_kernel<EPI, PL>;
    constexpr int bytes = pair_smem_bytes<EPI, PL>();
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

// Adds the parts of a product split over its reduction, in their order, and finishes the results: a thread a pack.
template <class EPI>
__global__ void __launch_bounds__(256) reduce_parts_kernel(const PartialOut in, const int parts, const int rows, const int cols, const int packs, const EPI epi) {
    constexpr int N = EPI::N;
    let_next_kernel_start();
    wait_for_previous_kernel();
    const int per_row = (cols + N - 1) / N, batch = (int)blockIdx.y;
    const long long items = (long long)per_row * rows;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < items; i += gridDim.x * 256LL) {
        const int row = (int)(i / per_row), col = (int)(i - (long long)row * per_row) * N, left = cols - col;
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
        epi.pack(batch, row, col, left, vec, v, columns, ahead);
    }
}
template <class EPI, int PL>
static int launch_pair_or_parts(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const EPI& epi, bool bf16, bool packs, const GemmRoute& route, float* scratch, cudaStream_t st) {
    if (route.split == 1) return launch_pair<EPI, PL>(A, B, s, epi, bf16, 1, st);
    PartialOut p;
    p.y = scratch;
    p.ld = (s.cols + 7) & ~7LL;
    p.batch = p.ld * s.rows;
    p.part = p.batch * s.batch;
    p.parts = route.split;
    const int rc = launch_pair<PartialOut, PL>(A, B, s, p, bf16, route.split, st);
    if (rc) return rc;
    const long long items = (long long)((s.cols + EPI::N - 1) / EPI::N) * s.rows, blocks = (items + 255) / 256;
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
    const long long side = (s.rows + 255) / 256, tiles = (s.symmetric ? side * (side + 1) / 2 : side * ((s.cols + 255) / 256)) * s.batch;
    const int blocks = (s.red + GEMM_BK - 1) / GEMM_BK;
    r.pair = s.rows > 128 && s.cols > 128 && tiles >= 32;
    if (!r.pair && s.rows > 128 && s.cols > 128 && blocks >= 64) {
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
