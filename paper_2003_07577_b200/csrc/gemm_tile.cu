// Tile kernel of the real-valued products: one 128 x TN tile of results a thread block, or a cluster of thread blocks that share
// its reduction.
//
// Warp 8 fetches operand tiles by TMA, warp 9 issues the MMAs, warps 0-7 take the sums out of tensor memory.
//  - Split products (PL = 2: operands as two fp16 planes hi + lo): three MMAs a step, hi*hi + hi*lo + lo*hi.  The tensor core
//    truncates when it adds to an accumulator, so that long sums drift by their length; every few (GemmShape::chunk) stages the accumulator
//    is therefore taken out and added up in registers, rounded to nearest, while the MMAs go on in a second one.
//  - Long sums of 16-bit operands leave the tensor core likewise, every GEMM_LONG stages.
//  - Few result rows (SWAP): the operand with many rows takes the 128 lanes, the few rows the N side of the MMA.  Such products
//    are bound by the bytes of the large operand.
//  - Few tiles and a long reduction: up to eight thread blocks of a cluster take a part of the reduction each; the sums meet in
//    shared memory, each block adds a share of the tile over all parts in block order and writes it.
#include "gemm_umma.cuh"
#include "gemm_tile.cuh"

namespace ebs {

static __device__ unsigned long long g_gemm_tile_timeouts = 0ull;

template <int TN, int PL>
__host__ __device__ constexpr int tile_stage_bytes() { return PL * (128 + TN) * GEMM_ROW_BYTES; }

// One launch: a product, or two that do not depend on each other.
template <class EPI>
struct TileLaunch {
    CUtensorMap a[2], b[2];                                      // A: the operand on the 128 lanes, B: the one on the TN columns
    TileArgs g[2];
    EPI epi[2];
    unsigned second;                                             // first thread block of the second product
};

template <class EPI, int TN, int PL, bool SWAP, bool CHUNKS>
__global__ void __launch_bounds__(320, 1) gemm_tile_kernel(const __grid_constant__ TileLaunch<EPI> launch) {
    // SWAP: lanes are the result's columns.  CHUNKS: sums leave tensor memory every g.chunk stages and go on in registers
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full[8], empty[8], acc_full[2], acc_empty[2], received;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    constexpr int STAGE = tile_stage_bytes<TN, PL>();
    constexpr int A_BYTES = 128 * GEMM_ROW_BYTES, B_BYTES = TN * GEMM_ROW_BYTES;
    constexpr int COLS = (CHUNKS ? 2 : 1) * TN < 32 ? 32 : (CHUNKS ? 2 : 1) * TN;            // TMEM columns: one accumulator, or two taken in turn
    uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int which = blockIdx.x >= launch.second;
    const TileArgs g = launch.g[which];                           // (copies: an indexed parameter is a load at every use)
    const EPI epi = launch.epi[which];
    const CUtensorMap *map_a = &launch.a[which], *map_b = &launch.b[which];
    if (warp >= 8 && lane == 0) asm volatile("prefetch.tensormap [%0];\n" ::"l"(warp == 8 ? map_a : map_b) : "memory");
    // parts of a tile follow one another (a cluster), then tiles along the lanes, along the columns, of the batch
    const int split = g.split;
    int tile = (int)(blockIdx.x - (which ? launch.second : 0u));
    if (tile >= g.blocks) return;                                 // (whole clusters of blocks; only where no block waits for another)
    const int part = tile % split;
    tile /= split;
    const int a0 = tile % g.tiles_a * 128;
    tile /= g.tiles_a;
    const int b0 = tile % g.tiles_b * TN, batch = tile / g.tiles_b;
    const int blocks = (g.red + GEMM_BK - 1) / GEMM_BK;
    const int kb0 = (int)((long long)blocks * part / split), kb1 = (int)((long long)blocks * (part + 1) / split);
    const int nkb = kb1 - kb0;
    const int chunk = CHUNKS ? g.chunk : (nkb > 0 ? nkb : 1);

    if (threadIdx.x == 0) {
        for (int s = 0; s < g.stages; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 8); }
        mbar_init(&received, 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_slot)), "r"((uint32_t)COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    const uint32_t tmem = uni(tmem_slot);
    let_next_kernel_start();
    wait_for_previous_kernel();

    float acc[CHUNKS ? TN / 2 : 1];                               // (this thread's sums)
    // How the results are shared out at the end: warps 0-7, a thread keeps its pack of columns and takes rows STRIDE apart, what the next one
    // needs from memory on its way.  One small loop: unrolled over eight rows the code of a tile's end, run once, took 2.5 us to arrive from
    // the second-level cache (128 x 128 results; 9 us from memory).
    constexpr int INNER = SWAP ? 128 : TN, OUTER = SWAP ? TN : 128, PITCH = INNER + 4;
    constexpr int N = EPI::N, PER_ROW = INNER / N, STRIDE = 256 / PER_ROW;
    static_assert(PER_ROW <= 64, "packs of a row");
    const int outer0 = SWAP ? b0 : a0, inner0 = SWAP ? a0 : b0;
    const int o_begin = OUTER * part / split, o_last = g.out_rows - outer0;
    int o_end = OUTER * (part + 1) / split;
    if (o_end > o_last) o_end = o_last;
    const int pack = (threadIdx.x % PER_ROW) * N, ocol = inner0 + pack, left = g.out_cols - ocol, first = o_begin + (int)threadIdx.x / PER_ROW;
    const bool vec = g.packs && left >= N, writes = warp < 8 && left > 0;
    typename EPI::Columns columns;
    typename EPI::Ahead next;
    if (writes) {
        epi.columns(ocol, left, vec, columns);
        if (first < o_end) epi.ahead(batch, outer0 + first, ocol, left, vec, next);
        epi.touch();
    }
    if (warp == 8) {
        const bool leader = elect_one();
        for (int i = 0; i < nkb; ++i) {
            const int s = i % g.stages, k = (kb0 + i) * GEMM_BK;
            if (!mbar_wait_warp(&empty[s], ((i / g.stages) & 1) ^ 1, &abort_flag, g.wait_limit)) break;
            if (leader) {
                const uint32_t base = smem_u32(tiles) + s * STAGE, bar = smem_u32(&full[s]);
                mbar_expect_tx(&full[s], STAGE);
#pragma unroll
                for (int p = 0; p < PL; ++p) {
                    const uint32_t at = base + p * A_BYTES, bt = base + PL * A_BYTES + p * B_BYTES;
                    const int z = batch * PL + p;
                    if (!g.a_mn) tma_load_3d(at, map_a, k, a0, z, bar);
                    else { tma_load_3d(at, map_a, a0, k, z, bar); tma_load_3d(at + 8192, map_a, a0 + 64, k, z, bar); }
                    if (!g.b_mn) tma_load_3d(bt, map_b, k, b0, z, bar);
                    else
#pragma unroll
                        for (int h = 0; h < (TN + 63) / 64; ++h) tma_load_3d(bt + h * 8192, map_b, b0 + h * 64, k, z, bar);
                }
            }
            __syncwarp();
        }
    } else if (warp == 9) {
        const uint32_t leader = elect_one() ? 1u : 0u;
        const uint32_t idesc = gemm_idesc(128, TN, g.bf16, g.a_mn, g.b_mn);
        const uint32_t a_step = g.a_mn ? 2048 >> 4 : 32 >> 4, b_step = g.b_mn ? 2048 >> 4 : 32 >> 4;
        for (int i = 0, c = 0, in_chunk = 0; i < nkb; ++i) {
            const int s = i % g.stages;
            if (CHUNKS && in_chunk == 0 && c >= 2 && !mbar_wait_warp(&acc_empty[c & 1], ((c >> 1) & 1) ^ 1, &abort_flag, g.wait_limit)) break;
            if (!mbar_wait_warp(&full[s], (i / g.stages) & 1, &abort_flag, g.wait_limit)) break;
            asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
            const int first = in_chunk;
            const uint32_t d = tmem + (CHUNKS ? (uint32_t)((c & 1) * TN) : 0u);
            uint64_t* out = &acc_full[c & 1];
            const bool last = ++in_chunk == chunk || i == nkb - 1;
            if (last) { in_chunk = 0; ++c; }
            if (g.test_flags & 1) continue;                       // (give-up test: nothing is ever issued)
            const uint32_t base = smem_u32(tiles) + s * STAGE;
            const uint32_t ah = tile_desc_lo(base, g.a_mn), bh = tile_desc_lo(base + PL * A_BYTES, g.b_mn);
            if (PL == 2)                                          // (the small products first: each MMA truncates at the size of what is there)
#pragma unroll
                for (int k = 0; k < GEMM_BK / 16; ++k) {
                    const uint32_t a = ah + k * a_step, b = bh + k * b_step;
                    umma_f16(leader, d, a, b + (B_BYTES >> 4), idesc, (first | k) != 0);
                    umma_f16(leader, d, a + (A_BYTES >> 4), b, idesc, 1u);
                }
#pragma unroll
            for (int k = 0; k < GEMM_BK / 16; ++k) umma_f16(leader, d, ah + k * a_step, bh + k * b_step, idesc, PL == 2 || (first | k) != 0);
            umma_commit_pred(leader, &empty[s]);
            if (last) umma_commit_pred(leader, out);
        }
    } else {
        const uint32_t row = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (warp >> 2) * (TN / 2);
        bool ok = true;
        if (CHUNKS) {
#pragma unroll
            for (int j = 0; j < TN / 2; ++j) acc[j] = 0.0f;
            const int chunks = (nkb + chunk - 1) / chunk;
            for (int c = 0; c < chunks && ok; ++c) {
                ok = mbar_wait_bounded(&acc_full[c & 1], (c >> 1) & 1, &abort_flag, g.wait_limit);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                constexpr int W = TN / 2 < 32 ? TN / 2 : 32;
#pragma unroll
                for (int j = 0; j < TN / 2; j += W) {
                    uint32_t v[W];
                    tmem_load<W>(row + (c & 1) * TN + j, v);
#pragma unroll
                    for (int e = 0; e < W; ++e) acc[j + e] += __uint_as_float(v[e]);
                }
                asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
                if (lane == 0) mbar_arrive(&acc_empty[c & 1]);
            }
        } else if (nkb > 0) {
            ok = mbar_wait_bounded(&acc_full[0], 0, &abort_flag, g.wait_limit);
            asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
        }
    }
    __syncthreads();                                              // every MMA is done: the stages become the exchange of sums
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    // exchange[outer][inner]: inner runs along a row of the results
    float* exchange = reinterpret_cast<float*>(tiles);
    if (warp < 8 && !abort_flag) {
        const uint32_t row = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (warp >> 2) * (TN / 2);
        const int l = (warp & 3) * 32 + lane, n0 = (warp >> 2) * (TN / 2);
        uint32_t raw[CHUNKS ? 1 : TN / 2];
        if constexpr (!CHUNKS) tmem_load<TN / 2>(row, raw);
#pragma unroll
        for (int j = 0; j < TN / 2; j += 8) {
            float f[8];
            if (CHUNKS) {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = acc[j + e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = nkb > 0 ? __uint_as_float(raw[j + e]) : 0.0f;
            }
            if (SWAP) {
#pragma unroll
                for (int e = 0; e < 8; ++e) exchange[(n0 + j + e) * PITCH + l] = f[e];
            } else {
                *reinterpret_cast<float4*>(exchange + l * PITCH + n0 + j) = make_float4(f[0], f[1], f[2], f[3]);
                *reinterpret_cast<float4*>(exchange + l * PITCH + n0 + j + 4) = make_float4(f[4], f[5], f[6], f[7]);
            }
        }
    }
    // Parts: each block of the cluster sends every other one its share of the tile in one bulk copy and adds what it gets in block order.
    // (Read out of the other blocks' memory by its own loads, the exchange took 3.6 us for 128 x 128 results in four parts.)
    constexpr int EXCHANGE = OUTER * PITCH * 4;
    const int share = EXCHANGE / split;                           // bytes
    float* shares = reinterpret_cast<float*>(tiles + EXCHANGE);   // [part][OUTER / split][PITCH]
    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
    if (split > 1) cluster_sync_all();
    else __syncthreads();
    bool skip = abort_flag != 0;
    for (int q = 0; q < split && split > 1; ++q) {                // (a part that gave up leaves no sums: no block of the cluster goes on)
        int f;
        asm volatile("ld.shared::cluster.s32 %0, [%1];\n" : "=r"(f) : "r"(cluster_addr((const void*)&abort_flag, q)));
        skip |= f != 0;
    }
    if (split > 1 && !skip) {
        if (threadIdx.x == 288) {
            mbar_expect_tx(&received, (uint32_t)EXCHANGE);
            if ((g.test_flags & 2) == 0 || part != 0)             // (give-up test: one part's sums never come)
                for (int q = 0; q < split; ++q)
                    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n" ::"r"(
                                     cluster_addr(reinterpret_cast<uint8_t*>(shares) + part * share, q)), "r"(smem_u32(exchange) + q * share), "r"(share), "r"(cluster_addr(&received, q))
                                 : "memory");
        }
        if (warp < 8) skip = !mbar_wait_bounded(&received, 0, &abort_flag, g.wait_limit);
    }
    bool holes = false;
    if (!skip && writes) {
#pragma unroll 1
        for (int o = first; o < o_end; o += STRIDE) {
            const typename EPI::Ahead here = next;
            if (o + STRIDE < o_end) epi.ahead(batch, outer0 + o + STRIDE, ocol, left, vec, next);
            float v[N];
            const float* at = split == 1 ? exchange + o * PITCH + pack : shares + (o - o_begin) * PITCH + pack;
#pragma unroll
            for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(&v[e]) = *reinterpret_cast<const float4*>(at + e);
#pragma unroll 1
            for (int q = 1; q < split; ++q) {
                at += share / 4;
#pragma unroll
                for (int e = 0; e < N; e += 4) {
                    const float4 t = *reinterpret_cast<const float4*>(at + e);
                    v[e] += t.x; v[e + 1] += t.y; v[e + 2] += t.z; v[e + 3] += t.w;
                }
            }
            holes |= epi.pack(batch, outer0 + o, ocol, left, vec, v, columns, here);
        }
    }
    if constexpr (EPI::HOLES) {
        __shared__ unsigned masks[64];
        if (__syncthreads_or(holes)) finish_infinite<10, 0>(epi.o, outer0 + o_begin, o_end - o_begin, inner0, min(INNER, g.out_cols - inner0), masks);
    }
    if (split > 1) cluster_sync_all();                            // no block leaves while its sums are on their way
    if (abort_flag) {
        giveup_drain();
        if (threadIdx.x == 0) atomicAdd(&g_gemm_tile_timeouts, 1ull);
    }
    __syncthreads();
    if (warp == 9)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"((uint32_t)COLS) : "memory");
}

unsigned long long gemm_tile_timeouts() {
    unsigned long long n = 0;
    return cudaMemcpyFromSymbol(&n, g_gemm_tile_timeouts, sizeof(n)) == cudaSuccess ? n : 0;
}

// The form of a product: which operand lies on the lanes, how wide a tile is, in how many parts its reduction is taken.
struct TileForm {
    bool swap;
    int tn, split;
};
static long long tile_count(const GemmShape& s, const TileForm& f) {
    const int lanes = f.swap ? s.cols : s.rows, columns = f.swap ? s.rows : s.cols;
    return (long long)((lanes + 127) / 128) * ((columns + f.tn - 1) / f.tn) * s.batch;
}
// Parts of the reduction (us, measured): a stage takes 0.32 (split products 0.9), two, four or eight parts 1.2, 1.6 and 2.4 to meet.
static float tile_time(const GemmShape& s, int planes, int log_parts) {
    static const float meet[4] = {0.0f, 1.2f, 1.6f, 2.4f};
    const int parts = 1 << log_parts, blocks = (s.red + GEMM_BK - 1) / GEMM_BK;
    return (planes == 2 ? 0.9f : 0.32f) * (float)((blocks + parts - 1) / parts) + meet[log_parts];
}
// Thread blocks that run at once: clusters of eight and four fill only part of the GPU (36 of four no longer run at once: 768 x 768
// orthogonalised in 321 us on 36, 202 on clusters of two).
static int tile_blocks(int log_parts) {
    const int sms = gemm_sm_count();
    return log_parts == 3 ? sms * 3 / 4 : log_parts == 2 ? sms * 7 / 8 : sms;
}
static TileForm tile_form(const GemmShape& s, bool a_mn, int planes) {
    TileForm f;
    f.swap = s.rows <= 64 && !a_mn;
    f.tn = f.swap ? (s.rows <= 16 ? 16 : s.rows <= 32 ? 32 : 64) : (s.cols <= 64 ? 64 : 128);
    const long long tiles = tile_count(s, f);
    const int blocks = (s.red + GEMM_BK - 1) / GEMM_BK;
    f.split = 1;
    float best = tile_time(s, planes, 0);
    for (int i = 1; i < 4; ++i) {
        const int parts = 1 << i;
        if (tiles * parts > tile_blocks(i) || blocks < parts) break;
        const float t = tile_time(s, planes, i);
        if (t < best) { best = t; f.split = parts; }
    }
    return f;
}

// Fills in one product of a launch; blocks: its thread blocks.
template <class EPI>
static int tile_product(TileLaunch<EPI>* l, int which, const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const EPI& epi, bool bf16, bool packs, const TileForm& f,
                        unsigned* blocks) {
    TileArgs& g = l->g[which];
    const int lanes = f.swap ? s.cols : s.rows, columns = f.swap ? s.rows : s.cols;
    const GemmOperand &la = f.swap ? B : A, &lb = f.swap ? A : B;
    g = {};
    g.tiles_a = (lanes + 127) / 128;
    g.tiles_b = (columns + f.tn - 1) / f.tn;
    g.split = f.split;
    g.red = s.red;
    g.out_rows = s.rows;
    g.out_cols = s.cols;
    g.batch = s.batch;
    g.a_mn = la.mn_major;
    g.b_mn = lb.mn_major;
    g.bf16 = bf16;
    g.chunk = A.planes == 2 ? s.chunk : GEMM_LONG;
    g.packs = packs;
    g.wait_limit = device_wait_limit();
    g.test_flags = device_test_flags();
    l->epi[which] = epi;
    const long long count = (long long)g.tiles_a * g.tiles_b * s.batch * f.split;
    if (count >= (1LL << 30)) return EBS_ERR_OVERFLOW;
    *blocks = (unsigned)count;
    g.blocks = (int)count;
    return gemm_operand_map(la, lanes, s.red, s.batch, 128, bf16, &l->a[which]) && gemm_operand_map(lb, columns, s.red, s.batch, f.tn, bf16, &l->b[which]) ? EBS_OK : EBS_ERR_CUDA;
}

template <class EPI, int TN, int PL, bool SWAP, bool CHUNKS>
static int launch_tile(TileLaunch<EPI>& l, unsigned blocks, int cluster, cudaStream_t st) {
    constexpr int STAGE = tile_stage_bytes<TN, PL>();
    constexpr int EXCHANGE = (SWAP ? TN * 132 : 128 * (TN + 4)) * 4;
    const int most = (220 * 1024) / STAGE;
    int deepest = 1;
    for (TileArgs& g : l.g) {
        const int kb = (g.red + GEMM_BK - 1) / GEMM_BK, mine = (kb + g.split - 1) / g.split;
        g.stages = most < 8 ? most : 8;
        if (g.stages > mine) g.stages = mine;
        if (g.stages > deepest) deepest = g.stages;
    }
    const int sums = cluster > 1 ? 2 * EXCHANGE : EXCHANGE, bytes = (deepest * STAGE > sums ? deepest * STAGE : sums) + 1024;
    auto kern = gemm_tile_kernel<EPI, TN, PL, SWAP, CHUNKS>;
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        if (check_cuda(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 225 * 1024))) return EBS_ERR_CUDA;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    return launch_chained(kern, dim3(blocks), 320, (size_t)bytes, st, cluster, l);
}
template <class EPI, int PL, bool CHUNKS>
static int launch_tile_chunks(TileLaunch<EPI>& l, unsigned blocks, const TileForm& f, cudaStream_t st) {
    if (f.swap) {
        if (f.tn == 16) return launch_tile<EPI, 16, PL, true, CHUNKS>(l, blocks, f.split, st);
        if (f.tn == 32) return launch_tile<EPI, 32, PL, true, CHUNKS>(l, blocks, f.split, st);
        return launch_tile<EPI, 64, PL, true, CHUNKS>(l, blocks, f.split, st);
    }
    if (f.tn == 64) return launch_tile<EPI, 64, PL, false, CHUNKS>(l, blocks, f.split, st);
    return launch_tile<EPI, 128, PL, false, CHUNKS>(l, blocks, f.split, st);
}
template <class EPI, int PL>
static int launch_tile_form(TileLaunch<EPI>& l, unsigned blocks, const TileForm& f, cudaStream_t st) {
    if constexpr (PL == 2) {
        return launch_tile_chunks<EPI, PL, true>(l, blocks, f, st);
    } else {
        bool whole = true;
        for (const TileArgs& g : l.g) whole = whole && ((g.red + GEMM_BK - 1) / GEMM_BK + g.split - 1) / g.split <= GEMM_LONG;
        return whole ? launch_tile_chunks<EPI, PL, false>(l, blocks, f, st) : launch_tile_chunks<EPI, PL, true>(l, blocks, f, st);
    }
}
template <class EPI, int PL>
static int launch_one(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const EPI& epi, bool bf16, bool packs, cudaStream_t st) {
    TileLaunch<EPI> l;
    const TileForm f = tile_form(s, A.mn_major, PL);
    unsigned blocks = 0;
    const int rc = tile_product(&l, 0, A, B, s, epi, bf16, packs, f, &blocks);
    if (rc) return rc;
    l.g[1] = l.g[0];
    l.second = blocks;
    return launch_tile_form<EPI, PL>(l, blocks, f, st);
}
template <class EPI, int PL>
static int launch_two(const TileTask (&t)[2], const EPI (&epi)[2], bool bf16, const bool (&packs)[2], cudaStream_t st) {
    // both in one launch where they have the same form
    TileForm f[2];
    for (int i = 0; i < 2; ++i) f[i] = tile_form(t[i].s, t[i].a.mn_major, PL);
    if (f[0].swap != f[1].swap || f[0].tn != f[1].tn) {
        const int rc = launch_one<EPI, PL>(t[0].a, t[0].b, t[0].s, epi[0], bf16, packs[0], st);
        return rc ? rc : launch_one<EPI, PL>(t[1].a, t[1].b, t[1].s, epi[1], bf16, packs[1], st);
    }
    // a launch has one size of cluster: each product is taken in as many parts, or whole; what ends first, from the sizes (parts chosen for
    // each alone did not all run at once: gradients of 256 x 1024 -> 1000 fp32 45.5 us, so 25.8)
    const long long tiles[2] = {tile_count(t[0].s, f[0]), tile_count(t[1].s, f[1])};
    int cluster = 1;
    float best = 0.0f;
    for (int i = 0; i < 4; ++i)
        for (int split = i ? 1 : 0; split < (i ? 4 : 1); ++split) {       // bit p: product p in parts
            const int parts = 1 << i;
            long long all = 0;
            float time = 0.0f;
            bool fits = true;
            for (int p = 0; p < 2; ++p) {
                const bool in_parts = split >> p & 1;
                const float mine = tile_time(t[p].s, PL, in_parts ? i : 0);
                fits = fits && (!in_parts || (t[p].s.red + GEMM_BK - 1) / GEMM_BK >= parts);
                all += tiles[p] * (in_parts ? parts : 1);
                time = mine > time ? mine : time;
            }
            if (i == 0) time *= (float)((all + tile_blocks(0) - 1) / tile_blocks(0));
            else if (!fits || all > tile_blocks(i)) continue;
            if (i && time >= best) continue;
            best = time;
            cluster = parts;
            for (int p = 0; p < 2; ++p) f[p].split = split >> p & 1 ? parts : 1;
        }
    TileLaunch<EPI> l;
    unsigned first = 0, second = 0;
    int rc = tile_product(&l, 0, t[0].a, t[0].b, t[0].s, epi[0], bf16, packs[0], f[0], &first);
    if (!rc) rc = tile_product(&l, 1, t[1].a, t[1].b, t[1].s, epi[1], bf16, packs[1], f[1], &second);
    if (rc) return rc;
    l.second = (first + cluster - 1) / cluster * cluster;
    TileForm both = f[0];
    both.split = cluster;
    return launch_tile_form<EPI, PL>(l, l.second + (second + cluster - 1) / cluster * cluster, both, st);
}

int launch_gemm_tile(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const GemmOut& out, int dtype, cudaStream_t st) {
    const bool packs = packs_ok(out, element_size(dtype));
    if (dtype == EBS_F32) return launch_one<LinearOut<float>, 2>(A, B, s, {out}, false, packs, st);
    if (dtype == EBS_F16) return launch_one<LinearOut<__half>, 1>(A, B, s, {out}, false, packs, st);
    return launch_one<LinearOut<__nv_bfloat16>, 1>(A, B, s, {out}, true, packs, st);
}
int launch_gemm_tiles(const TileTask (&t)[2], const GemmOut (&out)[2], int dtype, cudaStream_t st) {
    const bool packs[2] = {packs_ok(out[0], element_size(dtype)), packs_ok(out[1], element_size(dtype))};
    if (dtype == EBS_F32) return launch_two<LinearOut<float>, 2>(t, {{out[0]}, {out[1]}}, false, packs, st);
    if (dtype == EBS_F16) return launch_two<LinearOut<__half>, 1>(t, {{out[0]}, {out[1]}}, false, packs, st);
    return launch_two<LinearOut<__nv_bfloat16>, 1>(t, {{out[0]}, {out[1]}}, true, packs, st);
}
int launch_gemm_tile(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const PlanesOut& out, cudaStream_t st) {
    return launch_one<PlanesOut, 2>(A, B, s, out, false, out.ld % 4 == 0, st);
}
int launch_gemm_tile(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const FinalOut& out, int dtype, cudaStream_t st) {
    const bool packs = out.ld * (long long)element_size(dtype) % 16 == 0 && (out.batch * (long long)element_size(dtype)) % 16 == 0;
    if (dtype == EBS_F32) return launch_one<TypedFinal<float>, 2>(A, B, s, {out}, false, packs, st);
    if (dtype == EBS_F16) return launch_one<TypedFinal<__half>, 2>(A, B, s, {out}, false, packs, st);
    return launch_one<TypedFinal<__nv_bfloat16>, 2>(A, B, s, {out}, false, packs, st);
}

bool encode_map(CUtensorMap* map, CUtensorMapDataType type, const void* p, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box, bool narrow) {
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        return cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) == cudaSuccess &&
                       found == cudaDriverEntryPointSuccess
                   ? reinterpret_cast<Encode>(fn)
                   : nullptr;
    }();
    const cuuint32_t one[3] = {1, 1, 1};
    if (!encode) return false;
    for (int attempt = 0; attempt < 2; ++attempt) {
        if (encode(map, type, 3, const_cast<void*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, narrow ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS)
            return true;
        // a thread's first call: the driver wants a current context, which runtime calls make and this one does not
        int dev = 0;
        if (attempt || cudaGetDevice(&dev) != cudaSuccess || cudaSetDevice(dev) != cudaSuccess) return false;
    }
    return false;
}
bool gemm_operand_map(const GemmOperand& o, int mn, int red, int batch, int box_mn, bool bf16, CUtensorMap* map) {
    const cuuint64_t inner = o.mn_major ? mn : red, outer = o.mn_major ? red : mn;
    const long long slice = o.planes > 1 ? o.plane_stride : (batch > 1 ? o.batch_stride : o.ld * (long long)outer);
    const cuuint64_t dims[3] = {inner, outer, (cuuint64_t)batch * o.planes};
    const cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)slice * 2};
    const cuuint32_t box[3] = {64, o.mn_major ? 64u : (cuuint32_t)box_mn, 1};
    return encode_map(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, o.p, dims, strides, box, false);
}

int gemm_sm_count() {
    static int counts[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
    if (!counts[dev]) {
        int n = 0;
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return 148;
        counts[dev] = n;
    }
    return counts[dev];
}

}  // namespace ebs
