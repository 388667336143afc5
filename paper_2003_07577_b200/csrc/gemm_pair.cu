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

constexpr int PAIR_THREADS = 384;                                // three warpgroups: two that take sums out, one that fetches and issues (two of its warps idle)
constexpr int PAIR_HALF = 128 * GEMM_ROW_BYTES;                  // 128 rows of 64 elements
template <int PL> __host__ __device__ constexpr int pair_stage_bytes() { return 2 * PL * PAIR_HALF; }
template <int PL> __host__ __device__ constexpr int pair_stages() { return PL == 1 ? 5 : 3; }
template <int PL> __host__ __device__ constexpr int pair_patch_columns() { return PL == 1 ? 32 : 16; }
template <int PL> __host__ __device__ constexpr int pair_smem_bytes() {
    return 1024 + pair_stages<PL>() * pair_stage_bytes<PL>() + 8 * 32 * (pair_patch_columns<PL>() + 4) * 4;
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
__device__ __forceinline__ void pair_tile(int t, int tiles_m, int tiles_n, int symmetric, int& batch, int& tm, int& tn) {
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
                                                           const TileArgs g, const EPI epi) {
    extern __shared__ uint8_t smem_raw[];
    constexpr int S = pair_stages<PL>(), STAGE = pair_stage_bytes<PL>(), PC = pair_patch_columns<PL>(), PITCH = PC + 4;
    __shared__ uint64_t full[S], empty[S], acc_full[2], acc_empty[2];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)(blockIdx.x & 1), pairs = (int)(gridDim.x >> 1);
    const int nkb = (g.red + GEMM_BK - 1) / GEMM_BK, chunk = PL == 2 ? GEMM_CHUNK : nkb, chunks = (nkb + chunk - 1) / chunk;
    const int tiles_m = (g.out_rows + 255) / 256, tiles_n = (g.out_cols + 255) / 256, count = (g.symmetric ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n) * g.batch;

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
            int batch, tm, tn;
            pair_tile(t, tiles_m, tiles_n, g.symmetric, batch, tm, tn);
            const int a0 = tm * 256 + rank * 128, b0 = tn * 256 + rank * 128;
            for (int kb = 0; kb < nkb; ++kb, ++i) {
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
                for (int kb = 0; kb < nkb && ok; ++kb, ++i) {
                    const int s = i % S, in_chunk = kb % chunk;
                    if (in_chunk == 0 && c >= 2) ok = mbar_wait_cluster_warp(&acc_empty[c & 1], ((c >> 1) & 1) ^ 1, &abort_flag, g.wait_limit);
                    ok = ok && mbar_wait_warp(&full[s], (i / S) & 1, &abort_flag, g.wait_limit);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                    const bool last = in_chunk == chunk - 1 || kb == nkb - 1;
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
        float* patch = reinterpret_cast<float*>(tiles + S * STAGE) + warp * 32 * PITCH;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (warp >> 2) * 128;
        constexpr int N = EPI::N, PER_ROW = PC / N, ROWS = 32 / PER_ROW;
        int c = 0;
        bool ok = true;
        for (int t = (int)(blockIdx.x >> 1); t < count && ok; t += pairs) {
            int batch, tm, tn;
            pair_tile(t, tiles_m, tiles_n, g.symmetric, batch, tm, tn);
            const int row0 = tm * 256 + rank * 128 + (warp & 3) * 32, col0 = tn * 256 + (warp >> 2) * 128;
            constexpr int STEPS = 32 / ROWS;
            const int pack_col = (lane % PER_ROW) * N, pack_row = row0 + lane / PER_ROW;
            typename EPI::Columns columns;
            typename EPI::Ahead ahead[STEPS];
            auto load_ahead = [&](int column) {                   // what the packs of these columns need, before the sums are there
                const int col = col0 + column + pack_col, left = g.out_cols - col;
                const bool vec = g.packs && left >= N;
                if (left <= 0) return;
                epi.columns(col, left, vec, columns);
#pragma unroll
                for (int i = 0; i < STEPS; ++i)
                    if (pack_row + i * ROWS < g.out_rows) epi.ahead(batch, pack_row + i * ROWS, col, left, vec, ahead[i]);
            };
            auto write = [&](int column) {                        // the patch's columns of this warp's rows
                __syncwarp();
                const int col = col0 + column + pack_col, left = g.out_cols - col;
                const bool vec = g.packs && left >= N;
#pragma unroll
                for (int i = 0; i < STEPS; ++i) {
                    const int row = pack_row + i * ROWS;
                    float v[N];
                    const float* p = patch + (lane / PER_ROW + i * ROWS) * PITCH + pack_col;
#pragma unroll
                    for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(v + e) = *reinterpret_cast<const float4*>(p + e);
                    if (row < g.out_rows && left > 0) epi.pack(batch, row, col, left, vec, v, columns, ahead[i]);
                }
                if (EPI::N == 4 && PL == 2 && g.symmetric && tm != tn) {
                    // the mirror image: four rows of the patch along a row of the results
                    const int mrow = col0 + column + lane % PC;
#pragma unroll
                    for (int i = 0; i < 32 * PC / 4 / 32; ++i) {
                        const int r = (lane / PC + i * (32 / PC)) * 4, mcol = row0 + r, mleft = g.out_cols - mcol;
                        float v[N];
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = patch[(r + e) * PITCH + lane % PC];
                        if (mrow >= g.out_rows || mleft <= 0) continue;
                        epi.ahead(batch, mrow, mcol, mleft, mleft >= N, ahead[i % STEPS]);
                        epi.pack(batch, mrow, mcol, mleft, mleft >= N, v, columns, ahead[i % STEPS]);
                    }
                }
                __syncwarp();
            };
            if constexpr (PL == 2) {
                float acc[128];
#pragma unroll
                for (int j = 0; j < 128; ++j) acc[j] = 0.0f;
                for (int q = 0; q < chunks && ok; ++q, ++c) {
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
                for (int j = 0; j < 8; ++j) {
                    auto put = [&](const float* f) {
#pragma unroll
                        for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4*>(patch + lane * PITCH + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
                    };
                    switch (j) {                                  // (registers have no index)
                        case 0: put(acc); break;
                        case 1: put(acc + 16); break;
                        case 2: put(acc + 32); break;
                        case 3: put(acc + 48); break;
                        case 4: put(acc + 64); break;
                        case 5: put(acc + 80); break;
                        case 6: put(acc + 96); break;
                        default: put(acc + 112); break;
                    }
                    load_ahead(j * 16);
                    write(j * 16);
                }
            } else {
                ok = mbar_wait_bounded(&acc_full[c & 1], (c >> 1) & 1, &abort_flag, g.wait_limit);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#pragma unroll 1
                for (int j = 0; j < 128; j += 32) {
                    uint32_t v[32];
                    tmem_ld32_issue(lanes + (c & 1) * 256 + j, v);
                    load_ahead(j);
                    tmem_ld32_wait(v);
                    if (j == 96) {
                        asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
                        if (lane == 0) mbar_arrive_cluster(cluster_addr(&acc_empty[c & 1], 0));
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4*>(patch + lane * PITCH + e) = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                    write(j);
                }
                ++c;
            }
        }
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

template <class EPI, int PL>
static int launch_pair(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const EPI& epi, bool bf16, bool packs, cudaStream_t st) {
    const bool symmetric = s.symmetric && PL == 2 && EPI::N == 4;
    TileArgs g = {};
    g.red = s.red;
    g.out_rows = s.rows;
    g.out_cols = s.cols;
    g.batch = s.batch;
    g.symmetric = symmetric;
    g.a_mn = A.mn_major;
    g.b_mn = B.mn_major;
    g.bf16 = bf16;
    g.packs = packs;
    g.wait_limit = device_wait_limit();
    g.test_flags = device_test_flags();
    const long long side = (s.rows + 255) / 256, tiles = (symmetric ? side * (side + 1) / 2 : side * ((s.cols + 255) / 256)) * s.batch;
    if (tiles >= (1LL << 30)) return EBS_ERR_OVERFLOW;
    CUtensorMap a, b;
    if (!gemm_operand_map(A, s.rows, s.red, s.batch, 128, bf16, &a) || !gemm_operand_map(B, s.cols, s.red, s.batch, 128, bf16, &b)) return EBS_ERR_CUDA;
    auto kern = gemm_pair_kernel<EPI, PL>;
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        if (check_cuda(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, pair_smem_bytes<PL>()))) return EBS_ERR_CUDA;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    const int pairs = gemm_sm_count() / 2;
    return launch_chained(kern, dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs))), PAIR_THREADS, pair_smem_bytes<PL>(), st, 2, a, b, g, epi);
}

bool gemm_pair_pays(const GemmShape& s) {
    const long long tiles = (long long)((s.rows + 255) / 256) * ((s.cols + 255) / 256) * s.batch;
    return s.rows > 128 && s.cols > 128 && tiles >= 32;
}

int launch_gemm_pair(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const GemmOut& out, int dtype, cudaStream_t st) {
    const bool packs = packs_ok(out, element_size(dtype));
    if (dtype == EBS_F32) return launch_pair<LinearOut<float>, 2>(A, B, s, {out}, false, packs, st);
    if (dtype == EBS_F16) return launch_pair<LinearOut<__half>, 1>(A, B, s, {out}, false, packs, st);
    return launch_pair<LinearOut<__nv_bfloat16>, 1>(A, B, s, {out}, true, packs, st);
}
int launch_gemm_pair(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const PlanesOut& out, cudaStream_t st) {
    return launch_pair<PlanesOut, 2>(A, B, s, out, false, out.ld % 4 == 0, st);
}
int launch_gemm_pair(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const FinalOut& out, int dtype, cudaStream_t st) {
    const bool packs = out.ld * (long long)element_size(dtype) % 16 == 0 && (out.batch * (long long)element_size(dtype)) % 16 == 0;
    if (dtype == EBS_F32) return launch_pair<TypedFinal<float>, 2>(A, B, s, {out}, false, packs, st);
    if (dtype == EBS_F16) return launch_pair<TypedFinal<__half>, 2>(A, B, s, {out}, false, packs, st);
    return launch_pair<TypedFinal<__nv_bfloat16>, 2>(A, B, s, {out}, false, packs, st);
}

}  // namespace ebs
