// Layers of experts: products grouped by the rows of each expert, and their gradients.  See include/ebs.h.
//
// One persistent kernel, two forms.  Rows (forward and dx): tiles of rows of one expert x TN outputs, over the reduction of the layer; the last tile
// of an expert reads rows of the next one and leaves them out when it writes.  Weights (dW): tiles of an expert's gradient over the
// expert's own rows; what its last stage holds of other rows is cleared in shared memory before the tensor core reads it.  Offsets are read on the
// device only: a block finds its tiles by scanning them, 32 experts at a time.
//
// PAIR: two thread blocks on two SMs take 256 x 256 results (cta_group::2), each fetches its 128 rows of A and half of the columns of B: 128 x 256 results of
// one block read 192 bytes of shared memory a clock of the tensor core, which has 128 (16384 x 2048 -> 4096 over 16 experts, alone: 240 us, the tensor pipe 68% busy; a pair 220 us, 76%).
// Without: a block takes 128 x 128 or 128 x 64, where there are few tiles.
//
// One warp fetches by TMA, one issues the MMAs, the first 8 (pair: 16) take the sums of the finished tile out of tensor memory while the next one is
// multiplied (two accumulators).  Sums of more than 4096 terms leave the tensor core on the way, which truncates what it adds.  Results go
// through a patch of shared memory, 32 rows at a time, and leave by TMA where all 32 are the expert's; else, and where rows do not start on 16 bytes, neighbouring lanes write
// neighbouring bytes with ordinary stores: a row that is not the expert's is not written.
#include "gemm_tile.cuh"
#include "tensors.cuh"

namespace ebs {

static __device__ unsigned long long g_grouped_timeouts = 0ull;

struct GroupedArgs {
    const int* offsets;
    const void *bias, *residual;
    void *y, *z;
    long long ldy, ldr, ldz, y_expert;     // y_expert: elements between the results of two experts (weights)
    int m, experts, rows, cols, red;       // rows: of a weight gradient
    int tiles_n, b_mn, bf16, act, vec, bias_vec, tma;
    float alpha;
    unsigned wait_limit;
    int test_flags;
};

// The forms: 256 a pair's 256 x 256 results, 128 and 64 so many columns of 128 rows, one and two blocks an SM, FEW_ROWS 64 columns of 32 rows, two blocks an SM with eight stages of
// little more than the weights.  (The tensor core still takes 128 rows: those behind the 32 are whatever lies there, and so are the lanes of sums that nobody reads.)
constexpr int FEW_ROWS = 32;
template <int F> struct GroupedForm {
    static constexpr bool PAIR = F == 256;
    static constexpr int TN = F == FEW_ROWS ? 64 : F;
    static constexpr int A_ROWS = F == FEW_ROWS ? 32 : 128, B_COLS = PAIR ? TN / 2 : TN;             // rows of A and columns of B that a block fetches
    static constexpr int EPI_WARPS = PAIR ? 16 : 8, THREADS = PAIR ? 640 : 320;        // (pair: whole warpgroups, whose registers are dealt anew)
    static constexpr int STAGES = F == FEW_ROWS ? 8 : F == 64 ? 4 : 6, A_BYTES = A_ROWS * GEMM_ROW_BYTES, STAGE = A_BYTES + B_COLS * GEMM_ROW_BYTES;
    static constexpr int CQ = TN / (EPI_WARPS / 4);               // columns of a warp
    static constexpr int PATCH = 32 * 64;                         // 32 rows of 64 bytes
    static constexpr int BARRIERS = 256;
    static constexpr int SMEM = STAGES * STAGE + EPI_WARPS * PATCH + BARRIERS, BLOCKS = TN == 64 ? 2 : 1;
    static constexpr int ROWS = PAIR ? 256 : A_ROWS;              // rows of a tile
    static_assert(B_COLS * GEMM_ROW_BYTES + EPI_WARPS * PATCH >= (128 - A_ROWS) * GEMM_ROW_BYTES, "what the tensor core reads behind the last stage's rows is this block's memory");
};

// Rows of expert e; offsets that are out of order or out of range are taken as the nearest ones that are not.
__device__ __forceinline__ void expert_rows(const int* offsets, int m, int e, int& begin, int& count) {
    begin = min(max(__ldg(offsets + e), 0), m);
    count = min(max(__ldg(offsets + e + 1), begin), m) - begin;
}
struct GroupedTile {
    int expert, a0, a_end, b0;             // first and end row on the lanes, first column
    int red0, red_end;                     // weights: the expert's rows
    int nkb;
};
// The tiles in their order; a warp asks for ever larger ones.
template <bool DW, int ROWS>
struct GroupedTiles {
    int e0 = 0, before = 0;                // tiles of the experts below e0
    __device__ __forceinline__ bool find(const GroupedArgs& g, int t, int tile_cols, GroupedTile& tile) {
        if (DW) {
            const int tiles_m = (g.rows + ROWS - 1) / ROWS, per = tiles_m * g.tiles_n;
            tile.expert = t / per;
            if (tile.expert >= g.experts) return false;
            t -= tile.expert * per;
            int count;
            expert_rows(g.offsets, g.m, tile.expert, tile.red0, count);
            tile.red_end = tile.red0 + count;
            tile.nkb = (count + GEMM_BK - 1) / GEMM_BK;
            tile.a0 = t % tiles_m * ROWS;
            tile.a_end = g.rows;
            tile.b0 = t / tiles_m * tile_cols;
            return true;
        }
        const int lane = threadIdx.x & 31;
        for (; e0 < g.experts; e0 += 32) {
            int begin = 0, count = 0;
            if (e0 + lane < g.experts) expert_rows(g.offsets, g.m, e0 + lane, begin, count);
            const int mine = (count + ROWS - 1) / ROWS * g.tiles_n;
            int sum = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += v;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, t - before < sum);
            if (hit) {
                const int l = __ffs(hit) - 1, in = t - before - __shfl_sync(0xffffffffu, sum - mine, l);
                begin = __shfl_sync(0xffffffffu, begin, l);
                count = __shfl_sync(0xffffffffu, count, l);
                const int tiles_m = (count + ROWS - 1) / ROWS;
                tile.expert = e0 + l;
                // bands of 2048 rows, column by column within a band: the tiles under way at a time share few rows and columns (18944 rows of 4096 that
                // are one expert's, 2048 columns: 249 us row by row of all, whose operand is larger than the second-level cache, 223 so)
                constexpr int BAND = 2048 / ROWS;
                const int band = in / (BAND * g.tiles_n), first = band * BAND, height = min(tiles_m - first, BAND), rest = in - first * g.tiles_n;
                tile.a0 = begin + (first + rest % height) * ROWS;
                tile.a_end = begin + count;
                tile.b0 = rest / height * tile_cols;
                tile.red0 = tile.red_end = 0;
                tile.nkb = (g.red + GEMM_BK - 1) / GEMM_BK;
                return true;
            }
            before += __shfl_sync(0xffffffffu, sum, 31);
        }
        return false;
    }
};

// Chunk c (16 bytes) of row `row` of a patch; rows are 64 bytes, their chunks permuted so that eight lanes' rows meet no bank twice.
__device__ __forceinline__ uint4* patch_chunk(uint8_t* patch, int row, int c) { return reinterpret_cast<uint4*>(patch + row * 64 + ((c ^ ((row >> 1) & 3)) << 4)); }
// 32 values of this lane's row, through the warp's patch, to `rows` rows of 32 columns (`left` of them exist) from `to` on: by one TMA store (map; x, row, z: where)
// where all 32 rows are the expert's or the map ends where they do, else by the lanes.
template <typename T>
__device__ __forceinline__ void store_patch(uint8_t* patch, const float (&v)[32], T* to, long long ld, int rows, int left, bool vec, bool by_tma, const CUtensorMap* map, int x, int row, int z) {
    const int lane = threadIdx.x & 31;
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory");         // what was there is read
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c)
        *patch_chunk(patch, lane, c) =
            make_uint4(pair_word<T>(v[8 * c], v[8 * c + 1]), pair_word<T>(v[8 * c + 2], v[8 * c + 3]), pair_word<T>(v[8 * c + 4], v[8 * c + 5]), pair_word<T>(v[8 * c + 6], v[8 * c + 7]));
    if (by_tma) {
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            tma_store_3d(map, patch, x, row, z);
            tma_store_commit();
        }
        return;
    }
    __syncwarp();
    if (vec && left >= 32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = i * 8 + (lane >> 2), c = lane & 3;
            if (r < rows) *reinterpret_cast<uint4*>(to + r * ld + c * 8) = *patch_chunk(patch, r, c);
        }
    } else if ((ld & 1) == 0) {                                   // two elements a lane, two rows an access
        const int c = (lane & 15) * 2;
#pragma unroll 8
        for (int r = lane >> 4; r < rows; r += 2) {
            const uint32_t* from = reinterpret_cast<const uint32_t*>(patch_chunk(patch, r, c >> 3)) + ((c & 7) >> 1);
            if (c + 1 < left) *reinterpret_cast<uint32_t*>(to + r * ld + c) = *from;
            else if (c < left) to[r * ld + c] = *reinterpret_cast<const T*>(from);
        }
    } else if (lane < left)
#pragma unroll 8
        for (int r = 0; r < rows; ++r) to[r * ld + lane] = reinterpret_cast<const T*>(patch_chunk(patch, r, lane >> 3))[lane & 7];
}

// The other way: this lane's row of 32 columns, fetched by the lanes side by side.
template <typename T>
__device__ __forceinline__ void load_patch(uint8_t* patch, const T* from, long long ld, int rows, int left, bool vec, uint4 (&row)[4]) {
    const int lane = threadIdx.x & 31;
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory");         // what was there is read
    __syncwarp();
    if (vec && left >= 32) {
        uint4 u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i * 8 + (lane >> 2) < rows) u[i] = *reinterpret_cast<const uint4*>(from + (i * 8 + (lane >> 2)) * ld + (lane & 3) * 8);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i * 8 + (lane >> 2) < rows) *patch_chunk(patch, i * 8 + (lane >> 2), lane & 3) = u[i];
    } else if ((ld & 1) == 0) {                                   // two elements a lane, two rows an access, all on their way at once
        const int c = (lane & 15) * 2;
        uint32_t u[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = 2 * i + (lane >> 4);
            u[i] = 0u;
            if (r < rows && c + 1 < left) u[i] = *reinterpret_cast<const uint32_t*>(from + r * ld + c);
            else if (r < rows && c < left) *reinterpret_cast<T*>(&u[i]) = from[r * ld + c];
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = 2 * i + (lane >> 4);
            reinterpret_cast<uint32_t*>(patch_chunk(patch, r, c >> 3))[(c & 7) >> 1] = u[i];
        }
    } else
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
            T u[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) u[i] = h + i < rows && lane < left ? from[(h + i) * ld + lane] : from_f32<T>(0.0f);
#pragma unroll
            for (int i = 0; i < 16; ++i) reinterpret_cast<T*>(patch_chunk(patch, h + i, lane >> 3))[lane & 7] = u[i];
        }
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c) row[c] = *patch_chunk(patch, lane, c);      // (columns and rows that do not exist: whatever is there)
    __syncwarp();
}

// The sums of 32 columns of the warp's rows on their way out: row0 the warp's first row, rows how many it has.
template <typename T, bool DW>
__device__ __forceinline__ void finish_columns(const GroupedArgs& g, const GroupedTile& tile, uint8_t* patch, float (&v)[32], int row0, int rows, int col, int left, const CUtensorMap* map_y,
                                               const CUtensorMap* map_z) {
    const bool by_tma = g.tma && (DW || rows == 32);
    T* y = static_cast<T*>(g.y) + (DW ? tile.expert * g.y_expert : 0) + (long long)row0 * g.ldy + col;
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] *= g.alpha;
    if (!DW) {
        if (g.bias) {
            const T* b = static_cast<const T*>(g.bias) + (long long)tile.expert * g.cols + col;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float t[8];
                unpack<T>(load_raw(b + 8 * c, left - 8 * c, g.bias_vec && left >= 8 * c + 8), t);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[8 * c + i] += t[i];
            }
        }
        if (g.z) store_patch(patch, v, static_cast<T*>(g.z) + (long long)row0 * g.ldz + col, g.ldz, rows, left, g.vec, by_tma, map_z, col, row0, 0);
        switch (g.act) {
#define EBS_ACT_CASE(A) case A: _Pragma("unroll") for (int i = 0; i < 32; ++i) v[i] = activation<true>(v[i], A); break;
            EBS_ACT_CASE(EBS_ACT_RELU) EBS_ACT_CASE(EBS_ACT_GELU) EBS_ACT_CASE(EBS_ACT_GELU_TANH) EBS_ACT_CASE(EBS_ACT_SILU)
#undef EBS_ACT_CASE
            default: break;
        }
        if (g.residual) {
            uint4 r[4];
            load_patch(patch, static_cast<const T*>(g.residual) + (long long)row0 * g.ldr + col, g.ldr, rows, left, g.vec, r);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                float t[8];
                unpack<T>(r[c], t);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[8 * c + i] += t[i];
            }
        }
    }
    store_patch(patch, v, y, g.ldy, rows, left, g.vec, by_tma, map_y, col, row0, DW ? tile.expert : 0);
}

// DW: the form for weight gradients.  CHUNKS: sums leave tensor memory every GEMM_LONG stages and go on in registers.
template <typename T, int F, bool DW, bool CHUNKS>
__global__ void __launch_bounds__(GroupedForm<F>::THREADS, GroupedForm<F>::BLOCKS) grouped_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                                                              const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_z,
                                                                                              const __grid_constant__ GroupedArgs g) {
    extern __shared__ __align__(1024) uint8_t tiles[];            // (nothing static: two blocks' stages take an SM's memory but for a KB)
    using Form = GroupedForm<F>;
    constexpr bool PAIR = Form::PAIR;
    constexpr int TN = Form::TN, S = Form::STAGES, STAGE = Form::STAGE, A_BYTES = Form::A_BYTES, CQ = Form::CQ, EPI = Form::EPI_WARPS;
    static_assert(!DW || Form::A_ROWS == 128, "rows of a weight gradient are its lanes");
    uint64_t* full = reinterpret_cast<uint64_t*>(tiles + S * STAGE + EPI * Form::PATCH);
    uint64_t *empty = full + S, *ready = empty + S, *acc_full = ready + S, *acc_empty = acc_full + 2;
    uint32_t& tmem_slot = *reinterpret_cast<uint32_t*>(acc_empty + 2);
    volatile int& abort_flag = *reinterpret_cast<volatile int*>(acc_empty + 3);
    static_assert((3 * S + 4 + 2) * 8 <= Form::BARRIERS, "barriers");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = PAIR ? (int)(blockIdx.x & 1) : 0, step = PAIR ? (int)(gridDim.x >> 1) : (int)gridDim.x, start = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x;
    if (warp >= EPI && warp < EPI + 2 && lane == 0) asm volatile("prefetch.tensormap [%0];\n" ::"l"(warp == EPI ? &map_a : &map_b) : "memory");
    if (warp == 0 && lane == 0 && g.tma) asm volatile("prefetch.tensormap [%0];\n" ::"l"(&map_y) : "memory");
    if (threadIdx.x == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); mbar_init(&ready[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], PAIR ? 2 * EPI : EPI); }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == EPI + 1) {
        if (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_slot)), "r"(2u * TN) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;\n" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_slot)), "r"(2u * TN) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    __syncthreads();
    if (PAIR) cluster_sync_all();                                 // the partner's barriers are ready too
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    const uint32_t tmem = uni(tmem_slot);
    let_next_kernel_start();
    wait_for_previous_kernel();

    GroupedTiles<DW, Form::ROWS> order;
    GroupedTile tile;
    bool ok = true;
    // Rows of the last stage of a weight gradient that are the expert's; a remainder of 16 (an MMA's depth): the others of those 16 are cleared.
    auto last_rows = [&] { return tile.red_end - tile.red0 - (tile.nkb - 1) * GEMM_BK; };
    if (warp >= EPI) {
      // Pair: registers are dealt anew among the warpgroups: 4 * 128 * 104 + 128 * 56 = 60416 of the 640 * 96 = 61440 the block was launched with.
      if (PAIR) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;\n");
      if (warp == EPI) {
        const bool leader = elect_one();
        int i = 0;                                                // stages filled so far
        for (int t = start; ok && order.find(g, t, TN, tile); t += step) {
            const int a0 = tile.a0 + rank * 128, b0 = tile.b0 + rank * Form::B_COLS;
            const bool tail = PAIR && DW && tile.nkb > 0 && (last_rows() & 15) != 0;
            for (int kb = 0; kb < tile.nkb; ++kb, ++i) {
                const int s = i % S, k = tile.red0 + kb * GEMM_BK;
                ok = mbar_wait_warp(&empty[s], ((i / S) & 1) ^ 1, &abort_flag, g.wait_limit);
                if (!ok) break;
                if (leader) {
                    const uint32_t at = smem_u32(tiles) + s * STAGE, bt = at + A_BYTES;
                    // pair: both blocks' copies report to the first one, but for a last stage that each clears for itself
                    const bool own = !PAIR || (tail && kb == tile.nkb - 1);
                    const uint32_t to = PAIR ? cluster_addr(&full[s], own ? rank : 0) : smem_u32(&full[s]);
                    if (own) mbar_expect_tx(&full[s], STAGE);
                    else if (rank == 0) mbar_expect_tx(&full[s], 2 * STAGE);
                    auto load = [&](uint32_t dst, const CUtensorMap* map, int x, int y, int z) {
                        if (PAIR) tma_load_3d_pair(dst, map, x, y, z, to);
                        else tma_load_3d(dst, map, x, y, z, to);
                    };
                    if (DW) { load(at, &map_a, a0, k, 0); load(at + 8192, &map_a, a0 + 64, k, 0); }
                    else load(at, &map_a, k, a0, 0);
                    if (!DW && !g.b_mn) load(bt, &map_b, k, b0, tile.expert);
                    else
#pragma unroll
                        for (int h = 0; h < Form::B_COLS / 64; ++h) load(bt + h * 8192, &map_b, b0 + h * 64, k, DW ? 0 : tile.expert);
                }
                __syncwarp();
            }
        }
      } else if (warp == EPI + 1 && (rank == 0 || DW)) {          // (the second block of a pair only clears)
        const uint32_t leader = elect_one() ? 1u : 0u;
        const bool b_mn = DW || g.b_mn;
        const uint32_t idesc = gemm_idesc(PAIR ? 256 : 128, TN, g.bf16, DW, b_mn);
        const uint32_t a_step = DW ? 2048 >> 4 : 32 >> 4, b_step = b_mn ? 2048 >> 4 : 32 >> 4;
        int i = 0, c = 0;                                         // stages and accumulators so far
        unsigned cleared = 0u;                                    // bit s: phase of what a pair reports of cleared stages in place s
        for (int t = start; ok && order.find(g, t, TN, tile); t += step) {
            for (int kb = 0, in_chunk = 0; kb < tile.nkb; ++kb, ++i) {
                const int s = i % S;
                uint8_t* stage = tiles + s * STAGE;
                int steps = GEMM_BK / 16, valid = GEMM_BK;
                if (DW && kb == tile.nkb - 1) {
                    valid = last_rows();
                    steps = (valid + 15) / 16;
                }
                const bool tail = DW && (valid & 15) != 0;
                if (rank != 0 && !tail) continue;
                if (rank == 0 && in_chunk == 0 && c >= 2) ok = mbar_wait_cluster_warp(&acc_empty[c & 1], ((c >> 1) & 1) ^ 1, &abort_flag, g.wait_limit);
                // (the second block's barriers count cleared stages alone)
                ok = ok && mbar_wait_warp(&full[s], rank != 0 ? cleared >> s & 1u : (i / S) & 1, &abort_flag, g.wait_limit);
                if (!ok) break;
                if (tail) {                                       // a row is 128 bytes of every block of 64 columns
#pragma unroll
                    for (int b = 0; b < STAGE / 8192; ++b)
                        for (int o = valid * 128 + lane * 16; o < steps * 2048; o += 512) *reinterpret_cast<uint4*>(stage + b * 8192 + o) = make_uint4(0u, 0u, 0u, 0u);
                    asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
                    __syncwarp();
                    if (PAIR) {
                        if (rank == 0) ok = mbar_wait_cluster_warp(&ready[s], cleared >> s & 1u, &abort_flag, g.wait_limit);
                        else if (lane == 0) mbar_arrive_cluster(cluster_addr(&ready[s], 0));
                        cleared ^= 1u << s;
                        if (!ok) break;
                        if (rank != 0) continue;
                    }
                }
                asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                const uint32_t d = tmem + (uint32_t)((c & 1) * TN);
                uint64_t* done = &acc_full[c & 1];
                const int first = in_chunk;
                const bool last = ++in_chunk == (CHUNKS ? GEMM_LONG : tile.nkb) || kb == tile.nkb - 1;
                if (last) { in_chunk = 0; ++c; }
                if (g.test_flags & 1) continue;                   // (give-up test: nothing is ever issued)
                const uint32_t ah = tile_desc_lo(smem_u32(stage), DW), bh = tile_desc_lo(smem_u32(stage) + A_BYTES, b_mn);
#pragma unroll
                for (int k = 0; k < GEMM_BK / 16; ++k)
                    if (k < steps) {
                        if (PAIR) umma_f16_pair(leader, d, ah + k * a_step, bh + k * b_step, idesc, (first | k) != 0);
                        else umma_f16(leader, d, ah + k * a_step, bh + k * b_step, idesc, (first | k) != 0);
                    }
                if (PAIR) {
                    umma_commit_both(leader, cluster_addr(&empty[s], 0), cluster_addr(&empty[s], 1));
                    if (last) umma_commit_both(leader, cluster_addr(done, 0), cluster_addr(done, 1));
                } else {
                    umma_commit_pred(leader, &empty[s]);
                    if (last) umma_commit_pred(leader, done);
                }
            }
        }
      }
    } else {
        if (PAIR) asm volatile("setmaxnreg.inc.sync.aligned.u32 104;\n");
        uint8_t* patch = tiles + S * STAGE + warp * Form::PATCH;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (warp >> 2) * CQ;
        int c = 0;                                                // accumulators so far
        auto taken = [&] {                                        // this warp has its part of accumulator c
            asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if (PAIR) mbar_arrive_cluster(cluster_addr(&acc_empty[c & 1], 0));
                else mbar_arrive(&acc_empty[c & 1]);
            }
        };
        for (int t = start; ok && order.find(g, t, TN, tile); t += step) {
            const int row0 = tile.a0 + rank * 128 + (warp & 3) * 32, rows = min(min(tile.a_end, tile.a0 + Form::ROWS) - row0, 32);
            const int col0 = tile.b0 + (warp >> 2) * CQ;
            auto out = [&](float (&v)[32], int j) {
                const int left = g.cols - col0 - j;
                if (rows > 0 && left > 0) finish_columns<T, DW>(g, tile, patch, v, row0, rows, col0 + j, left, &map_y, &map_z);
            };
            if (CHUNKS) {
                float acc[CQ];
#pragma unroll
                for (int j = 0; j < CQ; ++j) acc[j] = 0.0f;
                for (int kb = 0; kb < tile.nkb && ok; kb += GEMM_LONG, ++c) {
                    ok = mbar_wait_bounded(&acc_full[c & 1], (c >> 1) & 1, &abort_flag, g.wait_limit);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                    if (rows > 0)
#pragma unroll
                        for (int j = 0; j < CQ; j += 32) {
                            uint32_t v[32];
                            tmem_load<32>(lanes + (c & 1) * TN + j, v);
#pragma unroll
                            for (int e = 0; e < 32; ++e) acc[j + e] += __uint_as_float(v[e]);
                        }
                    taken();
                }
                if (!ok) break;
#pragma unroll
                for (int j = 0; j < CQ; j += 32) {
                    float v[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = acc[j + e];
                    out(v, j);
                }
            } else {
                if (tile.nkb > 0) {
                    ok = mbar_wait_bounded(&acc_full[c & 1], (c >> 1) & 1, &abort_flag, g.wait_limit);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                }
#pragma unroll 1
                for (int j = 0; j < CQ; j += 32) {
                    uint32_t raw[32];
                    float v[32];
                    if (tile.nkb > 0) tmem_load<32>(lanes + (c & 1) * TN + j, raw);
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = tile.nkb > 0 ? __uint_as_float(raw[e]) : 0.0f;
                    if (j + 32 == CQ && tile.nkb > 0) taken();    // all sums are in registers: the next tile but one may begin
                    out(v, j);
                }
                c += tile.nkb > 0;
            }
        }
        if (lane == 0) tma_store_wait_all();
    }
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    if (abort_flag) {
        giveup_drain();
        if (threadIdx.x == 0) atomicAdd(&g_grouped_timeouts, 1ull);
    }
    if (PAIR) {
        asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
        cluster_sync_all();                                       // no block leaves while the other's MMAs or arrivals reach it
        if (warp == EPI + 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(2u * TN) : "memory");
    } else {
        __syncthreads();
        if (warp == EPI + 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(2u * TN) : "memory");
    }
}

unsigned long long grouped_timeouts() {
    unsigned long long n = 0;
    return cudaMemcpyFromSymbol(&n, g_grouped_timeouts, sizeof(n)) == cudaSuccess ? n : 0;
}

// ---------------------------------------------------------------------------------------------------- dz and dbias
// dz = dy * act'(z), stored times `store`, and the column sums of dz before its rounding, expert by expert.  A block has 256 columns of a chunk of rows; the
// sums of the part of chunk c that is expert e's go to place c + e (no two parts share one: the next part has the next chunk or a later expert).
struct GroupedDz {
    const void *dy, *z;
    void* dz;
    float* part;
    const int* offsets;
    long long ldy, ldz, lddz;
    int m, n, experts, act, chunk_rows, across, vec;
    float store;
};
template <typename T>
__global__ void __launch_bounds__(256, 4) grouped_dz_kernel(const __grid_constant__ GroupedDz g) {
    __shared__ float sums[8][256 + 4];
    __shared__ int owner[9];
    let_next_kernel_start();
    wait_for_previous_kernel();
    const int bx = (int)(blockIdx.x % (unsigned)g.across), chunk = (int)(blockIdx.x / (unsigned)g.across);
    const int lane = threadIdx.x & 31, y = threadIdx.x >> 5, col = bx * 256 + lane * 8, left = g.n - col;
    const int c0 = chunk * g.chunk_rows, c1 = min(c0 + g.chunk_rows, g.m);
    const T *dy = static_cast<const T*>(g.dy) + col, *z = static_cast<const T*>(g.z) + col;
    T* dz = static_cast<T*>(g.dz) + col;
    const bool vec = g.vec && left >= 8;
    // dz of one row's eight columns, out and left in v
    auto row_dz = [&](const uint4& a, const uint4& b, int r, float (&v)[8]) {
        float zv[8];
        unpack<T>(a, v);
        if (g.act) unpack<T>(b, zv);
        switch (g.act) {
#define EBS_SLOPE_CASE(A) case A: _Pragma("unroll") for (int i = 0; i < 8; ++i) v[i] *= activation_slope<true>(zv[i], A); break;
            EBS_SLOPE_CASE(EBS_ACT_RELU) EBS_SLOPE_CASE(EBS_ACT_GELU) EBS_SLOPE_CASE(EBS_ACT_GELU_TANH) EBS_SLOPE_CASE(EBS_ACT_SILU)
#undef EBS_SLOPE_CASE
            default: break;
        }
        if (!g.dz) return;
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = v[i] * g.store;
        store_pack(dz + r * g.lddz, t);                           // (its rows are padded to whole packs)
    };
    auto part_of = [&](int e, int begin, int end) {
        const int r0 = max(begin, c0), r1 = min(end, c1);
        float sum[8] = {};
        for (int r = r0 + y; r < r1 && left > 0; r += 16) {       // two rows under way
            uint4 a[2], b[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (r + 8 * u < r1) {
                    a[u] = load_raw(dy + (r + 8 * u) * g.ldy, left, vec);
                    if (g.act) b[u] = load_raw(z + (r + 8 * u) * g.ldz, left, vec);
                }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (r + 8 * u >= r1) break;
                float v[8];
                row_dz(a[u], b[u], r + 8 * u, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] += v[i];
            }
        }
        if (!g.part) return;
        __syncthreads();                                          // (the sums before are read)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[y][lane * 8 + i] = sum[i];
        __syncthreads();
        if (bx * 256 + (int)threadIdx.x < g.n) {
            float s = 0.0f;
#pragma unroll
            for (int q = 0; q < 8; ++q) s += sums[q][threadIdx.x];
            g.part[(long long)(chunk + e) * g.n + bx * 256 + threadIdx.x] = s;
        }
    };
    // Chunks of eight rows, where experts have few: a warp a row, whoever's it is (one expert after another, 65 rows of 29 experts of 3060 columns took 33 us).
    const bool by_row = g.chunk_rows == 8;
    if (by_row) {
        if (threadIdx.x < 9) owner[threadIdx.x] = -1;
        __syncthreads();
    }
    for (int e0 = 0; e0 < g.experts; e0 += 32) {
        int begin = 0, count = 0;
        if (e0 + lane < g.experts) expert_rows(g.offsets, g.m, e0 + lane, begin, count);
        unsigned hit = __ballot_sync(0xffffffffu, count > 0 && begin < c1 && begin + count > c0);
        while (hit) {                                             // (the same in every warp)
            const int l = __ffs(hit) - 1;
            hit &= hit - 1;
            const int b = __shfl_sync(0xffffffffu, begin, l), e = b + __shfl_sync(0xffffffffu, count, l);
            if (!by_row) part_of(e0 + l, b, e);
            else if (y == 0 && lane < 8 && c0 + lane >= b && c0 + lane < min(e, c1)) owner[lane] = e0 + l;
        }
    }
    if (!by_row) return;
    __syncthreads();
    float v[8] = {};
    if (owner[y] >= 0 && left > 0) {
        const int r = c0 + y;
        const uint4 a = load_raw(dy + r * g.ldy, left, vec);
        uint4 b = make_uint4(0u, 0u, 0u, 0u);
        if (g.act) b = load_raw(z + r * g.ldz, left, vec);
        row_dz(a, b, r, v);
    }
    if (!g.part) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[y][lane * 8 + i] = v[i];
    __syncthreads();
    if (bx * 256 + (int)threadIdx.x >= g.n) return;
    float s = 0.0f;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        if (owner[q] < 0) continue;
        s += sums[q][threadIdx.x];
        if (owner[q + 1] == owner[q]) continue;
        g.part[(long long)(chunk + owner[q]) * g.n + bx * 256 + threadIdx.x] = s;
        s = 0.0f;
    }
}
// dbias: an expert's chunks in their order, eight warps every eighth.
template <typename T>
__global__ void __launch_bounds__(256) grouped_dbias_kernel(const float* __restrict__ part, const int* __restrict__ offsets, int m, int n, int chunk_rows, int across, T* __restrict__ dbias) {
    __shared__ float sums[8][33];
    let_next_kernel_start();
    wait_for_previous_kernel();
    const int e = (int)(blockIdx.x / (unsigned)across), lane = threadIdx.x & 31, y = threadIdx.x >> 5, col = (int)(blockIdx.x % (unsigned)across) * 32 + lane;
    int begin, count;
    expert_rows(offsets, m, e, begin, count);
    float s = 0.0f;
    if (count > 0 && col < n) {
        const int last = (begin + count - 1) / chunk_rows;
#pragma unroll 4
        for (int c = begin / chunk_rows + y; c <= last; c += 8) s += part[(long long)(c + e) * n + col];
    }
    sums[y][lane] = s;
    __syncthreads();
    if (y == 0 && col < n) {
        for (int q = 1; q < 8; ++q) s += sums[q][lane];
        dbias[(long long)e * n + col] = from_f32<T>(s);
    }
}

// ---------------------------------------------------------------------------------------------------- the calls
struct GroupedOperand {
    const void* p;
    long long ld, expert;                  // elements between rows, between experts
};
// A 16-bit matrix as TMA wants it, copied to rows of whole 16 bytes where its own do not start on them.
static GroupedOperand plan_rows(const void* p, long long rows, int cols, long long ld, Carver& ws, CopyJobs* jobs) {
    if ((ld & 7) == 0) return {p, ld, 0};
    const long long ldd = round8(cols);
    void* to = ws.take<uint16_t>((size_t)rows * ldd);
    if (p && to && rows > 0) add_copy_rows(jobs, p, to, rows, cols, ld, ldd);
    return {to, ldd, 0};
}

template <typename T, int F, bool DW, bool CHUNKS>
static int launch_grouped(const CUtensorMap (&map)[4], const GroupedArgs& g, long long tiles, cudaStream_t st) {
    using Form = GroupedForm<F>;
    auto kern = grouped_kernel<T, F, DW, CHUNKS>;
    constexpr int SMEM = Form::SMEM;
    static_assert(Form::BLOCKS * (SMEM + 1024) <= 228 * 1024 && SMEM <= 227 * 1024, "shared memory of an SM: the blocks' and 1 KB that each takes besides");
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        if (check_cuda(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM))) return EBS_ERR_CUDA;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    constexpr int cluster = Form::PAIR ? 2 : 1;
    const long long at_once = (long long)gemm_sm_count() * Form::BLOCKS / cluster;
    return launch_chained(kern, dim3((unsigned)(cluster * (tiles < at_once ? tiles : at_once))), Form::THREADS, (size_t)SMEM, st, cluster, map[0], map[1], map[2], map[3], g);
}
// Tiles of `tile` rows there can be at most: one more than whole ones for each expert that has rows; and how many there are where all have the same number.
static long long most_row_tiles(int m, int experts, int tile) { return m / tile + (experts < m ? experts : m); }
static long long expected_row_tiles(int m, int experts, int tile) {
    const long long e = experts < m ? experts : m;
    return e * ((m / e + tile - 1) / tile);
}
// The form that ends first.  us a stage of 64 terms: of a tile alone on its SM (or pair), and of an SM's where two share it; and for a tile's results.  row_tiles(rows): tiles of that many.
// FEW_ROWS where experts have few (it is bound by the weights' bytes then), or where the others leave SMs without a tile.
template <class F>
static int grouped_form(const F& row_tiles, int cols, long long stages, bool weights, bool few_rows) {
    struct { int form, rows, cols, blocks; float stage, shared; } const forms[] = {
        {256, 256, 256, 74, 0.30f, 0.30f}, {128, 128, 128, 148, 0.18f, 0.18f}, {64, 128, 64, 296, 0.26f, 0.30f}, {FEW_ROWS, FEW_ROWS, 64, 296, 0.14f, 0.24f}};
    if (few_rows) return FEW_ROWS;
    int best = 64;
    float least = 0.0f;
    for (const auto& f : forms) {
        const long long tiles = row_tiles(f.rows) * ((cols + f.cols - 1) / f.cols);
        if (f.form == FEW_ROWS && (weights || tiles > 296)) continue;
        const float time = (float)((tiles + f.blocks - 1) / f.blocks) * ((float)stages * (tiles > 148 ? f.shared : f.stage) + 1.5f);
        if (least == 0.0f || time < least) { least = time; best = f.form; }
    }
    return best;
}
// row_tiles: of the form that was chosen.
template <typename T, bool DW>
static int launch_form(int form, const GemmOperand& a, int a_mn, int a_red, const GemmOperand& b, int b_cols, int b_red, int batch, GroupedArgs& g, long long row_tiles, bool chunks, cudaStream_t st) {
    CUtensorMap map[4] = {};
    const bool bf16 = std::is_same<T, __nv_bfloat16>::value;
    const int tn = form == FEW_ROWS ? 64 : form;
    if (!gemm_operand_map(a, a_mn, a_red, 1, form == FEW_ROWS ? FEW_ROWS : 128, bf16, &map[0]) || !gemm_operand_map(b, b_cols, b_red, batch, tn == 256 ? 128 : tn, bf16, &map[1])) return EBS_ERR_CUDA;
    g.bf16 = bf16;
    g.tma = DW ? result_map<T>(g.y, g.rows, g.cols, g.ldy, g.experts, g.y_expert, &map[2])
               : result_map<T>(g.y, g.m, g.cols, g.ldy, 1, 0, &map[2]) && result_map<T>(g.z, g.m, g.cols, g.ldz, 1, 0, &map[3]);
    g.tiles_n = (g.cols + tn - 1) / tn;
    g.wait_limit = device_wait_limit();
    g.test_flags = device_test_flags();
    const long long tiles = row_tiles * g.tiles_n;
    if (tiles >= (1LL << 30)) return EBS_ERR_OVERFLOW;
    switch (form) {
        case 256: return chunks ? launch_grouped<T, 256, DW, true>(map, g, tiles, st) : launch_grouped<T, 256, DW, false>(map, g, tiles, st);
        case 128: return chunks ? launch_grouped<T, 128, DW, true>(map, g, tiles, st) : launch_grouped<T, 128, DW, false>(map, g, tiles, st);
        case FEW_ROWS:
            if constexpr (!DW) return chunks ? launch_grouped<T, FEW_ROWS, DW, true>(map, g, tiles, st) : launch_grouped<T, FEW_ROWS, DW, false>(map, g, tiles, st);
            return EBS_ERR_UNSUPPORTED;
        default: return chunks ? launch_grouped<T, 64, DW, true>(map, g, tiles, st) : launch_grouped<T, 64, DW, false>(map, g, tiles, st);
    }
}
struct GroupedTensors {
    const void *x, *w, *bias, *residual, *dy, *z;
    void *y, *keep, *dx, *dw, *dbias;
    const int* offsets;
};
template <typename T>
static int rows_product(const GroupedTensors& t, int m, int experts, int cols, int red, const GroupedOperand& a, const GroupedOperand& w, bool b_mn, GroupedArgs& g, cudaStream_t st) {
    g.offsets = t.offsets;
    g.m = m;
    g.experts = experts;
    g.cols = cols;
    g.red = red;
    g.b_mn = b_mn;
    GemmOperand A(a.p, a.ld, false), B(w.p, w.ld, b_mn, 1, 0, w.expert);
    const bool chunks = red > GEMM_LONG * GEMM_BK;
    const int form = grouped_form([&](int rows) { return expected_row_tiles(m, experts, rows); }, cols, (red + GEMM_BK - 1) / GEMM_BK, false,
                                  m <= FEW_ROWS * (long long)(experts < m ? experts : m));
    return launch_form<T, false>(form, A, m, red, B, cols, red, experts, g, most_row_tiles(m, experts, form == 256 ? 256 : form == FEW_ROWS ? FEW_ROWS : 128), chunks, st);
}
static bool rows_ok(const void* p, long long ld) { return !p || (ld & 7) == 0; }

template <typename T>
static int grouped_forward(const ebs_linear_desc& d, int experts, const GroupedTensors& t, Carver& ws, bool run, cudaStream_t st) {
    if (d.m == 0) return EBS_OK;
    CopyJobs copies = {};
    const GroupedOperand x = plan_rows(t.x, d.m, d.k, d.ldx, ws, &copies);
    GroupedOperand w = plan_rows(t.w, (long long)experts * d.n, d.k, d.ldw, ws, &copies);
    w.expert = d.n * w.ld;
    if (!run) return EBS_OK;
    const int rc = launch_copies(copies, st);
    if (rc) return rc;
    GroupedArgs g = {};
    g.bias = t.bias; g.residual = t.residual; g.y = t.y; g.z = t.keep;
    g.ldy = d.ldy; g.ldr = d.ldr; g.ldz = d.ldz;
    g.act = d.act;
    g.alpha = 1.0f;
    g.vec = rows_ok(t.y, d.ldy) && rows_ok(t.keep, d.ldz) && rows_ok(t.residual, d.ldr);
    g.bias_vec = d.n % 8 == 0;
    return rows_product<T>(t, d.m, experts, d.n, d.k, x, w, false, g, st);
}
template <typename T>
static int grouped_backward(const ebs_linear_desc& d, int experts, const GroupedTensors& t, Carver& ws, bool run, cudaStream_t st) {
    if (d.m == 0) {
        if (!run) return EBS_OK;
        if (t.dw && check_cuda(cudaMemset2DAsync(t.dw, d.ldw * 2, 0, (size_t)d.k * 2, (size_t)experts * d.n, st))) return EBS_ERR_CUDA;
        if (t.dbias && check_cuda(cudaMemsetAsync(t.dbias, 0, (size_t)experts * d.n * 2, st))) return EBS_ERR_CUDA;
        return EBS_OK;
    }
    CopyJobs copies = {};
    GroupedOperand dz;
    void* stored = nullptr;
    if (d.act) {
        dz = GroupedOperand{stored = ws.take<uint16_t>((size_t)d.m * round8(d.n)), round8(d.n), 0};
        if (run && !t.dx && !t.dw) stored = nullptr;
    } else dz = plan_rows(t.dx || t.dw || !run ? t.dy : nullptr, d.m, d.n, d.ldy, ws, &copies);
    const GroupedOperand x = plan_rows(t.dw || !run ? t.x : nullptr, d.m, d.k, d.ldx, ws, &copies);
    GroupedOperand w = plan_rows(t.dx || !run ? t.w : nullptr, (long long)experts * d.n, d.k, d.ldw, ws, &copies);
    w.expert = d.n * w.ld;
    const int across = (d.n + 255) / 256;
    const long long want = (8LL * 148 + across - 1) / across, share = (d.m + want - 1) / want;        // about eight blocks an SM, at least 32 rows each, or eight
    const int chunk_rows = share <= 8 && (d.m < 32LL * experts || (d.m + 31) / 32 * across < 148) ? 8 : (int)(share > 32 ? share : 32), chunks = (d.m + chunk_rows - 1) / chunk_rows;
    float* part = ws.take<float>(((size_t)chunks + experts) * d.n);
    if (!run) return EBS_OK;
    int rc;
    if (stored || t.dbias) {
        if ((long long)chunks * across > 0x7fffffffLL || (long long)experts * ((d.n + 31) / 32) > 0x7fffffffLL) return EBS_ERR_OVERFLOW;
        GroupedDz g{t.dy, t.z, stored, t.dbias ? part : nullptr, t.offsets, d.ldy, d.ldz, round8(d.n), d.m, d.n, experts, d.act, chunk_rows, across,
                    (d.ldy & 7) == 0 && (!d.act || (d.ldz & 7) == 0), dz_store_scale(d)};
        if ((rc = launch_chained(grouped_dz_kernel<T>, dim3((unsigned)(chunks * across)), 256, 0, st, 1, g))) return rc;
        if (t.dbias && (rc = launch_chained(grouped_dbias_kernel<T>, dim3((unsigned)(experts * ((d.n + 31) / 32))), 256, 0, st, 1, (const float*)part, t.offsets, d.m, d.n, chunk_rows,
                                            (d.n + 31) / 32, static_cast<T*>(t.dbias))))
            return rc;
    }
    if ((rc = launch_copies(copies, st))) return rc;
    if (t.dx) {
        GroupedArgs g = {};
        g.y = t.dx;
        g.ldy = d.ldx;
        g.alpha = 1.0f / dz_store_scale(d);
        g.vec = rows_ok(t.dx, d.ldx);
        if ((rc = rows_product<T>(t, d.m, experts, d.k, d.n, dz, w, true, g, st))) return rc;
    }
    if (t.dw) {
        GroupedArgs g = {};
        g.offsets = t.offsets;
        g.m = d.m;
        g.experts = experts;
        g.rows = d.n;
        g.cols = d.k;
        g.y = t.dw;
        g.ldy = d.ldw;
        g.y_expert = d.n * d.ldw;
        g.alpha = 1.0f / dz_store_scale(d);
        g.vec = rows_ok(t.dw, d.ldw);
        const auto row_tiles = [&](int rows) { return (long long)experts * ((d.n + rows - 1) / rows); };
        const int form = grouped_form(row_tiles, d.k, ((d.m + experts - 1) / experts + GEMM_BK - 1) / GEMM_BK, true, false);
        GemmOperand A(dz.p, dz.ld, true), B(x.p, x.ld, true);
        const bool chunks = d.m > GEMM_LONG * GEMM_BK;
        if ((rc = launch_form<T, true>(form, A, d.n, d.m, B, d.k, d.m, 1, g, row_tiles(form == 256 ? 256 : 128), chunks, st))) return rc;
    }
    return EBS_OK;
}

// The descriptor of a layer of experts, strides filled in.
static int complete_grouped(const ebs_linear_desc* in, int experts, ebs_linear_desc* d) {
    const int rc = complete_linear(in, d);
    if (rc) return rc;
    if (experts < 1) return EBS_ERR_INVALID_ARG;
    if (d->dtype == EBS_F32) return EBS_ERR_UNSUPPORTED;
    if ((double)experts * d->n * (double)d->ldw > (double)(1LL << 40) || (long long)experts * d->n > (1LL << 31) || d->m > (1 << 30) - 128) return EBS_ERR_OVERFLOW;
    return EBS_OK;
}
static size_t grouped_workspace(const ebs_linear_desc& d, int experts, bool back) {
    Carver count{nullptr};
    const GroupedTensors none{};
    if (back) grouped_backward<__half>(d, experts, none, count, false, nullptr);
    else grouped_forward<__half>(d, experts, none, count, false, nullptr);
    return count.used;
}
// Whether the offsets lie apart from what the call writes.
static bool offsets_apart(const int* offsets, int experts, const Rows* t, int count, size_t size) {
    const uintptr_t o = (uintptr_t)offsets, oe = o + ((size_t)experts + 1) * 4;
    for (int i = 0; i < count; ++i) {
        if (!t[i].out || !t[i].p || t[i].rows <= 0) continue;
        const uintptr_t p = (uintptr_t)t[i].p;
        if (o < p + ((size_t)(t[i].rows - 1) * t[i].ld + t[i].cols) * size && p < oe) return false;
    }
    return true;
}

}  // namespace ebs

using namespace ebs;

extern "C" {

size_t ebs_grouped_workspace_bytes(const ebs_linear_desc* desc, int experts, int backward) {
    ebs_linear_desc d;
    if (complete_grouped(desc, experts, &d)) return 0;
    return grouped_workspace(d, experts, backward != 0);
}

int ebs_grouped_forward(const void* x_dev, const void* w_dev, const void* bias_dev, const void* residual_dev, const int* offsets_dev, int experts, const ebs_linear_desc* desc, void* y_dev,
                        void* z_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
    ebs_linear_desc d;
    const int rc = complete_grouped(desc, experts, &d);
    if (rc) return rc;
    if (!w_dev || !offsets_dev || ((uintptr_t)offsets_dev & 3u) || (d.m > 0 && (!x_dev || !y_dev))) return EBS_ERR_INVALID_ARG;
    const size_t need = grouped_workspace(d, experts, false);
    if (need && (!workspace_dev || workspace_bytes < need)) return EBS_ERR_INVALID_ARG;
    const long long all = (long long)experts * d.n;
    const Rows t[] = {{x_dev, d.m, d.k, d.ldx, false}, {w_dev, all, d.k, d.ldw, false}, {bias_dev, 1, all, all, false}, {residual_dev, d.m, d.n, d.ldr, false},
                      {y_dev, d.m, d.n, d.ldy, true}, {z_dev, d.m, d.n, d.ldz, true}, {need ? workspace_dev : nullptr, 1, (long long)(need / 2), (long long)(need / 2), true}};
    if (check_tensors(t, 7, 2, &t[3], &t[4]) || !offsets_apart(offsets_dev, experts, t, 7, 2)) return EBS_ERR_INVALID_ARG;
    Carver ws{static_cast<char*>(workspace_dev)};
    const GroupedTensors all_t{x_dev, w_dev, bias_dev, residual_dev, nullptr, nullptr, y_dev, z_dev, nullptr, nullptr, nullptr, offsets_dev};
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return d.dtype == EBS_F16 ? grouped_forward<__half>(d, experts, all_t, ws, true, st) : grouped_forward<__nv_bfloat16>(d, experts, all_t, ws, true, st);
}

int ebs_grouped_backward(const void* dy_dev, const void* x_dev, const void* w_dev, const void* z_dev, const int* offsets_dev, int experts, const ebs_linear_desc* desc, void* dx_dev,
                         void* dw_dev, void* dbias_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
    ebs_linear_desc d;
    const int rc = complete_grouped(desc, experts, &d);
    if (rc) return rc;
    if (!dx_dev && !dw_dev && !dbias_dev && d.m > 0) return EBS_ERR_INVALID_ARG;
    if (!offsets_dev || ((uintptr_t)offsets_dev & 3u)) return EBS_ERR_INVALID_ARG;
    if (d.m > 0 && (!dy_dev || (dx_dev && !w_dev) || (dw_dev && !x_dev) || (d.act && !z_dev))) return EBS_ERR_INVALID_ARG;
    const size_t need = grouped_workspace(d, experts, true);
    if (need && (!workspace_dev || workspace_bytes < need)) return EBS_ERR_INVALID_ARG;
    const long long all = (long long)experts * d.n;
    const Rows t[] = {{dy_dev, d.m, d.n, d.ldy, false}, {x_dev, d.m, d.k, d.ldx, false}, {w_dev, all, d.k, d.ldw, false}, {d.act ? z_dev : nullptr, d.m, d.n, d.ldz, false},
                      {dx_dev, d.m, d.k, d.ldx, true}, {dw_dev, all, d.k, d.ldw, true}, {dbias_dev, 1, all, all, true},
                      {need ? workspace_dev : nullptr, 1, (long long)(need / 2), (long long)(need / 2), true}};
    if (check_tensors(t, 8, 2, nullptr, nullptr) || !offsets_apart(offsets_dev, experts, t, 8, 2)) return EBS_ERR_INVALID_ARG;
    Carver ws{static_cast<char*>(workspace_dev)};
    const GroupedTensors all_t{x_dev, w_dev, nullptr, nullptr, dy_dev, z_dev, nullptr, nullptr, dx_dev, dw_dev, dbias_dev, offsets_dev};
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return d.dtype == EBS_F16 ? grouped_backward<__half>(d, experts, all_t, ws, true, st) : grouped_backward<__nv_bfloat16>(d, experts, all_t, ws, true, st);
}

}  // extern "C"
