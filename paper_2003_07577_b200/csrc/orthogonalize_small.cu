// Newton-Schulz orthogonalisation of matrices whose short side is at most 128: a cluster of thread blocks a matrix, all steps in one launch.
//
// X stays in shared memory as two fp16 planes, in blocks of 64 columns: [rows][128 bytes] with the 128-byte swizzle; each thread block
// of the cluster has its share of the blocks.  The same bytes are the K-major operands of the Gram product A = X X^T (the reduction runs
// along the rows) and the MN-major operand of X <- Q X (the reduction runs across them), so X is never rearranged.  (The update transposed,
// 128 columns of X on the lanes and X as the MN-major A operand, takes 145 clocks an MMA instead of 70.)
//   per step: the blocks' shares of A meet (each block adds eight columns in turn, in block order, and gives every block their planes);
//             Q = a I + b A + c A A -> planes, in every block;  X <- Q X in place, each block its own columns.
// What bounds it is the chain of dependent phases, not their work: a step of 64 x 576 on eight blocks takes 15000 clocks, of which the MMAs
// with their commits 3500, tensor memory to planes and shares 5500, the two meetings of the cluster 4500.  6 x 64 x 576, five steps: 45 us
// (a thread block a matrix: 58 us; a launch a product: 146 us); 128 x 1152: 89 us (a launch a product: 119 us).
#include "orthogonalize.cuh"

namespace ebs {

static __device__ unsigned long long g_ortho_small_timeouts = 0ull;

constexpr int SMALL_THREADS = 512, SMALL_WARPS = SMALL_THREADS / 32;
constexpr int SMALL_ISSUER = SMALL_WARPS - 2;                     // (up to 64 rows: its lanes of tensor memory hold none)
// Blocks of 64 columns in a thread block: their sums, two a result above 64 rows, fill tensor memory.
__host__ __device__ constexpr int small_blocks(int mp) { return mp > 64 ? 4 : 8; }
constexpr int SMALL_CLUSTER = 8;
constexpr int SMALL_BYTES = 226 * 1024;                           // of dynamic shared memory

struct SmallArgs {
    int rows, cols, tall, m, n, mp, blocks, most, cluster, steps; // mp: m padded to 16; blocks: of 64 columns of X, at most `most` a thread block
    int gram;                                                    // blocks of a Gram sum (the tensor core truncates long sums)
    float eps, first, last;                                      // powers of two of the first X; scale of the result
    unsigned wait_limit;
    int test_flags;
    OrthoFactors f;
};

// Byte of element (row, col) inside a block.
__device__ __forceinline__ uint32_t small_offset(int row, int col) { return (uint32_t)(row * 128 + (((col >> 3) ^ (row & 7)) << 4) + (col & 7) * 2); }
__device__ __forceinline__ uint32_t small_desc(uint32_t smem_addr, uint32_t leading) { return ((smem_addr >> 4) & 0x3FFFu) | ((leading >> 4) << 16); }
__device__ __forceinline__ void store_cluster(uint32_t addr, uint32_t v) { asm volatile("st.shared::cluster.b32 [%0], %1;\n" ::"r"(addr), "r"(v) : "memory"); }

template <typename T>
__global__ void __launch_bounds__(SMALL_THREADS, 1) ortho_small_kernel(const T* __restrict__ g_all, T* __restrict__ out_all, const __grid_constant__ SmallArgs p) {
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ uint64_t done[6];                                  // Gram, Q, four tiles of X
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    __shared__ double sums[SMALL_WARPS], norms[SMALL_CLUSTER];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = (warp & 3) * 32 + lane, group = warp >> 2;
    const int C = p.cluster, rank = (int)(blockIdx.x % C);
    const int mp = p.mp, plane = mp * 128, side = mp > 64 ? 2 * plane : plane;      // bytes of a block; of a plane of A
    const int first = p.blocks * rank / C, blocks = p.blocks * (rank + 1) / C - first;      // of X, here
    const int col0 = first * 64, cols = min(p.n - col0, blocks * 64);
    uint8_t *ah = smem, *al = ah + side;                          // A, later Q
    uint8_t *xh = al + side, *xl = xh + p.most * plane;
    float* shares = reinterpret_cast<float*>(xl + p.most * plane);      // [part][column of this block's][pitch]: sums of A
    const int share_chunks = (mp / 8 + C - 1) / C, pitch = mp + 4;      // eight columns each; their floats (no bank conflicts)
    const long long count = (long long)p.rows * p.cols;
    const T* g = g_all + blockIdx.x / C * count;
    T* out = out_all + blockIdx.x / C * count;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 6; ++i) mbar_init(&done[i], 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    // X to zero: the padding rows and columns stay so
    for (int i = threadIdx.x; i < 2 * p.most * plane / 16; i += SMALL_THREADS) reinterpret_cast<uint4*>(xh)[i] = make_uint4(0u, 0u, 0u, 0u);
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    const uint32_t tmem = uni(tmem_slot);
    let_next_kernel_start();
    wait_for_previous_kernel();

    // |G| in 64 bits, then X = G 2^e / (|G| + eps): two passes over this block's columns of X, eight packs of neighbouring elements of a
    // row of G on their way at a time
    constexpr int N = Pack<T>::N, U = 8;
    const int width = p.cols % N == 0 ? N : 1, per_row = (p.tall ? p.m : cols) / width, items = (p.tall ? cols : p.m) * per_row;
    const T* mine = g + (p.tall ? (long long)col0 * p.m : col0);
    auto each = [&](auto&& use) {                                 // use(row of X, column of X here, elements); tall: of X^T
        for (int i0 = threadIdx.x; i0 < items; i0 += U * SMALL_THREADS) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * SMALL_THREADS;
                if (i < items) raw[u] = load_raw(mine + (long long)(i / per_row) * p.cols + i % per_row * width, width, width == N);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * SMALL_THREADS;
                if (i >= items) break;
                float v[N];
                unpack<T>(raw[u], v);
                use(i / per_row, i % per_row * width, v);
            }
        }
    };
    double s = 0.0;
    each([&](int, int, const float (&v)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < width) s = fma((double)v[e], (double)v[e], s);
    });
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) sums[warp] = s;
    if (C > 1) cluster_sync_all();                                // (every block has started: its memory can be written)
    else __syncthreads();
    if (threadIdx.x < C) {
        s = 0.0;
        for (int i = 0; i < SMALL_WARPS; ++i) s += sums[i];
        asm volatile("st.shared::cluster.f64 [%0], %1;\n" ::"r"(cluster_addr(&norms[rank], threadIdx.x)), "d"(s) : "memory");
    }
    if (C > 1) cluster_sync_all();
    else __syncthreads();
    s = 0.0;
    for (int i = 0; i < C; ++i) s += norms[i];
    const double inv = (double)p.first / (sqrt(s) + (double)p.eps);
    each([&](int r, int c, const float (&v)[N]) {
        __align__(16) uint32_t hi_words[N / 2], lo_words[N / 2];
        const __half *hi = reinterpret_cast<const __half*>(hi_words), *lo = reinterpret_cast<const __half*>(lo_words);
#pragma unroll
        for (int e = 0; e < N; e += 2) split_pair((float)(v[e] * inv), e + 1 < width ? (float)(v[e + 1] * inv) : 0.0f, hi_words[e / 2], lo_words[e / 2]);
        if (width == N && !p.tall) {                              // a pack lies within 16 bytes of a row
            using V = typename std::conditional<N == 8, uint4, uint2>::type;
            const uint32_t at = (c >> 6) * plane + small_offset(r, c & 63);
            *reinterpret_cast<V*>(xh + at) = *reinterpret_cast<const V*>(hi);
            *reinterpret_cast<V*>(xl + at) = *reinterpret_cast<const V*>(lo);
            return;
        }
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (e >= width) break;
            const int to = p.tall ? c + e : r, col = p.tall ? r : c + e;
            const uint32_t at = (col >> 6) * plane + small_offset(to, col & 63);
            *reinterpret_cast<__half*>(xh + at) = hi[e];
            *reinterpret_cast<__half*>(xl + at) = lo[e];
        }
    });

    const uint32_t idesc_sym = uni(gemm_idesc(128, mp, false, false, false));
    const int chunks = (blocks + p.gram - 1) / p.gram;            // Gram sums
    const int x_tiles = (blocks + 1) / 2, k_steps = uni(mp / 16); // (operands of the issuing loops: the same register for all lanes)
    const int parts = mp > 64 ? 2 : 1;                            // sums of a result of Q and of X, over 64 terms each
    const bool rows_here = (warp & 3) * 32 < mp;                  // (whole warps: tensor memory is read by warps)
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    // between phases: what was written by threads, the other blocks' too (all), is seen by the MMAs
    auto phase = [&](bool all) {
        asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
        asm volatile("fence.proxy.async;\n" ::: "memory");
        if (all) {
            cluster_sync_all();
            asm volatile("fence.proxy.async;\n" ::: "memory");
        } else {
            __syncthreads();
        }
        asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    };
    // (a block that gave up takes part in the cluster's barriers to the end)
    auto issues = [&] { return warp == SMALL_ISSUER && (p.test_flags & 1) == 0 && __all_sync(0xffffffffu, abort_flag == 0); };      // (give-up test: nothing is ever issued)
    phase(false);
    for (int step = 0; step < p.steps; ++step) {
        if (issues()) {
            const uint32_t leader = elect_one() ? 1u : 0u;
            // (of each sum the small products first: an MMA truncates at the size of what is there)
            for (int b0 = 0; b0 < blocks; b0 += p.gram) {
                const uint32_t d = uni(tmem + (uint32_t)(b0 / p.gram * mp));
                const int b1 = b0 + p.gram < blocks ? b0 + p.gram : blocks;
                for (int b = b0; b < b1; ++b) {
                    const uint32_t h = uni(small_desc(smem_u32(xh) + b * plane, 16)), l = uni(small_desc(smem_u32(xl) + b * plane, 16));
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        umma_f16(leader, d, h + 2 * k, l + 2 * k, idesc_sym, ((b - b0) | k) != 0);
                        umma_f16(leader, d, l + 2 * k, h + 2 * k, idesc_sym, 1u);
                    }
                }
                for (int b = b0; b < b1; ++b) {
                    const uint32_t h = uni(small_desc(smem_u32(xh) + b * plane, 16));
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_f16(leader, d, h + 2 * k, h + 2 * k, idesc_sym, 1u);
                }
            }
            umma_commit_pred(leader, &done[0]);
        }
        auto side_offset = [&](int r, int c) { return (uint32_t)((c >> 6) * plane) + small_offset(r, c & 63); };
        if (mbar_wait_warp(&done[0], step & 1, &abort_flag, p.wait_limit) && rows_here) {
            asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#pragma unroll 1
            for (int c = group * 16; c < mp; c += 64) {
                __syncwarp();
                float v[2][8] = {};
#pragma unroll 1
                for (int q = 0; q < chunks; q += 2) {             // two sums on their way at once
                    uint32_t t[4][8];
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        if (q + h / 2 < chunks) tmem_ld8_issue(lanes + (q + h / 2) * mp + c + h % 2 * 8, t[h]);
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        if (q + h / 2 < chunks) {
                            tmem_ld8_wait(t[h]);
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[h % 2][i] += __uint_as_float(t[h][i]);
                        }
                }
                if (row >= mp) continue;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int at = c + 8 * h, j = at >> 3;
                    if (C == 1) {
                        uint32_t hi[4], lo[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) split_pair(v[h][2 * i] * p.f.gram[step], v[h][2 * i + 1] * p.f.gram[step], hi[i], lo[i]);
                        *reinterpret_cast<uint4*>(ah + side_offset(row, at)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                        *reinterpret_cast<uint4*>(al + side_offset(row, at)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                    } else {
                        const uint32_t to = cluster_addr(shares + ((rank * share_chunks + j / C) * 8) * pitch + row, j % C);
#pragma unroll
                        for (int i = 0; i < 8; ++i) store_cluster(to + i * pitch * 4, __float_as_uint(v[h][i]));
                    }
                }
            }
        }
        phase(C > 1);
        if (C > 1) {
            const int own = (mp / 8 - rank + C - 1) / C;          // chunks whose number is rank modulo C
            for (int i = threadIdx.x; i < own * mp * 4; i += SMALL_THREADS) {      // two columns of a row, neighbouring lanes 16 bytes of it
                const int j = i / (mp * 4), r = i / 4 - j * mp, e = i % 4 * 2;
                float v0 = 0.0f, v1 = 0.0f;
                const float* from = shares + (j * 8 + e) * pitch + r;
#pragma unroll 4
                for (int q = 0; q < C; ++q, from += share_chunks * 8 * pitch) {
                    v0 += from[0];
                    v1 += from[pitch];
                }
                uint32_t hi, lo;
                split_pair(v0 * p.f.gram[step], v1 * p.f.gram[step], hi, lo);
                const uint32_t at = side_offset(r, (j * C + rank) * 8 + e);
                for (int q = 0; q < C; ++q) {
                    store_cluster(cluster_addr(ah + at, q), hi);
                    store_cluster(cluster_addr(al + at, q), lo);
                }
            }
            phase(true);
        }
        if (issues()) {
            const uint32_t leader = elect_one() ? 1u : 0u;
            const uint32_t h = uni(small_desc(smem_u32(ah), 16)), l = uni(small_desc(smem_u32(al), 16));
            for (int kb = 0; kb < k_steps; kb += 4) {             // a sum for each block of 64 columns
                const uint32_t at = uni(kb * (plane >> 6)), d = uni(tmem + (uint32_t)((kb >> 2) * mp));
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (kb + k >= k_steps) break;
                    umma_f16(leader, d, h + at + 2 * k, l + at + 2 * k, idesc_sym, k != 0);
                    umma_f16(leader, d, l + at + 2 * k, h + at + 2 * k, idesc_sym, 1u);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (kb + k >= k_steps) break;
                    umma_f16(leader, d, h + at + 2 * k, h + at + 2 * k, idesc_sym, 1u);
                }
            }
            umma_commit_pred(leader, &done[1]);
        }
        if (mbar_wait_warp(&done[1], step & 1, &abort_flag, p.wait_limit) && rows_here) {
            asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#pragma unroll 1
            for (int c = group * 16; c < mp; c += 64) {           // Q in A's place
                __syncwarp();
                uint32_t t[4][8];
#pragma unroll
                for (int h = 0; h < 4; ++h)
                    if (h < 2 * parts) tmem_ld8_issue(lanes + h / 2 * mp + c + h % 2 * 8, t[h]);
#pragma unroll
                for (int h = 0; h < 4; ++h)
                    if (h < 2 * parts) tmem_ld8_wait(t[h]);
                if (row >= mp) continue;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (parts == 2)
#pragma unroll
                        for (int i = 0; i < 8; ++i) t[h][i] = __float_as_uint(__uint_as_float(t[h][i]) + __uint_as_float(t[h + 2][i]));
                    const int at = c + 8 * h;
                    uint4 *to_h = reinterpret_cast<uint4*>(ah + side_offset(row, at)), *to_l = reinterpret_cast<uint4*>(al + side_offset(row, at));
                    float vh[8], vl[8], v[8];
                    unpack<__half>(*to_h, vh);
                    unpack<__half>(*to_l, vl);
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        v[i] = fmaf(__uint_as_float(t[h][i]), p.f.quadratic[step], fmaf(vh[i] + vl[i], p.f.direct[step], row == at + i && row < p.m ? p.f.square_diag[step] : 0.0f));
#pragma unroll
                    for (int i = 0; i < 4; ++i) split_pair(v[2 * i], v[2 * i + 1], hi[i], lo[i]);
                    *to_h = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    *to_l = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
            }
        }
        phase(false);
        const bool final = step == p.steps - 1;
        const float factor = final ? p.last : p.f.next[step];
        if (issues()) {                                           // tiles of 128 columns
            const uint32_t leader = elect_one() ? 1u : 0u;
            const uint32_t q_h = uni(small_desc(smem_u32(ah), 16)), q_l = uni(small_desc(smem_u32(al), 16));
            for (int t = 0; t < x_tiles; ++t) {
                const uint32_t idesc_x = uni(gemm_idesc(128, 2 * t + 1 < blocks ? 128 : 64, false, false, true));
                const uint32_t h = uni(small_desc(smem_u32(xh) + 2 * t * plane, plane)), l = uni(small_desc(smem_u32(xl) + 2 * t * plane, plane));
                for (int kb = 0; kb < k_steps; kb += 4) {         // a sum for each 64 rows
                    const uint32_t at = uni(kb * (plane >> 6)), x_at = uni(128 * kb), d = uni(tmem + (uint32_t)((t * parts + (kb >> 2)) * 128));      // (16 rows of a block of X: 2048 bytes)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (kb + k >= k_steps) break;
                        umma_f16(leader, d, q_l + at + 2 * k, h + x_at + 128 * k, idesc_x, k != 0);
                        umma_f16(leader, d, q_h + at + 2 * k, l + x_at + 128 * k, idesc_x, 1u);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (kb + k >= k_steps) break;
                        umma_f16(leader, d, q_h + at + 2 * k, h + x_at + 128 * k, idesc_x, 1u);
                    }
                }
                umma_commit_pred(leader, &done[2 + t]);
            }
        }
        // 32 columns at a time, the groups of four warps take them in turn
        for (int col = group * 32; rows_here && col < cols; col += 128) {
            const int t = col >> 7;
            __syncwarp();
            if (!mbar_wait_warp(&done[2 + t], step & 1, &abort_flag, p.wait_limit)) break;
            asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
            uint32_t raw[32];
            tmem_load<32>(lanes + t * parts * 128 + (col & 127), raw);
            if (parts == 2) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    uint32_t more[8];
                    tmem_ld8(lanes + (t * 2 + 1) * 128 + (col & 127) + q * 8, more);
#pragma unroll
                    for (int i = 0; i < 8; ++i) raw[q * 8 + i] = __float_as_uint(__uint_as_float(raw[q * 8 + i]) + __uint_as_float(more[i]));
                }
            }
            if (row >= p.m) continue;
            if (final) {
                if (p.tall) {                                     // neighbouring lanes write neighbouring elements
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (col + i < cols) out[(long long)(col0 + col + i) * p.m + row] = from_f32<T>(__uint_as_float(raw[i]) * factor);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; i += N) {
                        float v[N];
#pragma unroll
                        for (int e = 0; e < N; ++e) v[e] = __uint_as_float(raw[i + e]) * factor;
                        if (col + i < cols) store_pack(out + (long long)row * p.n + col0 + col + i, v, cols - col - i, p.n % N == 0);
                    }
                }
                continue;
            }
            uint8_t* to = xh + (col >> 6) * plane;
#pragma unroll
            for (int i = 0; i < 32; i += 8) {
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) split_pair(__uint_as_float(raw[i + 2 * e]) * factor, __uint_as_float(raw[i + 2 * e + 1]) * factor, hi[e], lo[e]);
                const uint32_t at = small_offset(row, (col & 63) + i);
                *reinterpret_cast<uint4*>(to + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                *reinterpret_cast<uint4*>(to + p.most * plane + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
        }
        phase(false);
    }
    if (p.steps == 0)                                             // scale X alone
        for (int i = threadIdx.x; i < p.m * cols; i += SMALL_THREADS) {
            const int r = p.tall ? i % p.m : i / cols, c = p.tall ? i / p.m : i % cols;
            const uint32_t at = (c >> 6) * plane + small_offset(r, c & 63);
            out[p.tall ? (long long)(col0 + c) * p.m + r : (long long)r * p.n + col0 + c] =
                from_f32<T>(p.last * (__half2float(*reinterpret_cast<const __half*>(xh + at)) + __half2float(*reinterpret_cast<const __half*>(xl + at))));
        }
    if (abort_flag) {
        giveup_drain();
        if (threadIdx.x == 0) atomicAdd(&g_ortho_small_timeouts, 1ull);
    }
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(512u) : "memory");
}

unsigned long long ortho_small_timeouts() {
    unsigned long long n = 0;
    return cudaMemcpyFromSymbol(&n, g_ortho_small_timeouts, sizeof(n)) == cudaSuccess ? n : 0;
}

// A matrix on a cluster: thread blocks, blocks of columns each at most, and the shared memory they take: A, X, what an operand of 128 rows
// reads behind the last of them or, in the same place, the shares of A.
struct SmallForm {
    int cluster = 0, most = 0;                                    // cluster = 0: does not fit
    size_t bytes = 0;
};
static SmallForm small_form_of(int m, int n, int cluster) {
    const int mp = (m + 15) & ~15, blocks = (n + 63) / 64;
    SmallForm f;
    f.most = (blocks + cluster - 1) / cluster;
    const size_t plane = (size_t)mp * 128, shares = cluster > 1 ? (size_t)cluster * ((mp / 8 + cluster - 1) / cluster) * 8 * (mp + 4) * 4 : 0, behind = (size_t)(128 - mp) * 128;
    f.bytes = 2 * (mp > 64 ? 2 : 1) * plane + 2 * f.most * plane + (shares > behind ? shares : behind);
    if (f.most <= small_blocks(mp) && f.bytes <= SMALL_BYTES && cluster <= blocks) f.cluster = cluster;
    return f;
}
// As many blocks a matrix as run at once (18 clusters of eight no longer do), but two only where one does not hold it: what a half of the
// columns saves, the meeting of the sums costs.  Five steps in clusters of 1, 2, 4, 8: 64 x 576 59, 60, 51, 46 us, 100 x 300 65, 68, 64 us,
// 128 x 128 48, 58 us.
static SmallForm small_form(int batch, int rows, int cols) {
    const int m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    SmallForm best;
    if (m > 128 || n > 64 * small_blocks(m) * SMALL_CLUSTER) return best;
    const int sms = gemm_sm_count();
    for (int c = 1; c <= SMALL_CLUSTER; c *= 2) {
        const SmallForm f = small_form_of(m, n, c);
        if (f.cluster && (!best.cluster || (c != 2 && (long long)batch * c <= (c == 8 ? sms * 3 / 4 : sms)))) best = f;
    }
    return best;
}
bool ortho_small_fits(int rows, int cols) { return small_form(1, rows, cols).cluster != 0; }

template <typename T>
static int launch_small_typed(const void* g, void* out, int batch, const SmallArgs& a, size_t bytes, cudaStream_t st) {
    auto kern = ortho_small_kernel<T>;
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        if (check_cuda(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMALL_BYTES))) return EBS_ERR_CUDA;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    return launch_chained(kern, dim3((unsigned)(batch * a.cluster)), SMALL_THREADS, bytes, st, a.cluster, static_cast<const T*>(g), static_cast<T*>(out), a);
}
int launch_ortho_small(const void* g, void* out, int batch, int rows, int cols, int dtype, int steps, float eps, float first, float last, const OrthoFactors& f, cudaStream_t st) {
    const SmallForm form = small_form(batch, rows, cols);
    SmallArgs a;
    a.rows = rows; a.cols = cols; a.tall = rows > cols;
    a.m = a.tall ? cols : rows;
    a.n = a.tall ? rows : cols;
    a.mp = (a.m + 15) & ~15;
    a.blocks = (a.n + 63) / 64;
    a.most = form.most;
    a.cluster = form.cluster;
    const int sums = 512 / a.mp;                                  // of A that tensor memory has room for
    a.gram = (a.most + sums - 1) / sums;
    a.steps = steps;
    a.eps = eps; a.first = first; a.last = last;
    a.wait_limit = device_wait_limit();
    a.test_flags = device_test_flags();
    a.f = f;
    if (dtype == EBS_F32) return launch_small_typed<float>(g, out, batch, a, form.bytes, st);
    if (dtype == EBS_F16) return launch_small_typed<__half>(g, out, batch, a, form.bytes, st);
    return launch_small_typed<__nv_bfloat16>(g, out, batch, a, form.bytes, st);
}

}  // namespace ebs
