// Newton-Schulz orthogonalisation of small matrices: one thread block a matrix, all steps in one launch.
//
// X (short side at most 64) stays in shared memory as two fp16 planes, in blocks of 64 columns: [rows][128 bytes] with the 128-byte swizzle.
// The same bytes are the K-major operands of the Gram product A = X X^T (the reduction runs along the rows) and the MN-major operand of
// X <- Q X (the reduction runs across them), so X is never rearranged.  (The update transposed, 128 columns of X on the lanes and X as the
// MN-major A operand, takes 145 clocks an MMA instead of 70.)
//   per step: A, b I + c A -> planes;  Q = a I + A (b I + c A) -> planes;  X <- Q X in place, block by block.
// What bounds it is the chain of dependent phases (about a microsecond each for commit, tensor memory, planes), not their work.
#include "orthogonalize.cuh"

namespace ebs {

static __device__ unsigned long long g_ortho_small_timeouts = 0ull;

constexpr int SMALL_THREADS = 512, SMALL_WARPS = SMALL_THREADS / 32;
constexpr int SMALL_ISSUER = SMALL_WARPS - 2;                     // a warp whose lanes of tensor memory hold no rows
constexpr int SMALL_GRAM_COLS = 192, SMALL_Q_COL = 192;         // tensor memory: Gram chunks and Q; then four tiles of X over all of it

struct SmallArgs {
    int rows, cols, tall, m, n, mp, blocks, steps;                // mp: m padded to 16; blocks: of 64 columns of X
    float eps, first, last;                                      // powers of two of the first X; scale of the result
    unsigned wait_limit;
    int test_flags;
    OrthoFactors f;
};

// Byte of element (row, col) inside a block.
__device__ __forceinline__ uint32_t small_offset(int row, int col) { return (uint32_t)(row * 128 + (((col >> 3) ^ (row & 7)) << 4) + (col & 7) * 2); }
__device__ __forceinline__ uint32_t small_desc(uint32_t smem_addr, uint32_t leading) { return ((smem_addr >> 4) & 0x3FFFu) | ((leading >> 4) << 16); }

template <typename T>
__global__ void __launch_bounds__(SMALL_THREADS, 1) ortho_small_kernel(const T* __restrict__ g_all, T* __restrict__ out_all, const __grid_constant__ SmallArgs p) {
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ uint64_t done[6], freed[4];                       // Gram, Q, four places of tiles of X
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    __shared__ double sums[SMALL_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int mp = p.mp, plane = mp * 128;                        // bytes of a block
    uint8_t *ah = smem, *al = ah + plane, *lh = al + plane, *ll = lh + plane;      // A (later Q) and b I + c A
    uint8_t *xh = ll + plane, *xl = xh + p.blocks * plane;
    const long long count = (long long)p.rows * p.cols;
    const T* g = g_all + blockIdx.x * count;
    T* out = out_all + blockIdx.x * count;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 6; ++i) mbar_init(&done[i], 1);
        for (int i = 0; i < 4; ++i) mbar_init(&freed[i], (mp + 31) / 32);     // (the warps that have rows)
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
    }
    // everything to zero: the padding rows and columns stay so
    for (int i = threadIdx.x; i < (4 + 2 * p.blocks) * plane / 16; i += SMALL_THREADS) reinterpret_cast<uint4*>(smem)[i] = make_uint4(0u, 0u, 0u, 0u);
    asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
    const uint32_t tmem = uni(tmem_slot);
    let_next_kernel_start();
    wait_for_previous_kernel();

    // |G| in 64 bits, then X = G 2^e / (|G| + eps): two passes, eight packs of neighbouring elements of a row on their way at a time
    constexpr int N = Pack<T>::N, U = 8;
    const int width = p.cols % N == 0 ? N : 1, per_row = p.cols / width, items = p.rows * per_row;
    auto each = [&](auto&& use) {                                 // use(row of G, column, elements, how many)
        for (int i0 = threadIdx.x; i0 < items; i0 += U * SMALL_THREADS) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * SMALL_THREADS;
                if (i < items) raw[u] = load_raw(g + (long long)i * width, width, width == N);
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
    __syncthreads();
    s = 0.0;
    for (int i = 0; i < SMALL_WARPS; ++i) s += sums[i];
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
            const int row = p.tall ? c + e : r, col = p.tall ? r : c + e;
            const uint32_t at = (col >> 6) * plane + small_offset(row, col & 63);
            *reinterpret_cast<__half*>(xh + at) = hi[e];
            *reinterpret_cast<__half*>(xl + at) = lo[e];
        }
    });

    const uint32_t idesc_sym = uni(gemm_idesc(128, mp, false, false, false));
    const int chunks = (p.blocks + 3) / 4;                        // Gram sums of 256 columns each: the tensor core truncates long sums
    const int x_tiles = (p.blocks + 1) / 2, k_steps = uni(mp / 16);      // (operands of the issuing loops: the same register for all lanes)
    // planes of a symmetric matrix's rows: factor * v + diag on the diagonal (8 columns from col on)
    auto put = [&](uint8_t* hi_plane, uint8_t* lo_plane, int row, int col, const float (&v)[8], float factor, float diag) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            split_pair(v[2 * i] * factor + (row == col + 2 * i ? diag : 0.0f), v[2 * i + 1] * factor + (row == col + 2 * i + 1 ? diag : 0.0f), hi[i], lo[i]);
        *reinterpret_cast<uint4*>(hi_plane + small_offset(row, col)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4*>(lo_plane + small_offset(row, col)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    };
    // between phases: what was written by threads is seen by the MMAs
    auto phase = [&] {
        asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
        __syncthreads();
        asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
        return abort_flag == 0;
    };
    const bool issues = warp == SMALL_ISSUER && (p.test_flags & 1) == 0;      // (give-up test: nothing is ever issued)
    bool ok = phase();
    for (int step = 0; step < p.steps && ok; ++step) {
        if (issues) {
            const uint32_t leader = elect_one() ? 1u : 0u;
            // (of each sum the small products first: an MMA truncates at the size of what is there)
            for (int b0 = 0; b0 < p.blocks; b0 += 4) {
                const uint32_t d = uni(tmem + (uint32_t)((b0 >> 2) * mp));
                const int b1 = b0 + 4 < p.blocks ? b0 + 4 : p.blocks;
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
        const int row = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const bool rows_here = (warp & 3) * 32 < mp;              // (whole warps: tensor memory is read by warps)
        if (mbar_wait_warp(&done[0], step & 1, &abort_flag, p.wait_limit) && rows_here) {
            asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#pragma unroll 1
            for (int c = (warp >> 2) * 8; c < mp; c += SMALL_WARPS * 2) {
                float v[8] = {};
#pragma unroll 1
                for (int q0 = 0; q0 < chunks; q0 += 4) {          // four chunks on their way at once
                    uint32_t t[4][8];
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (q0 + q < chunks) tmem_ld8_issue(lanes + (q0 + q) * mp + c, t[q]);
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (q0 + q < chunks) {
                            tmem_ld8_wait(t[q]);
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] += __uint_as_float(t[q][i]);
                        }
                }
                if (row < mp) {
                    put(ah, al, row, c, v, p.f.gram[step], 0.0f);
                    put(lh, ll, row, c, v, p.f.linear[step], row < p.m ? p.f.linear_diag[step] : 0.0f);
                }
            }
        }
        if (!(ok = phase())) break;
        if (issues) {
            const uint32_t leader = elect_one() ? 1u : 0u;
            const uint32_t a_h = uni(small_desc(smem_u32(ah), 16)), a_l = uni(small_desc(smem_u32(al), 16)), l_h = uni(small_desc(smem_u32(lh), 16)), l_l = uni(small_desc(smem_u32(ll), 16));
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k >= k_steps) break;
                umma_f16(leader, tmem + SMALL_Q_COL, a_h + 2 * k, l_l + 2 * k, idesc_sym, k != 0);
                umma_f16(leader, tmem + SMALL_Q_COL, a_l + 2 * k, l_h + 2 * k, idesc_sym, 1u);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k >= k_steps) break;
                umma_f16(leader, tmem + SMALL_Q_COL, a_h + 2 * k, l_h + 2 * k, idesc_sym, 1u);
            }
            umma_commit_pred(leader, &done[1]);
        }
        if (mbar_wait_warp(&done[1], step & 1, &abort_flag, p.wait_limit) && rows_here) {
            asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#pragma unroll 1
            for (int c = (warp >> 2) * 8; c < mp; c += SMALL_WARPS * 2) {
                uint32_t t[8];
                float v[8];
                tmem_ld8(lanes + SMALL_Q_COL + c, t);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(t[i]);
                if (row < mp) put(ah, al, row, c, v, p.f.square[step], row < p.m ? p.f.square_diag[step] : 0.0f);      // Q in A's place
            }
        }
        if (!(ok = phase())) break;
        const bool final = step == p.steps - 1;
        const float factor = final ? p.last : p.f.next[step];
        // tiles of 128 columns in four places of tensor memory, a group of four warps each; the issuing warp runs ahead
        auto uses = [&](int place) { return step * ((x_tiles - place + 3) / 4); };       // of a place in the steps before
        if (issues) {
            const uint32_t leader = elect_one() ? 1u : 0u;
            const uint32_t q_h = uni(small_desc(smem_u32(ah), 16)), q_l = uni(small_desc(smem_u32(al), 16));
            for (int t = 0; t < x_tiles; ++t) {
                const int place = t & 3;
                if (t >= 4 && !mbar_wait_warp(&freed[place], (uses(place) + t / 4 - 1) & 1, &abort_flag, p.wait_limit)) break;
                asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
                const uint32_t idesc_x = uni(gemm_idesc(128, 2 * t + 1 < p.blocks ? 128 : 64, false, false, true));
                const uint32_t d = uni(tmem + place * 128);
                const uint32_t h = uni(small_desc(smem_u32(xh) + 2 * t * plane, plane)), l = uni(small_desc(smem_u32(xl) + 2 * t * plane, plane));
#pragma unroll
                for (int k = 0; k < 4; ++k) {                     // 16 rows of a block: 2048 bytes
                    if (k >= k_steps) break;
                    umma_f16(leader, d, q_l + 2 * k, h + 128 * k, idesc_x, k != 0);
                    umma_f16(leader, d, q_h + 2 * k, l + 128 * k, idesc_x, 1u);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (k >= k_steps) break;
                    umma_f16(leader, d, q_h + 2 * k, h + 128 * k, idesc_x, 1u);
                }
                umma_commit_pred(leader, &done[2 + place]);
            }
        }
        // (only the warps that free a place follow its barrier: it may be rounds ahead of any other)
        const int place = warp >> 2;
        for (int t = place; rows_here && t < x_tiles; t += 4) {
            if (!mbar_wait_warp(&done[2 + place], (uses(place) + t / 4) & 1, &abort_flag, p.wait_limit)) break;
            asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory");
#pragma unroll 1
            for (int col = t * 128; col < t * 128 + 128 && col < p.n; col += 32) {
                uint32_t raw[32];
                tmem_load<32>(lanes + place * 128 + (col & 127), raw);
                if (row >= p.m) continue;
                if (final) {
                    if (p.tall) {                                 // neighbouring lanes write neighbouring elements
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (col + i < p.n) out[(long long)(col + i) * p.m + row] = from_f32<T>(__uint_as_float(raw[i]) * factor);
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; i += N) {
                            float v[N];
#pragma unroll
                            for (int e = 0; e < N; ++e) v[e] = __uint_as_float(raw[i + e]) * factor;
                            if (col + i < p.n) store_pack(out + (long long)row * p.n + col + i, v, p.n - col - i, p.n % N == 0);
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
                    *reinterpret_cast<uint4*>(to + p.blocks * plane + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&freed[place]);
        }
        ok = phase();
    }
    if (p.steps == 0) {                                           // scale X alone
        for (int i = threadIdx.x; i < (int)count; i += SMALL_THREADS) {
            const int r = i / p.cols, c = i - r * p.cols, row = p.tall ? c : r, col = p.tall ? r : c;
            const uint32_t at = (col >> 6) * plane + small_offset(row, col & 63);
            out[i] = from_f32<T>(p.last * (__half2float(*reinterpret_cast<const __half*>(xh + at)) + __half2float(*reinterpret_cast<const __half*>(xl + at))));
        }
    }
    if (!ok) {
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

// Shared memory of a matrix: A, b I + c A and X, and what an operand of 128 rows reads behind the last of them.
static long long small_bytes(int m, int n) {
    const long long mp = (m + 15) & ~15, blocks = (n + 63) / 64;
    return (4 + 2 * blocks) * mp * 128 + 128 * 128;
}
bool ortho_small_fits(int rows, int cols) {
    const int m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    if (m > 64 || small_bytes(m, n) > 224 * 1024) return false;
    return ((n + 63) / 64 + 3) / 4 * ((m + 15) & ~15) <= SMALL_GRAM_COLS;
}

template <typename T>
static int launch_small_typed(const void* g, void* out, int batch, const SmallArgs& a, cudaStream_t st) {
    auto kern = ortho_small_kernel<T>;
    static bool attr_set[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        if (check_cuda(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 * 1024))) return EBS_ERR_CUDA;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    return launch_chained(kern, dim3((unsigned)batch), SMALL_THREADS, (size_t)small_bytes(a.m, a.n), st, 1, static_cast<const T*>(g), static_cast<T*>(out), a);
}
int launch_ortho_small(const void* g, void* out, int batch, int rows, int cols, int dtype, int steps, float eps, float first, float last, const OrthoFactors& f, cudaStream_t st) {
    SmallArgs a;
    a.rows = rows; a.cols = cols; a.tall = rows > cols;
    a.m = a.tall ? cols : rows;
    a.n = a.tall ? rows : cols;
    a.mp = (a.m + 15) & ~15;
    a.blocks = (a.n + 63) / 64;
    a.steps = steps;
    a.eps = eps; a.first = first; a.last = last;
    a.wait_limit = device_wait_limit();
    a.test_flags = device_test_flags();
    a.f = f;
    if (dtype == EBS_F32) return launch_small_typed<float>(g, out, batch, a, st);
    if (dtype == EBS_F16) return launch_small_typed<__half>(g, out, batch, a, st);
    return launch_small_typed<__nv_bfloat16>(g, out, batch, a, st);
}

}  // namespace ebs
