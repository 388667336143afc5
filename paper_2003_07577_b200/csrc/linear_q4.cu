// Layers with weights of 4 bits and a scale for each group of them: packing, reading back, and the product with a few rows.  See include/ebs.h.
//
// The product is bound by the weights' bytes (half a byte a weight and the scales), and next by the instructions that turn codes into operands (one row through 8192 -> 28672 bf16: 27 to 29 us,
// 4.1 to 4.4 TB/s, the logic pipe 62% busy; packing 134 million fp32 weights 114 us, 5.3 TB/s).  Weights lie in
// tiles of 16 outputs x 64 inputs, 512 bytes, in the order in which the lanes of a warp need them for four mma.sync m16n8k16: one 16-byte
// load a lane.  A word holds the eight codes (+ 8) of a lane for one MMA, those of operand register i in bits 4i .. 4i+3 and 16+4i .. 16+4i+3, so that a mask and the bits of
// a power of two make two 16-bit numbers of them at once.  Codes and 16-bit activations multiply exactly; a tile's sum over 64 inputs (32, where
// a group has no more; with few rows of 16-bit activations two tiles', where it has 128) leaves the MMA in fp32 and is multiplied by its group's scale there.  fp32 activations go as three bf16 planes of
// 8 bits each, which hold all 24.
//
// MMA k index (step s, half h, lane group t = lane % 4, element j) stands for input (s / 2) * 32 + t * 8 + (s % 2) * 4 + h * 2 + j of the 64: a lane's share
// of a row of activations is two runs of eight neighbouring elements, which it loads from the row as it lies in memory.
#include "gemm_tile.cuh"
#include "tensors.cuh"

namespace ebs {

constexpr int Q4_ROWS = 16, Q4_K = 64, Q4_TILE_BYTES = 512;

struct Q4Layout {
    int tiles, kbs, groups;                // tiles of 16 outputs, of 64 inputs, groups of a row
    size_t codes, scales;                  // bytes of all experts' codes (rounded up), of their scales
};
static Q4Layout q4_layout(const ebs_q4_desc& d) {
    Q4Layout l;
    l.tiles = (d.n + Q4_ROWS - 1) / Q4_ROWS;
    l.kbs = (d.k + Q4_K - 1) / Q4_K;
    l.groups = (d.k + d.group - 1) / d.group;
    l.codes = round256((size_t)d.experts * l.tiles * l.kbs * Q4_TILE_BYTES);
    l.scales = (size_t)d.experts * l.tiles * l.groups * Q4_ROWS * element_size(d.dtype);
    return l;
}
static int check_q4(const ebs_q4_desc* d) {
    if (!d || d->experts < 1 || d->n < 1 || d->k < 1 || !real_dtype(d->dtype)) return EBS_ERR_INVALID_ARG;
    if (d->group != 32 && d->group != 64 && d->group != 128) return EBS_ERR_INVALID_ARG;
    if (d->n > (1 << 30) || d->k > (1 << 30) || (double)d->experts * d->n * d->k > (double)(1LL << 40)) return EBS_ERR_OVERFLOW;
    const Q4Layout l = q4_layout(*d);
    if ((long long)d->experts * l.tiles * l.kbs >= (1LL << 31)) return EBS_ERR_OVERFLOW;
    return EBS_OK;
}

// ---------------------------------------------------------------------------------------------------- packing
// Input of element e (0 .. 7) of run r (0, 1) of a lane; its code lies in word 2 * r + e / 4 of the lane's four.
__device__ __forceinline__ int q4_input(int r, int lane, int e) { return r * 32 + (lane & 3) * 8 + e; }

// Eight neighbouring elements of a row, of which `left` exist.
template <typename S>
__device__ __forceinline__ void load8(const S* p, int left, bool vec, float (&v)[8]) {
    if (vec && left >= 8) {
        constexpr int N = Pack<S>::N;
#pragma unroll
        for (int i = 0; i < 8 / N; ++i) {
            float t[N];
            load_pack<S>(p + i * N, t);
#pragma unroll
            for (int e = 0; e < N; ++e) v[i * N + e] = t[e];
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < left ? to_f32(p[e]) : 0.0f;
}

// floor(w / s + 1/2) of eight weights, exactly, in the low bits of each word.  The quotient by the reciprocal (inv = 1 / s) is off by less than 2^-19; with 2^-16 taken off first its floor (a
// sum with 1.5 * 2^23, rounded down) is the code or one less, and the sign of a fused multiply-add's remainder tells which.  (Only those near a border by their remainders, the rest rounded:
// fp32 weights the same, but two of five of a warp's loads of bf16 weights hold one such, and 235 million took 385 us, so 287.)  wide: quotients may leave -8 .. 7 (a scale of few bits).
__device__ __forceinline__ void q4_codes(const float (&v)[8], float s, float inv, bool wide, uint32_t (&code)[8]) {
    constexpr float WHOLE = 12582912.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float r = __fadd_rd(fmaf(v[e], inv, 0.5f - 0x1p-16f), WHOLE), left = fmaf(-((r - WHOLE) + 0.5f), s, v[e]);
        code[e] = __float_as_uint(r) + 1u - (__float_as_uint(left) >> 31);
    }
    if (wide)
#pragma unroll
        for (int e = 0; e < 8; ++e) code[e] = (uint32_t)min(max((int)(code[e] - __float_as_uint(WHOLE)), -8), 7);
}

template <typename S>
struct Q4Pack {
    const S* w;
    uint4* codes;
    void* scales;
    long long ldw;
    unsigned units;                        // warps' pieces of work
    int n, k, tiles, kbs, groups;
};
// Eight rows of a piece of weights as the lanes of a warp have them, for matrices whose rows start anywhere: in memory the lanes take neighbouring elements, here their own eight (an element
// a lane in 32 places of memory takes 32 accesses: 4.6 million weights of rows of 198 fp16 values packed and read back in 36 us).
template <typename S, int COLS> struct Q4Stage { S row[8][COLS + 16 / sizeof(S)]; };

// A warp packs 16 rows x KB tiles of 64 inputs, which hold whole groups of G: the largest magnitudes, scales and codes from one load.
template <typename S, typename T, int G, bool VEC>
__global__ void __launch_bounds__(256) q4_pack_kernel(const __grid_constant__ Q4Pack<S> g) {
    constexpr int KB = G == 128 ? 2 : 1, N = Pack<S>::N, W = 8 / N;
    constexpr bool AHEAD = VEC && sizeof(S) == 2;
    let_next_kernel_start();
    wait_for_previous_kernel();
    __shared__ __align__(16) Q4Stage<S, KB * Q4_K> stages[VEC ? 1 : 8];
    const int lane = threadIdx.x & 31, gid = lane >> 2;
    Q4Stage<S, KB * Q4_K>& stage = stages[VEC ? 0 : threadIdx.x >> 5];
    const unsigned across = (unsigned)((g.kbs + KB - 1) / KB);
    for (unsigned u = blockIdx.x * 8u + (threadIdx.x >> 5); u < g.units; u += gridDim.x * 8u) {
        const long long tile = u / across;                        // of all experts
        const int kb0 = (int)(u % across) * KB;
        const long long expert = (unsigned)tile / (unsigned)g.tiles;
        const int row0 = (int)((unsigned)tile % (unsigned)g.tiles) * Q4_ROWS;
        uint32_t word[KB][4];
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) word[b][i] = 0x88888888u;
        // All loads of a row before the first is used (a branch a load: 140 us, so 114); of 16-bit weights the second half's (rows gid + 8) before the first half's codes are found (235 million
        // bf16 287 us, so 214).
        uint4 raw[KB][2][W], next[KB][2][W];
        const auto load = [&](int half, uint4 (&raw)[KB][2][W]) {
            const int row = row0 + gid + 8 * half;
            const S* p = g.w + (expert * g.n + row) * g.ldw + kb0 * Q4_K;
            if (!VEC) {
                __syncwarp();                                     // (what was there is read)
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int h = 0; h < 2 * KB; ++h) {
                        const int at = row0 + 8 * half + i, c = kb0 * Q4_K + h * 32 + lane;
                        stage.row[i][h * 32 + lane] = at < g.n && c < g.k ? g.w[(expert * g.n + at) * g.ldw + c] : from_f32<S>(0.0f);
                    }
                __syncwarp();
                p = stage.row[gid];
            }
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int c = b * Q4_K + q4_input(r, lane, 0), left = !VEC ? 8 : row < g.n ? g.k - kb0 * Q4_K - c : 0;
#pragma unroll
                    for (int i = 0; i < W; ++i) raw[b][r][i] = left >= 8 ? reinterpret_cast<const uint4*>(p + c)[i] : make_uint4(0u, 0u, 0u, 0u);
                    if (left > 0 && left < 8)
#pragma unroll
                        for (int e = 0; e < 7; ++e)
                            if (e < left) reinterpret_cast<S*>(&raw[b][r][e / N])[e % N] = p[c + e];
                }
        };
        load(0, raw);
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {                    // rows gid and gid + 8
            const int row = row0 + gid + 8 * half;
            float v[KB][2][8];
            unsigned top[KB][2];
            if (AHEAD && half == 0) load(1, next);
            if (!AHEAD && half == 1) load(1, raw);
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        float t[N];
                        unpack<S>(raw[b][r][i], t);
#pragma unroll
                        for (int e = 0; e < N; ++e) v[b][r][i * N + e] = t[e];
                        if (AHEAD) raw[b][r][i] = next[b][r][i];
                    }
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    unsigned t = 0u;                              // (as integers: a NaN is larger than an infinity)
#pragma unroll
                    for (int e = 0; e < 8; ++e) t = max(t, __float_as_uint(v[b][r][e]) & 0x7fffffffu);
                    t = max(t, __shfl_xor_sync(0xffffffffu, t, 1));
                    top[b][r] = max(t, __shfl_xor_sync(0xffffffffu, t, 2));
                }
            if (G >= 64)
#pragma unroll
                for (int b = 0; b < KB; ++b) top[b][0] = top[b][1] = max(top[b][0], top[b][1]);
            if (G == 128) top[0][0] = top[0][1] = top[KB - 1][0] = top[KB - 1][1] = max(top[0][0], top[KB - 1][0]);
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const T kept = from_f32<T>(__fmul_rn(__uint_as_float(top[b][r]), 1.0f / 7.0f));
                    float s = to_f32(kept);
                    const int group = ((kb0 + b) * Q4_K + r * 32) / G;
                    if ((lane & 3) == 0 && (G == 32 || r == 0) && (G != 128 || b == 0) && group < g.groups)
                        static_cast<T*>(g.scales)[(tile * g.groups + group) * Q4_ROWS + 2 * gid + half] = row < g.n ? kept : from_f32<T>(0.0f);
                    if (!(s > 0.0f) || (__float_as_uint(s) & 0x7f800000u) == 0x7f800000u) continue;          // (codes of zero)
                    if (s < 1e-30f) {                                        // times 2^100: no reciprocal overflows, no remainder is lost
                        s *= 1.2676506e30f;
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[b][r][e] *= 1.2676506e30f;
                        top[b][r] = __float_as_uint(__uint_as_float(top[b][r]) * 1.2676506e30f);
                    }
                    const float inv = 1.0f / s;
                    uint32_t code[8], part[2] = {0u, 0u};
                    q4_codes(v[b][r], s, inv, __uint_as_float(top[b][r]) * inv > 7.4f, code);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        // register 2 * h + half of the MMA, element j; the code + 8 is the code with its sign bit turned
                        const int at = 8 * ((e >> 1) & 1) + 16 * (e & 1);
                        part[e >> 2] |= (code[e] << at) & (15u << at);
                    }
                    word[b][2 * r] ^= part[0] << (4 * half);
                    word[b][2 * r + 1] ^= part[1] << (4 * half);
                }
        }
#pragma unroll
        for (int b = 0; b < KB; ++b)
            if (kb0 + b < g.kbs) g.codes[(tile * g.kbs + kb0 + b) * 32 + lane] = make_uint4(word[b][0], word[b][1], word[b][2], word[b][3]);
    }
}

template <typename D>
struct Q4Unpack {
    const uint4* codes;
    const void* scales;
    D* w;
    long long ldw;
    unsigned units;
    int n, k, tiles, kbs, groups, shift;       // groups of 2^shift inputs
};
template <typename T, typename D, bool VEC>
__global__ void __launch_bounds__(256) q4_unpack_kernel(const __grid_constant__ Q4Unpack<D> g) {
    __shared__ __align__(16) Q4Stage<D, Q4_K> stages[VEC ? 1 : 8];
    let_next_kernel_start();
    wait_for_previous_kernel();
    constexpr int N = Pack<D>::N;
    const int lane = threadIdx.x & 31, gid = lane >> 2;
    Q4Stage<D, Q4_K>& stage = stages[VEC ? 0 : threadIdx.x >> 5];
    for (unsigned u = blockIdx.x * 8u + (threadIdx.x >> 5); u < g.units; u += gridDim.x * 8u) {
        const long long tile = u / (unsigned)g.kbs, expert = (unsigned)tile / (unsigned)g.tiles;
        const int kb = (int)(u % (unsigned)g.kbs), row0 = (int)((unsigned)tile % (unsigned)g.tiles) * Q4_ROWS;
        const uint4 q = g.codes[(long long)u * 32 + lane];
        const uint32_t word[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (!VEC) __syncwarp();                             // (what was there is read)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = row0 + gid + 8 * half, c = kb * Q4_K + q4_input(r, lane, 0);
                if (row >= g.n || c >= g.k) continue;
                const float s = to_f32(static_cast<const T*>(g.scales)[(tile * g.groups + ((kb * Q4_K + r * 32) >> g.shift)) * Q4_ROWS + 2 * gid + half]);
                D* to = VEC ? g.w + (expert * g.n + row) * g.ldw + c : &stage.row[gid][c - kb * Q4_K];
                const int left = VEC ? g.k - c : 8;
#pragma unroll
                for (int i = 0; i < 8 / N; ++i) {
                    float t[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const int j = i * N + e;
                        t[e] = s * (float)((int)(word[2 * r + (j >> 2)] >> (4 * (2 * ((j >> 1) & 1) + half) + 16 * (j & 1)) & 15u) - 8);
                    }
                    store_pack(to + i * N, t, left - i * N, left >= 8);
                }
            }
            if (!VEC) {
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int at = row0 + 8 * half + i, c = kb * Q4_K + h * 32 + lane;
                        if (at < g.n && c < g.k) g.w[(expert * g.n + at) * g.ldw + c] = stage.row[i][h * 32 + lane];
                    }
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------------- the product
__device__ __forceinline__ uint4 load_stream(const uint4* p) {      // read once: not kept in the first-level cache
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// (w & mask) | bits in one instruction (the compiler makes two of it: the two constants do not fit one).
__device__ __forceinline__ uint32_t masked(uint32_t w, uint32_t mask, uint32_t bits) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;\n" : "=r"(r) : "r"(w), "r"(mask), "r"(bits));
    return r;
}
// Operand registers of one MMA from a word of codes: the values code - 8.
template <typename T> struct Q4Operand;
template <> struct Q4Operand<__half> {
    // 0x6400: 1024, whose last bit is 1, so that a code in the low bits adds itself, one four bits up 16 times itself
    static __device__ __forceinline__ void make(uint32_t w, uint32_t (&a)[4]) {
        const uint32_t v = w >> 8;
        const __half2 low = __floats2half2_rn(-1032.0f, -1032.0f), sixteenth = __floats2half2_rn(0.0625f, 0.0625f), high = __floats2half2_rn(-72.0f, -72.0f);
        auto bits = [](uint32_t x) { return *reinterpret_cast<__half2*>(&x); };
        auto raw = [](__half2 x) { return *reinterpret_cast<uint32_t*>(&x); };
        a[0] = raw(__hadd2(bits(masked(w, 0x000f000fu, 0x64006400u)), low));
        a[1] = raw(__hfma2(bits(masked(w, 0x00f000f0u, 0x64006400u)), sixteenth, high));
        a[2] = raw(__hadd2(bits(masked(v, 0x000f000fu, 0x64006400u)), low));
        a[3] = raw(__hfma2(bits(masked(v, 0x00f000f0u, 0x64006400u)), sixteenth, high));
    }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static __device__ __forceinline__ void mma_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {       // the sum begins
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
    }
};
template <> struct Q4Operand<__nv_bfloat16> {
    // 0x4300: 128, whose last bit is 1
    static __device__ __forceinline__ void make(uint32_t w, uint32_t (&a)[4]) {
        const __nv_bfloat162 low = __floats2bfloat162_rn(-136.0f, -136.0f);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = masked(w >> (4 * i), 0x000f000fu, 0x43004300u);
            const __nv_bfloat162 v = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&x), low);
            a[i] = *reinterpret_cast<const uint32_t*>(&v);
        }
    }
    static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    }
    static __device__ __forceinline__ void mma_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {       // the sum begins
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
            : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
    }
};
template <> struct Q4Operand<float> : Q4Operand<__nv_bfloat16> {};

// fp32 x = high + middle + low, each what the one before left cut to bf16 (the upper half of its word): exact.  An infinity or a NaN is all in the first.  The low bits first.
__device__ __forceinline__ void q4_planes(float x, uint32_t (&t)[3]) {
    uint32_t bits = __float_as_uint(x);
    const bool finite = (bits & 0x7f800000u) != 0x7f800000u;
    if (!finite && (bits & 0x007fffffu) != 0u) bits |= 0x00400000u;
    const float r = finite ? x - __uint_as_float(bits & 0xffff0000u) : 0.0f;
    t[2] = bits;
    t[1] = __float_as_uint(r);
    t[0] = __float_as_uint(r - __uint_as_float(t[1] & 0xffff0000u));
}
__device__ __forceinline__ void q4_planes(float x, float y, uint32_t (&b)[3]) {
    uint32_t s[3], t[3];
    q4_planes(x, s);
    q4_planes(y, t);
#pragma unroll
    for (int p = 0; p < 3; ++p) b[p] = __byte_perm(s[p], t[p], 0x7632);
}
// A lane's activations of one row for 64 inputs: PL planes of two words for each of the four MMAs.  x: the lane's first element; left: elements of the row from there on.
template <typename T, bool PREPARED> struct Q4Acts {
    using X = T;
    static constexpr int PL = 1;
    uint32_t b[1][8];
    __device__ __forceinline__ void load(const T* x, long long, int left, bool whole) {
        if (whole) {
            const uint4 u = *reinterpret_cast<const uint4*>(x), v = *reinterpret_cast<const uint4*>(x + 32);
            b[0][0] = u.x; b[0][1] = u.y; b[0][2] = u.z; b[0][3] = u.w;
            b[0][4] = v.x; b[0][5] = v.y; b[0][6] = v.z; b[0][7] = v.w;
            return;
        }
        const uint16_t* p = reinterpret_cast<const uint16_t*>(x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int at = (i >> 2) * 32 + (i & 3) * 2;
            b[0][i] = (at < left ? (uint32_t)p[at] : 0u) | (at + 1 < left ? (uint32_t)p[at + 1] << 16 : 0u);
        }
    }
};
template <> struct Q4Acts<float, false> {
    using X = float;
    static constexpr int PL = 3;
    uint32_t b[3][8];
    __device__ __forceinline__ void load(const float* x, long long, int left, bool whole) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = (i >> 1) * 32 + (i & 1) * 4;
            float4 v;
            if (whole) v = *reinterpret_cast<const float4*>(x + at);
            else v = make_float4(at < left ? x[at] : 0.0f, at + 1 < left ? x[at + 1] : 0.0f, at + 2 < left ? x[at + 2] : 0.0f, at + 3 < left ? x[at + 3] : 0.0f);
            uint32_t t[3], u[3];
            q4_planes(v.x, v.y, t);
            q4_planes(v.z, v.w, u);
#pragma unroll
            for (int p = 0; p < 3; ++p) { b[p][2 * i] = t[p]; b[p][2 * i + 1] = u[p]; }
        }
    }
};
// (planes of whole tiles, q4_planes_kernel)
template <> struct Q4Acts<float, true> {
    using X = uint16_t;
    static constexpr int PL = 3;
    uint32_t b[3][8];
    __device__ __forceinline__ void load(const uint16_t* x, long long plane, int, bool) {
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            const uint4 u = *reinterpret_cast<const uint4*>(x + p * plane), v = *reinterpret_cast<const uint4*>(x + p * plane + 32);
            b[p][0] = u.x; b[p][1] = u.y; b[p][2] = u.z; b[p][3] = u.w;
            b[p][4] = v.x; b[p][5] = v.y; b[p][6] = v.z; b[p][7] = v.w;
        }
    }
};
// Planes of fp32 rows, each padded with zeros to whole tiles of 64: [plane][row][ldd].  A thread takes eight elements.
__global__ void __launch_bounds__(256) q4_planes_kernel(const float* __restrict__ x, long long ldx, int k, int ldd, long long packs, uint16_t* __restrict__ to) {
    let_next_kernel_start();
    wait_for_previous_kernel();
    const int across = ldd / 8;
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < packs; i += gridDim.x * 256LL) {
        const long long row = i / across;
        const int c = (int)(i - row * across) * 8;
        float v[8];
        load8<float>(x + row * ldx + c, k - c, (ldx & 3) == 0, v);
        uint4 out[3];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            uint32_t t[3];
            q4_planes(v[2 * h], v[2 * h + 1], t);
#pragma unroll
            for (int p = 0; p < 3; ++p) reinterpret_cast<uint32_t*>(&out[p])[h] = t[p];
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<uint4*>(to + (p * (packs / across) + row) * ldd + c) = out[p];
    }
}

constexpr int q4_mt(int nt) { return nt >= 4 ? 2 : 1; }             // tiles of 16 outputs a block takes: with many rows their activations serve two

struct Q4Args {
    const void *x, *scales, *bias, *residual;
    const uint4* codes;
    const int* offsets;
    void* y;
    long long ldx, ldr, ldy, plane;        // plane: elements between the planes of prepared activations
    int m, n, k, experts, tiles, kbs, groups, slots, act;
};

// The `slot`-th piece of up to `most` rows of an expert, in the order of the experts: the expert, its rows.  Offsets that are out of order or
// out of range are taken as the nearest ones that are not.
__device__ __forceinline__ bool q4_slot(const Q4Args& g, int slot, int most, int& expert, int& row0, int& rows) {
    if (!g.offsets) {
        expert = 0;
        row0 = slot * most;
        rows = min(most, g.m - row0);
        return rows > 0;
    }
    const int lane = threadIdx.x & 31;
    for (int e0 = 0; e0 < g.experts; e0 += 32) {
        const int e = e0 + lane;
        int begin = 0, count = 0;
        if (e < g.experts) {
            begin = min(max(g.offsets[e], 0), g.m);
            count = min(max(g.offsets[e + 1], begin), g.m) - begin;
        }
        const int pieces = (count + most - 1) / most;
        int sum = pieces;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, slot < sum);
        if (hit) {
            const int l = __ffs(hit) - 1;
            const int piece = slot - __shfl_sync(0xffffffffu, sum - pieces, l);
            expert = e0 + l;
            row0 = __shfl_sync(0xffffffffu, begin, l) + piece * most;
            rows = min(most, __shfl_sync(0xffffffffu, count, l) - piece * most);
            return true;
        }
        slot -= __shfl_sync(0xffffffffu, sum, 31);
    }
    return false;
}

// The scales of outputs gid and gid + 8 of a tile.
__device__ __forceinline__ float2 scale_pair(const float* p) { return *reinterpret_cast<const float2*>(p); }
__device__ __forceinline__ float2 scale_pair(const __half* p) { return __half22float2(*reinterpret_cast<const __half2*>(p)); }
__device__ __forceinline__ float2 scale_pair(const __nv_bfloat16* p) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(p)); }

// A block: 16 * MT outputs of up to 8 * NT rows; its WARPS warps share the reduction and add up in shared memory, in their order.  Columns of the MMA beyond the last row
// take its activations again and are not written.
template <typename T, int NT, int WARPS> constexpr int q4_blocks() { return NT == 1 && sizeof(T) == 2 ? 32 / WARPS : NT >= 4 ? 8 / WARPS : 16 / WARPS; }      // of an SM
template <typename T, bool PREPARED, int NT, int MT, int G, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, (q4_blocks<T, NT, WARPS>())) q4_kernel(const __grid_constant__ Q4Args g) {
    extern __shared__ float sums[];                                 // [warp][row][16 * MT outputs]
    constexpr int COLS = Q4_ROWS * MT, ROWS = 8 * NT, D = MT == 1 ? 4 : 2;
    // Tiles whose sum meets a scale: a group's two where that leaves the registers for it, and of 16-bit types alone.  Eight steps of the tensor core cut 2^-20 of a sum of one sign at
    // most, and those types round 2^-12 or 2^-9 of it; three planes make 24 steps, the second tile's on top of the whole first one's sum: 2^-20 seen, 2^-22 with a scale each.
    constexpr int UNIT = G == 128 && NT <= 2 && sizeof(T) == 2 ? 2 : 1;
    using Acts = Q4Acts<T, PREPARED>;
    using X = typename Acts::X;
    using Operand = Q4Operand<T>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    let_next_kernel_start();
    wait_for_previous_kernel();
    const int slot = (int)(blockIdx.x % (unsigned)g.slots), tile0 = (int)(blockIdx.x / (unsigned)g.slots) * MT;
    int expert, row0, rows;
    if (!q4_slot(g, slot, ROWS, expert, row0, rows)) return;
    const int units = (g.kbs + UNIT - 1) / UNIT, kb0 = (int)((long long)units * warp / WARPS) * UNIT, kb1 = min((int)((long long)units * (warp + 1) / WARPS) * UNIT, g.kbs);
    const X* x[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) x[i] = static_cast<const X*>(g.x) + (long long)(row0 + min(gid + 8 * i, rows - 1)) * g.ldx + tig * 8 + (long long)kb0 * Q4_K;
    const uint4* codes[MT];
    const T* scales[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const long long tile = (long long)expert * g.tiles + min(tile0 + t, g.tiles - 1);
        codes[t] = g.codes + (tile * g.kbs + kb0) * 32 + lane;
        scales[t] = static_cast<const T*>(g.scales) + tile * g.groups * Q4_ROWS + 2 * gid;
    }
    float acc[MT][NT][4], c[MT][NT][4];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[t][i][e] = 0.0f;

    // one tile of 64 inputs, `ahead` of the pointers; begin: its sum begins here, end: it meets its scale
    auto multiply = [&](const uint4 (&w)[MT], int kb, int ahead, bool whole, bool begin, bool end) {
        constexpr int Q = G == 32 ? 2 : 1, R = 4 / Q;
        auto load = [&](Acts& b, int i) { b.load(x[i] + ahead * Q4_K, g.plane, g.k - kb * Q4_K - tig * 8, whole); };
        auto scale_of = [&](int t, int q) { return scale_pair(scales[t] + (G == 32 ? min(kb * 2 + q, g.groups - 1) : G == 64 ? kb : kb >> 1) * Q4_ROWS); };
        auto sum = [&](const uint32_t (&a)[4][4], const Acts& b, const float2& s, int t, int i, int q) {
#pragma unroll
            for (int p = 0; p < Acts::PL; ++p)
#pragma unroll
                for (int r = R * q; r < R * q + R; ++r) {
                    if (p == 0 && r == R * q && begin) Operand::mma_first(c[t][i], a[r], b.b[p][2 * r], b.b[p][2 * r + 1]);
                    else Operand::mma(c[t][i], a[r], b.b[p][2 * r], b.b[p][2 * r + 1]);
                }
            if (end) {
                acc[t][i][0] = fmaf(c[t][i][0], s.x, acc[t][i][0]);
                acc[t][i][1] = fmaf(c[t][i][1], s.x, acc[t][i][1]);
                acc[t][i][2] = fmaf(c[t][i][2], s.y, acc[t][i][2]);
                acc[t][i][3] = fmaf(c[t][i][3], s.y, acc[t][i][3]);
            }
        };
        if constexpr (NT <= 2) {                                    // (activations first: 8192 -> 28672 27 us, operands first 32)
            Acts b[NT];
#pragma unroll
            for (int i = 0; i < NT; ++i) load(b[i], i);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const uint32_t word[4] = {w[t].x, w[t].y, w[t].z, w[t].w};
                uint32_t a[4][4];
#pragma unroll
                for (int r = 0; r < 4; ++r) Operand::make(word[r], a[r]);
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    float2 s = make_float2(0.0f, 0.0f);
                    if (end) s = scale_of(t, q);
#pragma unroll
                    for (int i = 0; i < NT; ++i) sum(a, b[i], s, t, i, q);
                }
            }
        } else {                                                    // (operands first: they stay, a row's activations come and go)
            uint32_t a[MT][4][4];
            float2 s[MT][Q];
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const uint32_t word[4] = {w[t].x, w[t].y, w[t].z, w[t].w};
#pragma unroll
                for (int r = 0; r < 4; ++r) Operand::make(word[r], a[t][r]);
#pragma unroll
                for (int q = 0; q < Q; ++q) s[t][q] = end ? scale_of(t, q) : make_float2(0.0f, 0.0f);
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                Acts b;
                load(b, i);
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int q = 0; q < Q; ++q) sum(a[t], b, s[t][q], t, i, q);
            }
        }
    };
    const int whole = PREPARED ? kb1 : min(kb1, g.k / Q4_K);        // tiles that are all there
    uint4 w[D][MT];                                                 // D tiles under way: a place is loaded anew when it is used
#pragma unroll
    for (int d = 0; d < D; ++d)
#pragma unroll
        for (int t = 0; t < MT; ++t)
            if (kb0 + d < kb1) w[d][t] = load_stream(codes[t] + d * 32);
#pragma unroll 1
    for (int kb = kb0; kb < kb1; kb += D) {
        if (kb + D <= whole) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                multiply(w[d], kb + d, d, true, d % UNIT == 0, d % UNIT == UNIT - 1);
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    if (kb + D + d < kb1) w[d][t] = load_stream(codes[t] + (D + d) * 32);
            }
        } else {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                if (kb + d >= kb1) break;
                multiply(w[d], kb + d, d, kb + d < whole, d % UNIT == 0, d % UNIT == UNIT - 1 || kb + d == kb1 - 1);
            }
            break;                                                  // (the warp's last tiles: no more than D, since at most the last one is not whole)
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) codes[t] += D * 32;
#pragma unroll
        for (int i = 0; i < NT; ++i) x[i] += D * Q4_K;
    }
    float* mine = sums + warp * ROWS * COLS;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[(8 * i + 2 * tig + (e & 1)) * COLS + t * Q4_ROWS + gid + 8 * (e >> 1)] = acc[t][i][e];
    __syncthreads();
    const T* bias = g.bias ? static_cast<const T*>(g.bias) + (long long)expert * g.n : nullptr;
    for (int i = threadIdx.x; i < rows * COLS; i += WARPS * 32) {
        const int r = i / COLS, col = tile0 * Q4_ROWS + i % COLS;
        if (col >= g.n) continue;
        float v = 0.0f;
#pragma unroll
        for (int q = 0; q < WARPS; ++q) v += sums[q * ROWS * COLS + i];
        if (bias) v += to_f32(bias[col]);
        if (g.act) v = activation<sizeof(T) == 2>(v, g.act);
        if (g.residual) v += to_f32(static_cast<const T*>(g.residual)[(long long)(row0 + r) * g.ldr + col]);
        static_cast<T*>(g.y)[(long long)(row0 + r) * g.ldy + col] = from_f32<T>(v);
    }
}

// How a product is run, from its sizes alone.
struct Q4Route {
    int nt;                                // rows that a block takes at a time, in eights: from those an expert has in the mean, twice that so that most experts' weights are read once
    bool prepared, copied;                 // x goes through the workspace as planes (fp32) or as it is, since its rows start anywhere
    int warps;                             // that share a tile's reduction
    long long pieces, blocks;              // pieces of rows: at most one for each expert that has rows, and one more for each full piece
    size_t workspace;
};
static Q4Route q4_route(const ebs_linear_desc& d, const ebs_q4_desc& q) {
    Q4Route r = {};
    const long long rows = q.experts == 1 ? d.m : 2LL * (((long long)d.m + q.experts - 1) / q.experts);
    const int most = d.dtype == EBS_F32 ? 4 : 8, tiles = (d.n + Q4_ROWS - 1) / Q4_ROWS, kbs = (d.k + Q4_K - 1) / Q4_K;
    r.nt = 1;
    while (r.nt < most && 8LL * r.nt < rows) r.nt *= 2;
    r.pieces = q.experts > 1 ? (long long)(q.experts < d.m ? q.experts : d.m) + d.m / (8 * r.nt) : (d.m + 8LL * r.nt - 1) / (8 * r.nt);
    r.blocks = r.pieces * ((tiles + q4_mt(r.nt) - 1) / q4_mt(r.nt));
    // (4096 -> 14336 of four rows, 57344 tiles: 30.4 us split where they are used, 19.4 with the launch that prepares them, which costs 2)
    r.prepared = d.dtype == EBS_F32 && r.blocks * kbs >= 8192;
    r.copied = !r.prepared && d.m > 1 && d.ldx * (long long)element_size(d.dtype) % 16 != 0;
// (14336 -> 4096: 15.6 us with 8 warps a tile, of which two blocks an SM have work, 9.9 with 16)
    // Short reductions: two, whose blocks are many at a time (58 experts of 64 -> 8435 fp32, nine rows: 36 us with eight, 14 with two).  Four where their blocks fill the SMs
    // (12 rows of two experts of 3392 -> 23270 38 us with eight, 29 with four; 4096 -> 14336, three quarters of a round, 9.6 and 10.9).
    const int four = r.nt == 1 && d.dtype != EBS_F32 ? 148 * 8 : 148 * 4;
    r.warps = r.nt == 1 && r.blocks < 148 * 3 && kbs >= 32 ? 16 : r.nt > 2 ? 8 : kbs <= 4 ? 2 : r.blocks >= four ? 4 : 8;
    r.workspace = r.prepared ? round256((size_t)d.m * kbs * Q4_K * 3 * 2) : r.copied ? round256((size_t)d.m * round8(d.k) * element_size(d.dtype)) : 0;
    return r;
}
template <typename T, bool PREPARED, int NT, int G, int WARPS>
static int launch_q4(const Q4Args& g, const Q4Route& r, cudaStream_t st) {
    constexpr int SMEM = WARPS * 8 * NT * Q4_ROWS * q4_mt(NT) * 4;
    auto kern = q4_kernel<T, PREPARED, NT, q4_mt(NT), G, WARPS>;
    if (SMEM > 48 * 1024) {
        static bool attr_set[64] = {};
        int dev = 0;
        cudaGetDevice(&dev);
        if (dev < 0 || dev >= 64 || !attr_set[dev]) {
            if (check_cuda(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM))) return EBS_ERR_CUDA;
            if (dev >= 0 && dev < 64) attr_set[dev] = true;
        }
    }
    return launch_chained(kern, dim3((unsigned)r.blocks), WARPS * 32, SMEM, st, 1, g);
}
template <typename T, bool PREPARED, int NT, int WARPS = 8>
static int launch_q4_group(const Q4Args& g, const Q4Route& r, int group, cudaStream_t st) {
    return group == 32 ? launch_q4<T, PREPARED, NT, 32, WARPS>(g, r, st) : group == 64 ? launch_q4<T, PREPARED, NT, 64, WARPS>(g, r, st) : launch_q4<T, PREPARED, NT, 128, WARPS>(g, r, st);
}
template <typename T, bool PREPARED>
static int launch_q4_rows(Q4Args& g, const Q4Route& r, int group, cudaStream_t st) {
    if (r.blocks > 0x7fffffffLL) return EBS_ERR_OVERFLOW;
    g.slots = (int)r.pieces;
    switch (r.nt) {
        case 1:
            switch (r.warps) {
                case 16: return launch_q4_group<T, PREPARED, 1, 16>(g, r, group, st);
                case 2: return launch_q4_group<T, PREPARED, 1, 2>(g, r, group, st);
                case 4: return launch_q4_group<T, PREPARED, 1, 4>(g, r, group, st);
                default: return launch_q4_group<T, PREPARED, 1>(g, r, group, st);
            }
        case 2:
            switch (r.warps) {
                case 2: return launch_q4_group<T, PREPARED, 2, 2>(g, r, group, st);
                case 4: return launch_q4_group<T, PREPARED, 2, 4>(g, r, group, st);
                default: return launch_q4_group<T, PREPARED, 2>(g, r, group, st);
            }
        case 4: return launch_q4_group<T, PREPARED, 4>(g, r, group, st);
        default:
            if constexpr (sizeof(T) == 2) return launch_q4_group<T, PREPARED, 8>(g, r, group, st);
            else return EBS_ERR_UNSUPPORTED;
    }
}

template <typename S, typename T>
static int launch_pack_typed(const ebs_q4_desc& d, const void* w, long long ldw, void* packed, cudaStream_t st) {
    const Q4Layout l = q4_layout(d);
    const int kb = d.group == 128 ? 2 : 1;
    Q4Pack<S> g{static_cast<const S*>(w), static_cast<uint4*>(packed), static_cast<char*>(packed) + l.codes, ldw, (unsigned)(d.experts * (long long)l.tiles * ((l.kbs + kb - 1) / kb)),
                d.n, d.k, l.tiles, l.kbs, l.groups};
    const unsigned blocks = (g.units + 7u) / 8u;
    const dim3 grid(blocks < 148 * 64 ? blocks : 148 * 64);
    const bool vec = ldw * (long long)sizeof(S) % 16 == 0;
    if (d.group == 32) return launch_chained(vec ? q4_pack_kernel<S, T, 32, true> : q4_pack_kernel<S, T, 32, false>, grid, 256, 0, st, 1, g);
    if (d.group == 64) return launch_chained(vec ? q4_pack_kernel<S, T, 64, true> : q4_pack_kernel<S, T, 64, false>, grid, 256, 0, st, 1, g);
    return launch_chained(vec ? q4_pack_kernel<S, T, 128, true> : q4_pack_kernel<S, T, 128, false>, grid, 256, 0, st, 1, g);
}
template <typename S>
static int launch_pack(const ebs_q4_desc& d, const void* w, long long ldw, void* packed, cudaStream_t st) {
    if (d.dtype == EBS_F32) return launch_pack_typed<S, float>(d, w, ldw, packed, st);
    if (d.dtype == EBS_F16) return launch_pack_typed<S, __half>(d, w, ldw, packed, st);
    return launch_pack_typed<S, __nv_bfloat16>(d, w, ldw, packed, st);
}
template <typename T, typename D>
static int launch_unpack_typed(const ebs_q4_desc& d, const void* packed, void* w, long long ldw, cudaStream_t st) {
    const Q4Layout l = q4_layout(d);
    Q4Unpack<D> g{static_cast<const uint4*>(packed), static_cast<const char*>(packed) + l.codes, static_cast<D*>(w), ldw, (unsigned)(d.experts * (long long)l.tiles * l.kbs), d.n, d.k,
                  l.tiles, l.kbs, l.groups, d.group == 32 ? 5 : d.group == 64 ? 6 : 7};
    const unsigned blocks = (g.units + 7u) / 8u;
    const dim3 grid(blocks < 148 * 64 ? blocks : 148 * 64);
    if (ldw * (long long)sizeof(D) % 16 == 0) return launch_chained(q4_unpack_kernel<T, D, true>, grid, 256, 0, st, 1, g);
    return launch_chained(q4_unpack_kernel<T, D, false>, grid, 256, 0, st, 1, g);
}
template <typename D>
static int launch_unpack(const ebs_q4_desc& d, const void* packed, void* w, long long ldw, cudaStream_t st) {
    if (d.dtype == EBS_F32) return launch_unpack_typed<float, D>(d, packed, w, ldw, st);
    if (d.dtype == EBS_F16) return launch_unpack_typed<__half, D>(d, packed, w, ldw, st);
    return launch_unpack_typed<__nv_bfloat16, D>(d, packed, w, ldw, st);
}

// Checks of the two calls that bring weights to 4 bits and back; packed_out: which of the two is written.
static int check_weights(const ebs_q4_desc* d, const void* w, int w_dtype, long long* ldw, const void* packed, bool packed_out) {
    const int rc = check_q4(d);
    if (rc) return rc;
    if (!w || !packed || !real_dtype(w_dtype)) return EBS_ERR_INVALID_ARG;
    if (*ldw == 0) *ldw = d->k;
    if (*ldw < d->k) return EBS_ERR_INVALID_ARG;
    const long long rows = (long long)d->experts * d->n;
    if (*ldw > (1LL << 40) / rows) return EBS_ERR_OVERFLOW;
    const size_t size = element_size(w_dtype);
    const Q4Layout l = q4_layout(*d);
    const long long bytes = (long long)((l.codes + l.scales) / size);
    const Rows t[] = {{w, rows, d->k, *ldw, !packed_out}, {packed, 1, bytes, bytes, packed_out}};
    return check_tensors(t, 2, size, nullptr, nullptr);
}

// The two descriptors of a product together, strides filled in.
static int check_product(const ebs_linear_desc* desc, const ebs_q4_desc* q, ebs_linear_desc* d) {
    int rc = check_q4(q);
    if (rc || (rc = complete_linear(desc, d))) return rc;
    return d->n != q->n || d->k != q->k || d->dtype != q->dtype ? EBS_ERR_INVALID_ARG : EBS_OK;
}

}  // namespace ebs

using namespace ebs;

extern "C" {

size_t ebs_q4_packed_bytes(const ebs_q4_desc* desc) {
    if (check_q4(desc)) return 0;
    const Q4Layout l = q4_layout(*desc);
    return l.codes + round256(l.scales);
}

int ebs_pack_weights_q4(const void* w_dev, int w_dtype, const ebs_q4_desc* desc, long long ldw, void* packed_dev, void* stream) {
    const int rc = check_weights(desc, w_dev, w_dtype, &ldw, packed_dev, true);
    if (rc) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (w_dtype == EBS_F32) return launch_pack<float>(*desc, w_dev, ldw, packed_dev, st);
    if (w_dtype == EBS_F16) return launch_pack<__half>(*desc, w_dev, ldw, packed_dev, st);
    return launch_pack<__nv_bfloat16>(*desc, w_dev, ldw, packed_dev, st);
}

int ebs_unpack_weights_q4(const void* packed_dev, const ebs_q4_desc* desc, void* w_dev, int w_dtype, long long ldw, void* stream) {
    const int rc = check_weights(desc, w_dev, w_dtype, &ldw, packed_dev, false);
    if (rc) return rc;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (w_dtype == EBS_F32) return launch_unpack<float>(*desc, packed_dev, w_dev, ldw, st);
    if (w_dtype == EBS_F16) return launch_unpack<__half>(*desc, packed_dev, w_dev, ldw, st);
    return launch_unpack<__nv_bfloat16>(*desc, packed_dev, w_dev, ldw, st);
}

size_t ebs_linear_q4_workspace_bytes(const ebs_linear_desc* desc, const ebs_q4_desc* q4) {
    ebs_linear_desc d;
    return check_product(desc, q4, &d) ? 0 : q4_route(d, *q4).workspace;
}

int ebs_linear_q4_forward(const void* x_dev, const void* packed_dev, const void* bias_dev, const void* residual_dev, const int* offsets_dev, const ebs_linear_desc* desc,
                          const ebs_q4_desc* q4, void* y_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
    ebs_linear_desc d;
    int rc = check_product(desc, q4, &d);
    if (rc) return rc;
    if (!packed_dev || (d.m > 0 && (!x_dev || !y_dev)) || (!offsets_dev && q4->experts != 1) || ((uintptr_t)offsets_dev & 3u)) return EBS_ERR_INVALID_ARG;
    const size_t size = element_size(d.dtype), need = ebs_linear_q4_workspace_bytes(desc, q4);
    if (need && (!workspace_dev || workspace_bytes < need)) return EBS_ERR_INVALID_ARG;
    const Q4Layout l = q4_layout(*q4);
    auto flat = [&](const void* p, size_t bytes, bool out) { return Rows{p, 1, (long long)(bytes / size), (long long)(bytes / size), out}; };
    const Rows t[] = {{x_dev, d.m, d.k, d.ldx, false}, flat(packed_dev, l.codes + l.scales, false), flat(bias_dev, (size_t)q4->experts * d.n * size, false),
                      {residual_dev, d.m, d.n, d.ldr, false}, {y_dev, d.m, d.n, d.ldy, true}, flat(need ? workspace_dev : nullptr, need, true)};
    if (check_tensors(t, 6, size, &t[3], &t[4])) return EBS_ERR_INVALID_ARG;
    if (offsets_dev) {
        const uintptr_t o = (uintptr_t)offsets_dev, oe = o + ((size_t)q4->experts + 1) * 4, y = (uintptr_t)y_dev, w = (uintptr_t)workspace_dev;
        if (d.m > 0 && o < y + ((size_t)(d.m - 1) * d.ldy + d.n) * size && y < oe) return EBS_ERR_INVALID_ARG;
        if (need && o < w + need && w < oe) return EBS_ERR_INVALID_ARG;
    }
    if (d.m == 0) return EBS_OK;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const Q4Route r = q4_route(d, *q4);
    Q4Args g{x_dev, static_cast<const char*>(packed_dev) + l.codes, bias_dev, residual_dev, static_cast<const uint4*>(packed_dev), offsets_dev, y_dev, d.ldx, d.ldr, d.ldy, 0,
             d.m, d.n, d.k, q4->experts, l.tiles, l.kbs, l.groups, 0, d.act};
    if (r.prepared || r.copied) {
        g.x = workspace_dev;
        g.ldx = r.prepared ? (long long)l.kbs * Q4_K : round8(d.k);
    }
    if (r.prepared) {
        const long long packs = d.m * (g.ldx / 8), blocks = (packs + 255) / 256;
        g.plane = d.m * g.ldx;
        if ((rc = launch_chained(q4_planes_kernel, dim3((unsigned)(blocks < 1184 ? blocks : 1184)), 256, 0, st, 1, static_cast<const float*>(x_dev), d.ldx, d.k, (int)g.ldx, packs,
                                 static_cast<uint16_t*>(workspace_dev))))
            return rc;
    } else if (r.copied) {                                         // (fp32 rows as twice as many 16-bit elements)
        const int halves = (int)(size / 2);
        CopyJobs jobs = {};
        add_copy_rows(&jobs, x_dev, workspace_dev, d.m, d.k * halves, d.ldx * halves, g.ldx * halves);
        if ((rc = launch_copies(jobs, st))) return rc;
    }
    if (d.dtype == EBS_F32) return r.prepared ? launch_q4_rows<float, true>(g, r, q4->group, st) : launch_q4_rows<float, false>(g, r, q4->group, st);
    if (d.dtype == EBS_F16) return launch_q4_rows<__half, false>(g, r, q4->group, st);
    return launch_q4_rows<__nv_bfloat16, false>(g, r, q4->group, st);
}

}  // extern "C"
