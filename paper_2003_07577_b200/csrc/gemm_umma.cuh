// Matrix products of 16-bit operands on tcgen05.mma, operands by TMA: pieces shared by the tile kernel (gemm_tile.cu) and the
// persistent pair kernel (gemm_pair.cu).
//
// Shared-memory tiles are 64 elements (128 bytes) wide with the 128-byte swizzle, whichever way an operand lies in memory:
//  - reduction along a row (K-major): [rows][64 k], 8-row groups 1024 bytes apart; the 16-element step of one MMA is 32 bytes;
//  - reduction across rows (MN-major): blocks of [64 k][64 rows], a block 8192 bytes, 8-k groups 1024 bytes apart; the step is
//    16 rows of the block, 2048 bytes.  No operand is ever transposed in memory.
#pragma once

#include <cuda.h>

#include <type_traits>

#include "conv_frame.cuh"
#include "conv_umma.cuh"
#include "gemm.cuh"

namespace ebs {

constexpr int GEMM_BK = 64;                     // reduction elements of a stage
constexpr int GEMM_ROW_BYTES = 128;

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n" ::"r"(dst), "l"(map),
                 "r"(x), "r"(y), "r"(z), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
// Bounded wait of a converged warp that has nothing else to do: no sleep between polls.
__device__ __forceinline__ bool mbar_wait_warp(uint64_t* bar, uint32_t parity, volatile int* abort_flag, unsigned limit) {
    const uint32_t addr = smem_u32(bar);
    for (unsigned it = 0; it < limit; ++it) {
        uint32_t done;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}\n"
            : "=r"(done) : "r"(addr), "r"(parity) : "memory");
        if (__all_sync(0xffffffffu, done != 0)) return true;
        if (__any_sync(0xffffffffu, *abort_flag != 0)) return false;
    }
    *abort_flag = 1;
    return false;
}

// Descriptor words of a 128-byte-swizzled tile: the low word takes the start address, the high word is constant.
__device__ __forceinline__ uint32_t tile_desc_lo(uint32_t smem_addr, bool mn_major) {
    return ((smem_addr >> 4) & 0x3FFFu) | ((mn_major ? 8192u >> 4 : 1u) << 16);      // leading offset: next 64-row block
}
constexpr uint32_t TILE_DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);           // 8-row groups, descriptor version, 128-byte swizzle

// Columns of this warp's 32 lanes out of tensor memory.
__device__ __forceinline__ void tmem_ld8_issue(uint32_t taddr, uint32_t (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld8_wait(uint32_t (&v)[8]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;\n" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]) :: "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&v)[8]) {
    tmem_ld8_issue(taddr, v);
    tmem_ld8_wait(v);
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
template <int W>
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t (&v)[W]) {
    if constexpr (W == 8) tmem_ld8(taddr, v);
    else if constexpr (W == 16) tmem_ld16(taddr, v);
    else if constexpr (W == 32) { tmem_ld32_issue(taddr, v); tmem_ld32_wait(v); }
    else {
        uint32_t a[32], b[32];
        tmem_ld32_issue(taddr, a);
        tmem_ld32_issue(taddr + 32, b);
        tmem_ld32_wait(a);
        tmem_ld32_wait(b);
#pragma unroll
        for (int i = 0; i < 32; ++i) { v[i] = a[i]; v[32 + i] = b[i]; }
    }
}

// Instruction descriptor: fp32 sums, both operands fp16 (0) or bf16 (1).
__host__ __device__ constexpr uint32_t gemm_idesc(int m, int n, bool bf16, bool a_mn, bool b_mn) {
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void umma_f16(uint32_t leader, uint32_t tmem_d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %3};\n\t"
        "mov.b64 db, {%2, %3};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "setp.ne.b32 q, %6, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}\n"
        :: "r"(tmem_d), "r"(a_lo), "r"(b_lo), "r"(TILE_DESC_HI), "r"(idesc), "r"(accumulate), "r"(leader)
        : "memory");
}

// Host side: a three-dimensional tensor map, of 64-byte rows with their swizzle (narrow) or 128-byte ones.
bool encode_map(CUtensorMap* map, CUtensorMapDataType type, const void* p, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box, bool narrow);
// Tensor map of an operand.  mn: its rows or columns in the result, red: the reduction; box_mn: rows a K-major box takes.
// False: the driver has no tensor maps, or refused this one.
bool gemm_operand_map(const GemmOperand& o, int mn, int red, int batch, int box_mn, bool bf16, CUtensorMap* map);

// Stages of 64 reduction elements that are summed in the tensor core before they go on in registers: it truncates what it adds to an
// accumulator (sums of one sign, measured: 6.4e-9 of the sum an element).  Split products: few.  16-bit operands: GEMM_LONG, which costs 2.6e-5
// of the sum, a twentieth of what fp16 rounds (131072 elements in one accumulator: 8e-4).
constexpr int GEMM_CHUNK = 4, GEMM_LONG = 64;

// Shape of a product D = A B over `red`; D has `rows` x `cols` (row-major results) as the caller sees them.
struct GemmShape {
    int rows, cols, red, batch;
    bool symmetric = false;                // the result is known to be symmetric: one half of it need not be summed
    int chunk = GEMM_CHUNK;                // split products: stages summed in the tensor core at a time
};

int gemm_sm_count();

// What becomes of the sums, N neighbouring columns of a row at a time (`left` of them exist; vec: all do, at addresses of whole 16 bytes):
// `columns` and `ahead` load what is needed, `touch` reads the parameters that `pack` will use, which finishes and stores.  HOLES: it may leave
// elements (and then says so) whose results finish_infinite has.

// The results of a linear layer or of its gradients.
template <typename T>
struct LinearOut {
    static constexpr int N = Pack<T>::N;
    static constexpr bool HOLES = sizeof(T) == 4;
    using Columns = GemmColumns<T>;
    using Ahead = GemmAhead;
    GemmOut o;
    __device__ __forceinline__ void touch() const { asm volatile("" ::"l"(o.y), "l"(o.z), "l"(o.ldz), "l"(o.ldy), "f"(o.alpha), "r"(o.act)); }
    // an element at a time: what its column and its place need from memory, then the rest
    struct Column { float bias; int exp; };
    struct Place { float residual; int row_exp; };
    __device__ __forceinline__ void column(int col, Column& c) const {
        c.bias = o.bias ? to_f32(static_cast<const T*>(o.bias)[col]) : 0.0f;
        if (sizeof(T) == 4) c.exp = o.col_exp[col];
    }
    __device__ __forceinline__ void place(long long row, int col, Place& p) const {
        if (o.residual) p.residual = to_f32(static_cast<const T*>(o.residual)[row * o.ldr + col]);
        if (sizeof(T) == 4) p.row_exp = o.row_exp[row];
    }
    __device__ __forceinline__ bool one(int, long long row, int col, float v, const Column& c, const Place& p) const {
        if (sizeof(T) == 4) {
            bool hole = false;
            if (abs(c.exp) <= SCALE_PLAIN && abs(p.row_exp) <= SCALE_PLAIN) v *= power_of_two(p.row_exp) * power_of_two(c.exp);
            else v = unscale(v, p.row_exp, c.exp, hole);
            if (hole) return true;
        }
        v = fmaf(v, o.alpha, c.bias);
        if (o.z) static_cast<T*>(o.z)[row * o.ldz + col] = from_f32<T>(v);
        if (o.act) v = activation<sizeof(T) == 2>(v, o.act);
        if (o.residual) v += p.residual;
        static_cast<T*>(o.y)[row * o.ldy + col] = from_f32<T>(v);
        return false;
    }
    __device__ __forceinline__ void columns(int col, int left, bool vec, Columns& c) const { gemm_columns<T>(o, col, left, vec, c); }
    __device__ __forceinline__ void ahead(int, long long row, int col, int left, bool vec, Ahead& a) const { gemm_ahead<T>(o, row, col, left, vec, a); }
    __device__ __forceinline__ bool pack(int, long long row, int col, int left, bool vec, float (&v)[N], const Columns& c, const Ahead& a) const {
        return gemm_store_pack<T>(o, row, col, left, vec, v, c, a);
    }
};

// Results kept for further products, as two fp16 planes hi + lo (the value times a power of two of the caller's choice, folded into the
// factors): alpha * sum + diag * (row == col), and a second matrix alpha2 * sum + diag2 * (row == col) of the same form where y2 is
// set.  Rows are padded to whole groups of eight elements, so that a pack is always whole.
struct PlanesOut {
    static constexpr int N = 4;
    static constexpr bool HOLES = false;
    struct Columns {};
    struct Ahead {};
    __half* y;
    __half* y2;
    long long ld, plane, batch;            // of either: elements between rows, planes, matrices of a batch
    float alpha, diag, alpha2, diag2;
    __device__ __forceinline__ void touch() const { asm volatile("" ::"l"(y), "l"(y2), "l"(plane), "f"(alpha), "f"(diag2)); }
    __device__ __forceinline__ void columns(int, int, bool, Columns&) const {}
    __device__ __forceinline__ void ahead(int, long long, int, int, bool, Ahead&) const {}
    __device__ __forceinline__ void store(__half* q, long long row, int col, const float (&v)[N], float factor, float on_diag) const {
        float t[4];
        uint2 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = v[i] * factor + (row == col + i ? on_diag : 0.0f);
        split_pair(t[0], t[1], hi.x, lo.x);
        split_pair(t[2], t[3], hi.y, lo.y);
        *reinterpret_cast<uint2*>(q) = hi;
        *reinterpret_cast<uint2*>(q + plane) = lo;
    }
    __device__ __forceinline__ bool pack(int b, long long row, int col, int, bool, float (&v)[N], const Columns&, const Ahead&) const {
        const long long at = b * batch + row * ld + col;
        store(y + at, row, col, v, alpha, diag);
        if (y2) store(y2 + at, row, col, v, alpha2, diag2);
        return false;
    }
};

// The last product of an orthogonalisation: alpha * sum, rounded to the caller's type.
struct FinalOut {
    void* y;
    long long ld, batch;
    float alpha;
};
template <typename T>
struct TypedFinal {
    static constexpr int N = Pack<T>::N;
    static constexpr bool HOLES = false;
    struct Columns {};
    struct Ahead {};
    FinalOut o;
    struct Column {};
    struct Place {};
    __device__ __forceinline__ void column(int, Column&) const {}
    __device__ __forceinline__ void place(long long, int, Place&) const {}
    __device__ __forceinline__ bool one(int b, long long row, int col, float v, const Column&, const Place&) const {
        static_cast<T*>(o.y)[b * o.batch + row * o.ld + col] = from_f32<T>(v * o.alpha);
        return false;
    }
    __device__ __forceinline__ void touch() const { asm volatile("" ::"l"(o.y), "l"(o.batch), "f"(o.alpha)); }
    __device__ __forceinline__ void columns(int, int, bool, Columns&) const {}
    __device__ __forceinline__ void ahead(int, long long, int, int, bool, Ahead&) const {}
    __device__ __forceinline__ bool pack(int b, long long row, int col, int left, bool vec, float (&v)[N], const Columns&, const Ahead&) const {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= o.alpha;
        store_pack(static_cast<T*>(o.y) + b * o.batch + row * o.ld + col, v, left, vec);
        return false;
    }
};

// A part of the sums, for reduce_parts: fp32, the parts behind one another (the pair kernel alone writes them).
struct PartialOut {
    float* y;                              // [part][batch][rows][ld], ld a multiple of four
    long long ld, batch, part;
    int parts;
};

// ebs_test_set_device_wait's settings.
unsigned device_wait_limit();
int device_test_flags();

}  // namespace ebs
