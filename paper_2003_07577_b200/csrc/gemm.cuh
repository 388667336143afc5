// Shared pieces of the real-valued operators (linear.cu, orthogonalize.cu): element types, activations, what happens to a
// sum on its way out.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ebs_internal.cuh"

namespace ebs {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Two values as fp16 pairs hi + lo, both rounded to nearest: 22 bits (one conversion instruction a pair).
__device__ __forceinline__ void split_pair(float a, float b, uint32_t& hi, uint32_t& lo) {
    const __half2 h = __floats2half2_rn(a, b);
    const float2 f = __half22float2(h);
    const __half2 l = __floats2half2_rn(a - f.x, b - f.y);
    hi = *reinterpret_cast<const uint32_t*>(&h);
    lo = *reinterpret_cast<const uint32_t*>(&l);
}
// Two values in one 32-bit word of 16-bit elements.
template <typename T> __device__ __forceinline__ uint32_t pair_word(float a, float b);
template <> __device__ __forceinline__ uint32_t pair_word<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pair_word<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

inline size_t element_size(int dtype) { return dtype == EBS_F32 ? 4 : 2; }
inline bool real_dtype(int dtype) { return dtype == EBS_F32 || dtype == EBS_F16 || dtype == EBS_BF16; }

// Elementary functions at the accuracy of the results' type: fp32 results take CUDA's functions, 16-bit results (rounding 2^-9 or 2^-12)
// the hardware exponential and reciprocal (relative error about 2^-21).
__device__ __forceinline__ float fast_reciprocal(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float fast_exp(float v) {           // 2^(v log2 e)
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v * 1.44269504f));
    return r;
}
template <bool FAST> __device__ __forceinline__ float exp_of(float v) { return FAST ? fast_exp(v) : expf(v); }
template <bool FAST> __device__ __forceinline__ float reciprocal(float v) { return FAST ? fast_reciprocal(v) : 1.0f / v; }
// The logistic function of v and its complement, neither taken as a difference: both keep their relative accuracy.
template <bool FAST>
__device__ __forceinline__ void logistic(float v, float& s, float& rest) {
    const float t = exp_of<FAST>(-fabsf(v)), r = reciprocal<FAST>(1.0f + t), tr = t * r;
    s = v >= 0.0f ? r : tr;
    rest = v >= 0.0f ? tr : r;
}
// (1 + erf(z / sqrt 2)) / 2, and exp(-z^2 / 2).  16-bit results: Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26, absolute
// error 1.5e-7; the exponential serves both.
template <bool FAST>
__device__ __forceinline__ void normal_cdf(float z, float& cdf, float& bell) {
    if (FAST) {
        const float a = fabsf(z) * 0.70710678f, t = fast_reciprocal(fmaf(0.3275911f, a, 1.0f));
        bell = fast_exp(-a * a);
        const float half_tail = 0.5f * bell * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
        cdf = z >= 0.0f ? 1.0f - half_tail : half_tail;
    } else {
        bell = expf(-0.5f * z * z);
        cdf = 0.5f * (1.0f + erff(z * 0.70710678f));
    }
}
// act(z) and act'(z) as include/ebs.h states them.  (1 + tanh u) / 2 is the logistic function of 2u.
template <bool FAST>
__device__ __forceinline__ float activation(float z, int act) {
    float s, e;
    switch (act) {
        case EBS_ACT_RELU: return z > 0.0f ? z : 0.0f;
        case EBS_ACT_GELU: normal_cdf<FAST>(z, s, e); return z * s;
        case EBS_ACT_GELU_TANH: logistic<FAST>(1.59576912f * (z + 0.044715f * z * z * z), s, e); return z * s;
        case EBS_ACT_SILU: logistic<FAST>(z, s, e); return z * s;
        default: return z;
    }
}
template <bool FAST>
__device__ __forceinline__ float activation_slope(float z, int act) {
    float s, rest, e;
    switch (act) {
        case EBS_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
        case EBS_ACT_GELU: normal_cdf<FAST>(z, s, rest); return fmaf(z * 0.39894228f, rest, s);
        case EBS_ACT_GELU_TANH:
            logistic<FAST>(1.59576912f * (z + 0.044715f * z * z * z), s, rest);
            // (s times rest is below 2^-149 from |z| = 20 on; the polynomial there would leave the type's range and make zero times infinity of it.
            // z - z: zero, and NaN for an infinite z, as the other two give)
            e = fminf(fmaxf(z, -20.0f), 20.0f) + (z - z);
            return s * (1.0f + e * rest * (1.59576912f * (1.0f + 0.134145f * e * e)));
        case EBS_ACT_SILU:
            logistic<FAST>(z, s, rest);
            return s * (1.0f + z * rest);
        default: return 1.0f;
    }
}

// Kernels of one call start while the one before them still runs (programmatic launches): each waits here, before it touches memory, for
// that one's end and results ...
__device__ __forceinline__ void wait_for_previous_kernel() { asm volatile("griddepcontrol.wait;\n" ::: "memory"); }
// ... and lets the next one start once all its own blocks run.  A block that holds tensor memory calls this after it got it: the next
// kernel's blocks may take what is left.
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory"); }

template <typename... P, typename... A>
inline int launch_chained(void (*kern)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster, A&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return check_cuda(cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...));
}

// Powers of two that fp32 operands are scaled by before they are split (linear.cu): one exponent a row or column.
constexpr int SCALE_NAN = 1 << 20;         // the row holds a NaN: so do all its results
constexpr int SCALE_INF = 1 << 21;         // it holds an infinity: its results are found from the fp32 operands (finish_infinite)

// fp32 operands of a split product, for rows and columns with infinities: a[i * a_row + r * a_red], b[j * b_col + r * b_red].
struct GemmFp32 {
    const float *a = nullptr, *b = nullptr;
    long long a_row = 0, a_red = 0, b_col = 0, b_red = 0;
    int red = 0;
};

// What becomes of the sum v of output (row, col):
//   v *= 2^(row_exp[row] + col_exp[col])       (split fp32 operands)
//   z = alpha * v + bias[col];  y = act(z) + residual
struct GemmOut {
    const void* bias = nullptr;
    const void* residual = nullptr;
    void* z = nullptr;
    void* y = nullptr;
    const int* row_exp = nullptr;
    const int* col_exp = nullptr;
    GemmFp32 fp32;
    long long ldr = 0, ldz = 0, ldy = 0;
    float alpha = 1.0f;
    int act = EBS_ACT_NONE;
};

// v * 2^e without an overflow on the way.
__device__ __forceinline__ float scale_pow2(float v, int e) {
    e = e < -252 ? -252 : e;                               // (nothing of a sum below 2^100 is left there)
    const int h = e >> 1;
    return v * __int_as_float((h + 127) << 23) * __int_as_float((e - h + 127) << 23);
}
// 16 bytes of elements of a row, of which `left` exist; vec: they all do, and the address is a multiple of 16 bytes.
template <typename T> struct Pack { static constexpr int N = 16 / sizeof(T); };
template <typename T>
__device__ __forceinline__ uint4 load_raw(const T* p, int left, bool vec) {
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
    if (vec) return *reinterpret_cast<const uint4*>(p);
    T* e = reinterpret_cast<T*>(&u);
#pragma unroll
    for (int i = 0; i < Pack<T>::N; ++i)
        if (i < left) e[i] = p[i];
    return u;
}
template <typename T>
__device__ __forceinline__ void unpack(const uint4& u, float (&v)[16 / sizeof(T)]) {
    const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
    for (int i = 0; i < Pack<T>::N; ++i) v[i] = to_f32(e[i]);
}
template <typename T>
__device__ __forceinline__ void load_pack(const T* p, float (&v)[16 / sizeof(T)]) {
    unpack<T>(*reinterpret_cast<const uint4*>(p), v);
}
template <typename T>
__device__ __forceinline__ void store_pack(T* p, const float (&v)[16 / sizeof(T)], int left = Pack<T>::N, bool vec = true, unsigned holes = 0u) {
    uint4 u;
    if constexpr (sizeof(T) == 2) u = make_uint4(pair_word<T>(v[0], v[1]), pair_word<T>(v[2], v[3]), pair_word<T>(v[4], v[5]), pair_word<T>(v[6], v[7]));
    else u = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    const T* e = reinterpret_cast<const T*>(&u);
    if (vec && holes == 0u) *reinterpret_cast<uint4*>(p) = u;
    else
#pragma unroll
        for (int i = 0; i < Pack<T>::N; ++i)
            if (i < left && (holes >> i & 1u) == 0u) p[i] = e[i];
}

// Packs of neighbouring columns of one row.  What a pack needs from memory is loaded ahead: what depends on the columns once for all
// rows of a thread, what depends on the row before the sums arrive.
constexpr int SCALE_PLAIN = 60;            // exponents up to this size multiply as floats: no product of two leaves the type's range
template <typename T>
struct GemmColumns {
    uint4 bias;
    int exp[sizeof(T) == 4 ? Pack<T>::N : 1];
    bool plain;
};
struct GemmAhead {
    uint4 residual;
    int row_exp;
};
template <typename T>
__device__ __forceinline__ void gemm_columns(const GemmOut& o, int col, int left, bool vec, GemmColumns<T>& c) {
    c.bias = make_uint4(0u, 0u, 0u, 0u);
    if (o.bias) c.bias = load_raw(static_cast<const T*>(o.bias) + col, left, vec);
    if constexpr (sizeof(T) == 4) {
        c.plain = true;
#pragma unroll
        for (int i = 0; i < Pack<T>::N; ++i) {
            c.exp[i] = i < left ? o.col_exp[col + i] : 0;
            c.plain = c.plain && abs(c.exp[i]) <= SCALE_PLAIN;
        }
    }
}
template <typename T>
__device__ __forceinline__ void gemm_ahead(const GemmOut& o, long long row, int col, int left, bool vec, GemmAhead& a) {
    if (o.residual) a.residual = load_raw(static_cast<const T*>(o.residual) + row * o.ldr + col, left, vec);
    if (sizeof(T) == 4) a.row_exp = o.row_exp[row];
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }
// The sum v of a row and a column with these exponents.  A hole: one of them holds an infinity and none a NaN; finish_infinite has its result.
__device__ __forceinline__ float unscale(float v, int row_exp, int col_exp, bool& hole) {
    const int e = row_exp + col_exp;
    const bool nan = row_exp == SCALE_NAN || col_exp == SCALE_NAN;
    hole = !nan && e >= SCALE_NAN / 2;
    return nan ? __int_as_float(0x7fffffff) : hole ? 0.0f : scale_pow2(v, e);
}
// Results with an infinity in their row of a or column of b: rows row0 .. row0 + rows - 1, columns col0 .. col0 + cols - 1 of fp32 results, by
// the block's first WARPS warps, which meet at named barrier BARRIER; masks: 64 words of shared memory.  Every term with an infinite factor is an infinity
// or a NaN, so that the finite ones do not matter and a result is known from two bits: whether a term is plus (or a NaN), whether one is minus
// infinity (or a NaN).  32 x 32 results at a time, the warps share the reduction; only where a value is not finite the 32 x 32 products of that place
// are looked at.  4096 x 4096 over 4096 with an infinity in every row: 35 ms, bound by reading both operands once a square.  (Summed one by one where the
// results leave it took 0.4 s and held up warps whose waits are bounded.)
template <int WARPS, int BARRIER>
static __device__ __noinline__ void finish_infinite(const GemmOut o, long long row0, int rows, int col0, int cols, unsigned* masks) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const GemmFp32 g = o.fp32;
    const int begin = (int)((long long)g.red * warp / WARPS), end = (int)((long long)g.red * (warp + 1) / WARPS);
    auto meet = [&] { asm volatile("bar.sync %0, %1;\n" ::"n"(BARRIER), "n"(WARPS * 32) : "memory"); };
    auto finite = [](float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; };
#pragma unroll 1
    for (int rb = 0; rb < rows; rb += 32)
#pragma unroll 1
        for (int cb = 0; cb < cols; cb += 32) {
            const long long row = row0 + rb + lane;
            const int col = col0 + cb + lane;
            const bool row_there = rb + lane < rows, col_there = cb + lane < cols;
            const int re = row_there ? o.row_exp[row] : 0, ce = col_there ? o.col_exp[col] : 0;
            if (!__any_sync(0xffffffffu, re == SCALE_INF || ce == SCALE_INF)) continue;       // (the same in every warp)
            meet();                                               // (the previous masks are read)
            if (warp == 0) masks[lane] = masks[32 + lane] = 0u;
            meet();
            const float *a = g.a + row * g.a_row, *b = g.b + col * g.b_col;      // lanes: rows of a, columns of b
            unsigned plus = 0u, minus = 0u;                       // of this lane's row, a bit a column
#pragma unroll 1
            for (int r = begin; r < end; r += 8) {
                const float *at = a + r * g.a_red, *bt = b + r * g.b_red;
                float av[8], bv[8];
#pragma unroll
                for (int i = 0; i < 8; ++i, at += g.a_red, bt += g.b_red) {
                    const bool there = r + i < end;
                    av[i] = there && row_there ? *at : 0.0f;
                    bv[i] = there && col_there ? *bt : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (!__any_sync(0xffffffffu, !finite(av[i]) || !finite(bv[i]))) continue;
#pragma unroll 1
                    for (int j = 0; j < 32; ++j) {
                        const float bj = __shfl_sync(0xffffffffu, bv[i], j), p = av[i] * bj;
                        const bool counts = !finite(av[i]) || !finite(bj), nan = p != p;
                        plus |= (counts && (p > 0.0f || nan) ? 1u : 0u) << j;
                        minus |= (counts && (p < 0.0f || nan) ? 1u : 0u) << j;
                    }
                }
            }
            if (plus) atomicOr(&masks[lane], plus);
            if (minus) atomicOr(&masks[32 + lane], minus);
            meet();
#pragma unroll 1
            for (int r = warp; r < 32; r += WARPS) {              // lanes: columns
                const int x = __shfl_sync(0xffffffffu, re, r);
                if (rb + r >= rows || !col_there || x == SCALE_NAN || ce == SCALE_NAN || (x != SCALE_INF && ce != SCALE_INF)) continue;
                const bool p = masks[r] >> lane & 1u, m = masks[32 + r] >> lane & 1u;
                const long long to = row0 + rb + r;
                float v = __uint_as_float(p && m ? 0x7fffffffu : p ? 0x7f800000u : 0xff800000u);
                v = fmaf(v, o.alpha, o.bias ? static_cast<const float*>(o.bias)[col] : 0.0f);
                if (o.z) static_cast<float*>(o.z)[to * o.ldz + col] = v;
                if (o.act) v = activation<false>(v, o.act);
                if (o.residual) v += static_cast<const float*>(o.residual)[to * o.ldr + col];
                static_cast<float*>(o.y)[to * o.ldy + col] = v;
            }
        }
}
// True: holes were left, elements that finish_infinite writes.
template <typename T>
__device__ __forceinline__ bool gemm_store_pack(const GemmOut& o, long long row, int col, int left, bool vec, float (&v)[16 / sizeof(T)], const GemmColumns<T>& c,
                                                const GemmAhead& a) {
    constexpr int N = Pack<T>::N;
    constexpr bool FAST = sizeof(T) == 2;
    float t[N];
    unsigned holes = 0u;
    if constexpr (sizeof(T) == 4) {
        if (c.plain && abs(a.row_exp) <= SCALE_PLAIN) {
            const float f = power_of_two(a.row_exp);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= f * power_of_two(c.exp[i]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                bool hole;
                v[i] = unscale(v[i], a.row_exp, c.exp[i], hole);
                holes |= (hole && i < left ? 1u : 0u) << i;
            }
        }
    }
    unpack<T>(c.bias, t);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = fmaf(v[i], o.alpha, t[i]);           // (alpha: a power of two, the product is exact)
    if (o.z) store_pack(static_cast<T*>(o.z) + row * o.ldz + col, v, left, vec, holes);
    switch (o.act) {                                        // (outside the loop: one branch a pack)
#define EBS_ACT_CASE(A) case A: _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = activation<FAST>(v[i], A); break;
        EBS_ACT_CASE(EBS_ACT_RELU) EBS_ACT_CASE(EBS_ACT_GELU) EBS_ACT_CASE(EBS_ACT_GELU_TANH) EBS_ACT_CASE(EBS_ACT_SILU)
#undef EBS_ACT_CASE
        default: break;
    }
    if (o.residual) {
        unpack<T>(a.residual, t);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += t[i];
    }
    store_pack(static_cast<T*>(o.y) + row * o.ldy + col, v, left, vec, holes);
    return holes != 0u;
}
// Whether every row of the outputs and of the residual starts on 16 bytes.
inline bool packs_ok(const GemmOut& o, size_t size) {
    auto ok = [&](const void* p, long long ld) { return !p || (((uintptr_t)p & 15) == 0 && (ld * (long long)size) % 16 == 0); };
    return ok(o.y, o.ldy) && ok(o.z, o.ldz) && ok(o.residual, o.ldr) && ok(o.bias, 0);
}

// An operand in memory for the tensor cores: `planes` 16-bit matrices (one behind the other, plane_stride elements apart) for
// each of `batch` (batch_stride apart), with the reduction along a row (mn_major = false: rows = the result's rows or columns) or
// across rows (mn_major = true: rows = reduction).  Base and strides are multiples of 16 bytes.
struct GemmOperand {
    const void* p = nullptr;
    long long ld = 0;
    bool mn_major = false;
    int planes = 1;
    long long plane_stride = 0, batch_stride = 0;
    GemmOperand() = default;
    GemmOperand(const void* p_, long long ld_, bool mn_major_, int planes_ = 1, long long plane_stride_ = 0, long long batch_stride_ = 0)
        : p(p_), ld(ld_), mn_major(mn_major_), planes(planes_), plane_stride(plane_stride_), batch_stride(batch_stride_) {}
};

}  // namespace ebs
