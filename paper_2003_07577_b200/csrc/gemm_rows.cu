// Products with a few rows: y = x W^T for one row of x of 16-bit values, or up to four of fp32, bound by the bytes of W.
//
// A warp takes R rows of W over the whole reduction; its lanes run along them with 16-byte loads, the next ones on their way while these are
// multiplied.  x comes from the first-level cache (it is the same for every warp); sums are fp32 multiply-adds: a weight is used once per row
// of x, too seldom for the tensor core's tiles to pay.
#include "gemm_tile.cuh"

namespace ebs {

constexpr int ROWS_WARPS = 4;

template <typename T, int M, int R, bool VEC>
__global__ void __launch_bounds__(ROWS_WARPS * 32) gemm_rows_kernel(const T* __restrict__ x, long long ldx, const T* __restrict__ w, long long ldw, int m, int n, int k, const GemmOut o) {
    constexpr int N = VEC ? Pack<T>::N : 1, U = M <= 2 ? 8 / R : 4 / R;    // U packs of R rows at a time, twice
    let_next_kernel_start();
    wait_for_previous_kernel();
    const int lane = threadIdx.x & 31, row0 = (int)(blockIdx.x * ROWS_WARPS + (threadIdx.x >> 5)) * R;
    if (row0 >= n) return;
    float acc[M][R];
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int r = 0; r < R; ++r) acc[i][r] = 0.0f;
    const T* rows[R];                                             // (rows past the end: the last one once more)
#pragma unroll
    for (int r = 0; r < R; ++r) rows[r] = w + (long long)(row0 + r < n ? row0 + r : n - 1) * ldw;
    const T* xr[M];                                               // (rows of x past the last likewise)
#pragma unroll
    for (int i = 0; i < M; ++i) xr[i] = x + (long long)(i < m ? i : m - 1) * ldx;
    const int packs = k / N;
    auto load = [&](int p0, uint4 (&raw)[U][R]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = p0 + u * 32;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                raw[u][r] = make_uint4(0u, 0u, 0u, 0u);
                if (p >= packs) continue;
                if constexpr (VEC) raw[u][r] = __ldcs(reinterpret_cast<const uint4*>(rows[r] + (size_t)p * N));
                else raw[u][r].x = __float_as_uint(to_f32(rows[r][p]));
            }
        }
    };
    // every load of x before the first multiplication: one wait, not one a row
    auto multiply = [&](int p0, const uint4 (&raw)[U][R]) {
        uint4 xs[U][M];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int p = p0 + u * 32 < packs ? p0 + u * 32 : 0;
#pragma unroll
            for (int i = 0; i < M; ++i) {
                if constexpr (VEC) xs[u][i] = *reinterpret_cast<const uint4*>(xr[i] + (size_t)p * N);
                else xs[u][i].x = __float_as_uint(to_f32(xr[i][p]));
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (p0 + u * 32 >= packs) break;                      // (zero weights would turn an infinite x into NaN)
            float wv[R][N];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if constexpr (VEC) unpack<T>(raw[u][r], wv[r]);
                else wv[r][0] = __uint_as_float(raw[u][r].x);
            }
#pragma unroll
            for (int i = 0; i < M; ++i) {
                float xv[N];
                if constexpr (VEC) unpack<T>(xs[u][i], xv);
                else xv[0] = __uint_as_float(xs[u][i].x);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int e = 0; e < N; ++e) acc[i][r] = fmaf(wv[r][e], xv[e], acc[i][r]);
            }
        }
    };
    uint4 here[U][R], next[U][R];
    load(lane, here);
    for (int p0 = lane; p0 < packs; p0 += 2 * U * 32) {
        load(p0 + U * 32, next);
        multiply(p0, here);
        load(p0 + 2 * U * 32, here);
        multiply(p0 + U * 32, next);
    }
    if (VEC && packs * N + lane < k) {                            // what is left of a row
        const int c = packs * N + lane;
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const float xv = to_f32(xr[i][c]);
#pragma unroll
            for (int r = 0; r < R; ++r) acc[i][r] = fmaf(to_f32(rows[r][c]), xv, acc[i][r]);
        }
    }
    float mine = 0.0f;                                            // lane i * R + r keeps the sum of (i, r)
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float v = acc[i][r];
#pragma unroll
            for (int s = 16; s > 0; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
            if (lane == i * R + r) mine = v;
        }
    const int row = lane / R, col = row0 + lane % R;
    if (lane >= M * R || row >= m || col >= n) return;
    float v = mine;
    if (o.bias) v += to_f32(static_cast<const T*>(o.bias)[col]);
    if (o.z) static_cast<T*>(o.z)[row * o.ldz + col] = from_f32<T>(v);
    if (o.act) v = activation<sizeof(T) == 2>(v, o.act);
    if (o.residual) v += to_f32(static_cast<const T*>(o.residual)[row * o.ldr + col]);
    static_cast<T*>(o.y)[row * o.ldy + col] = from_f32<T>(v);
}

template <typename T, int M, int R>
static int launch_rows_shape(const void* x, long long ldx, const void* w, long long ldw, int m, int n, int k, const GemmOut& o, cudaStream_t st) {
    const bool vec = ldx % Pack<T>::N == 0 && ldw % Pack<T>::N == 0;
    const long long warps = (n + R - 1LL) / R;
    return launch_chained(vec ? gemm_rows_kernel<T, M, R, true> : gemm_rows_kernel<T, M, R, false>, dim3((unsigned)((warps + ROWS_WARPS - 1) / ROWS_WARPS)), ROWS_WARPS * 32, 0, st, 1,
                          static_cast<const T*>(x), ldx, static_cast<const T*>(w), ldw, m, n, k, o);
}
// One row of W a warp until every SM has 16 warps, then two: x is read half as often.
template <typename T, int M>
static int launch_rows(const void* x, long long ldx, const void* w, long long ldw, int m, int n, int k, const GemmOut& o, cudaStream_t st) {
    if (n <= 16 * 148) return launch_rows_shape<T, M, 1>(x, ldx, w, ldw, m, n, k, o, st);
    return launch_rows_shape<T, M, 2>(x, ldx, w, ldw, m, n, k, o, st);
}
template <typename T>
static int launch_rows_typed(const void* x, long long ldx, const void* w, long long ldw, int m, int n, int k, const GemmOut& o, cudaStream_t st) {
    if (m == 1) return launch_rows<T, 1>(x, ldx, w, ldw, m, n, k, o, st);
    if constexpr (sizeof(T) == 4) {
        if (m == 2) return launch_rows<T, 2>(x, ldx, w, ldw, m, n, k, o, st);
        if (m <= 4) return launch_rows<T, 4>(x, ldx, w, ldw, m, n, k, o, st);
    }
    return EBS_ERR_UNSUPPORTED;                                   // (the caller asks for no other)
}
int launch_gemm_rows(const void* x, long long ldx, const void* w, long long ldw, int m, int n, int k, const GemmOut& o, int dtype, cudaStream_t st) {
    if (dtype == EBS_F32) return launch_rows_typed<float>(x, ldx, w, ldw, m, n, k, o, st);
    if (dtype == EBS_F16) return launch_rows_typed<__half>(x, ldx, w, ldw, m, n, k, o, st);
    return launch_rows_typed<__nv_bfloat16>(x, ldx, w, ldw, m, n, k, o, st);
}

}  // namespace ebs
