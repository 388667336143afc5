// Matrix products of the real-valued operators.
#include "gemm.cuh"

namespace ebs {

// 64 x 64 outputs a thread block, 4 x 4 a thread, the reduction 16 at a time through shared memory, sums in fp32.
template <typename T, typename TO>
__global__ void __launch_bounds__(256) gemm_kernel(const GemmIn in, const GemmOut out) {
    __shared__ float as[16][65], bs[16][65];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int j0 = blockIdx.x * 64;
    const T* a = static_cast<const T*>(in.a) + blockIdx.z * in.batch_a;
    const T* b = static_cast<const T*>(in.b) + blockIdx.z * in.batch_b;
    for (long long i0 = (long long)blockIdx.y * 64; i0 < in.rows; i0 += (long long)gridDim.y * 64) {
        float acc[4][4] = {};
        for (int r0 = 0; r0 < in.red; r0 += 16) {
            for (int e = threadIdx.x; e < 1024; e += 256) {
                // neighbouring threads along whichever index is contiguous
                const int ra = in.a_red == 1 ? e & 15 : e >> 6, ia = in.a_red == 1 ? e >> 4 : e & 63;
                as[ra][ia] = r0 + ra < in.red && i0 + ia < in.rows ? to_f32(a[(i0 + ia) * in.a_row + (r0 + ra) * in.a_red]) : 0.0f;
                const int rb = in.b_red == 1 ? e & 15 : e >> 6, jb = in.b_red == 1 ? e >> 4 : e & 63;
                bs[rb][jb] = r0 + rb < in.red && j0 + jb < in.cols ? to_f32(b[(long long)(j0 + jb) * in.b_col + (r0 + rb) * in.b_red]) : 0.0f;
            }
            __syncthreads();
            const int n = in.red - r0 < 16 ? in.red - r0 : 16;
            for (int r = 0; r < n; ++r) {
                float av[4], bv[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) { av[t] = as[r][ty + 16 * t]; bv[t] = bs[r][tx + 16 * t]; }
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int u = 0; u < 4; ++u) acc[t][u] = fmaf(av[t], bv[u], acc[t][u]);
            }
            __syncthreads();
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i0 + ty + 16 * t < in.rows && j0 + tx + 16 * u < in.cols)
                    gemm_store<TO>(out, blockIdx.z, i0 + ty + 16 * t, j0 + tx + 16 * u, acc[t][u]);
    }
}

template <typename T, typename TO>
static int launch_typed(const GemmIn& in, const GemmOut& out, cudaStream_t st) {
    const long long by = (in.rows + 63LL) / 64;
    const dim3 grid((in.cols + 63) / 64, (unsigned)(by < 65535 ? by : 65535), in.batch);
    gemm_kernel<T, TO><<<grid, 256, 0, st>>>(in, out);
    return check_cuda(cudaGetLastError());
}

int launch_gemm(const GemmIn& in, const GemmOut& out, int dtype, int out_dtype, cudaStream_t st) {
    if (dtype == EBS_F32 && out_dtype == EBS_F32) return launch_typed<float, float>(in, out, st);
    if (dtype == EBS_F32 && out_dtype == EBS_F16) return launch_typed<float, __half>(in, out, st);
    if (dtype == EBS_F32 && out_dtype == EBS_BF16) return launch_typed<float, __nv_bfloat16>(in, out, st);
    if (dtype == EBS_F16) return launch_typed<__half, __half>(in, out, st);
    return launch_typed<__nv_bfloat16, __nv_bfloat16>(in, out, st);
}

}  // namespace ebs
