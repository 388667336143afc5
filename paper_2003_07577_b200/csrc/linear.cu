// Real-valued layers: y = act(x W^T + bias) + residual and its gradients.  See include/ebs.h.
#include "gemm.cuh"

namespace ebs {

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
static size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }

// One tensor of a call: `rows` rows of `cols` elements, `ld` elements apart.
struct Rows {
    const void* p;
    long long rows, cols, ld;
    bool out;
};

// Whether two tensors share an element.  Rows of the same stride may interleave (column ranges of one buffer).
static bool overlap(const Rows& a, const Rows& b, size_t size) {
    if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0) return false;
    const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
    const uintptr_t ea = pa + ((a.rows - 1) * a.ld + a.cols) * size, eb = pb + ((b.rows - 1) * b.ld + b.cols) * size;
    if (pa >= eb || pb >= ea) return false;
    if (a.ld != b.ld) return true;
    const long long pitch = a.ld * (long long)size;
    long long d = ((long long)(pb - pa)) % pitch;
    if (d < 0) d += pitch;
    return !(d >= a.cols * (long long)size && pitch - d >= b.cols * (long long)size);
}

// The descriptor with its strides filled in, or an error.
static int complete(const ebs_linear_desc* in, ebs_linear_desc* d) {
    if (!in) return EBS_ERR_INVALID_ARG;
    *d = *in;
    if (d->m < 0 || d->n < 1 || d->k < 1 || !real_dtype(d->dtype) || d->act < EBS_ACT_NONE || d->act > EBS_ACT_SILU)
        return EBS_ERR_INVALID_ARG;
    const long long limit = 1LL << 40;
    long long* ld[5] = {&d->ldx, &d->ldw, &d->ldy, &d->ldr, &d->ldz};
    for (int i = 0; i < 5; ++i) {
        const long long dense = i < 2 ? d->k : d->n;
        if (*ld[i] == 0) *ld[i] = dense;
        if (*ld[i] < dense) return EBS_ERR_INVALID_ARG;
        if (*ld[i] > limit / (i == 1 ? d->n : (d->m > 0 ? d->m : 1))) return EBS_ERR_OVERFLOW;
    }
    return EBS_OK;
}

static int check_tensors(const Rows* t, int count, size_t size, const Rows* same_a, const Rows* same_b) {
    for (int i = 0; i < count; ++i) {
        if (!aligned16(t[i].p)) return EBS_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j) {
            if (!t[i].out && !t[j].out) continue;
            if (((&t[i] == same_a && &t[j] == same_b) || (&t[j] == same_a && &t[i] == same_b)) && t[i].p == t[j].p && t[i].ld == t[j].ld) continue;
            if (overlap(t[i], t[j], size)) return EBS_ERR_INVALID_ARG;
        }
    }
    return EBS_OK;
}

// A half-precision dz is kept halved: the steepest slope (1.13) times the type's largest value would not fit.
static float dz_store_scale(const ebs_linear_desc& d) { return d.dtype == EBS_F16 && d.act ? 0.5f : 1.0f; }

// dz = dy * act'(z), stored times `store`, and the column sums of dz before its rounding: 32 columns a thread block, every row.
template <typename T>
__global__ void __launch_bounds__(256) linear_dz_kernel(const T* dy, long long ldy, const T* z, long long ldz, int m, int n, int act, float store, T* dz, T* dbias) {
    __shared__ float part[8][33];
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), lane_row = threadIdx.x >> 5;
    float sum = 0.0f;
    if (col < n) {
        for (long long r = lane_row; r < m; r += 8) {
            float v = to_f32(dy[r * ldy + col]);
            if (act) v *= activation_slope(to_f32(z[r * ldz + col]), act);
            if (dz) dz[r * n + col] = from_f32<T>(v * store);
            sum += v;
        }
    }
    part[lane_row][threadIdx.x & 31] = sum;
    __syncthreads();
    if (lane_row == 0 && col < n && dbias) {
        for (int i = 1; i < 8; ++i) sum += part[i][threadIdx.x];
        dbias[col] = from_f32<T>(sum);
    }
}

template <typename T>
static int launch_dz(const void* dy, const void* z, const ebs_linear_desc& d, void* dz, void* dbias, cudaStream_t st) {
    linear_dz_kernel<T><<<(d.n + 31) / 32, 256, 0, st>>>(static_cast<const T*>(dy), d.ldy, static_cast<const T*>(z), d.ldz, d.m, d.n, d.act, dz_store_scale(d), static_cast<T*>(dz), static_cast<T*>(dbias));
    return check_cuda(cudaGetLastError());
}

static size_t linear_workspace(const ebs_linear_desc& d, bool backward) {
    return backward && d.act ? round256((size_t)d.m * d.n * element_size(d.dtype)) : 0;
}

}  // namespace ebs

using namespace ebs;

extern "C" {

size_t ebs_linear_workspace_bytes(const ebs_linear_desc* desc, int backward) {
    ebs_linear_desc d;
    if (complete(desc, &d)) return 0;
    return linear_workspace(d, backward != 0);
}

int ebs_linear_forward(const void* x, const void* w, const void* bias, const void* residual, const ebs_linear_desc* desc, void* y, void* z,
                       void* workspace, size_t workspace_bytes, void* stream) {
    ebs_linear_desc d;
    const int rc = complete(desc, &d);
    if (rc) return rc;
    if (!w || (d.m > 0 && (!x || !y))) return EBS_ERR_INVALID_ARG;
    const size_t size = element_size(d.dtype), need = linear_workspace(d, false);
    if (need && (!workspace || workspace_bytes < need)) return EBS_ERR_INVALID_ARG;
    const Rows t[] = {{x, d.m, d.k, d.ldx, false}, {w, d.n, d.k, d.ldw, false}, {bias, 1, d.n, d.n, false}, {residual, d.m, d.n, d.ldr, false},
                      {y, d.m, d.n, d.ldy, true}, {z, d.m, d.n, d.ldz, true}, {need ? workspace : nullptr, 1, (long long)(need / size), (long long)(need / size), true}};
    if (check_tensors(t, 7, size, &t[3], &t[4])) return EBS_ERR_INVALID_ARG;
    if (d.m == 0) return EBS_OK;
    GemmIn in{x, w, d.ldx, 1, d.ldw, 1, 0, 0, d.m, d.n, d.k};
    GemmOut o;
    o.bias = bias; o.residual = residual; o.z = z; o.y = y; o.act = d.act;
    o.ldr = d.ldr; o.ldz = d.ldz; o.ldy = d.ldy;
    return launch_gemm(in, o, d.dtype, d.dtype, static_cast<cudaStream_t>(stream));
}

int ebs_linear_backward(const void* dy, const void* x, const void* w, const void* z, const ebs_linear_desc* desc, void* dx, void* dw, void* dbias,
                        void* workspace, size_t workspace_bytes, void* stream) {
    ebs_linear_desc d;
    int rc = complete(desc, &d);
    if (rc) return rc;
    if (!dx && !dw && !dbias && d.m > 0) return EBS_ERR_INVALID_ARG;
    if (d.m > 0 && (!dy || (dx && !w) || (dw && !x) || (d.act && !z))) return EBS_ERR_INVALID_ARG;
    const size_t size = element_size(d.dtype), need = linear_workspace(d, true);
    if (need && (!workspace || workspace_bytes < need)) return EBS_ERR_INVALID_ARG;
    const Rows t[] = {{dy, d.m, d.n, d.ldy, false}, {x, d.m, d.k, d.ldx, false}, {w, d.n, d.k, d.ldw, false}, {d.act ? z : nullptr, d.m, d.n, d.ldz, false},
                      {dx, d.m, d.k, d.ldx, true}, {dw, d.n, d.k, d.ldw, true}, {dbias, 1, d.n, d.n, true},
                      {need ? workspace : nullptr, 1, (long long)(need / size), (long long)(need / size), true}};
    if (check_tensors(t, 8, size, nullptr, nullptr)) return EBS_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const void* dz = dy;
    long long lddz = d.ldy;
    if (dbias || d.act) {
        void* out = d.act ? workspace : nullptr;
        if (d.dtype == EBS_F32) rc = launch_dz<float>(dy, z, d, out, dbias, st);
        else if (d.dtype == EBS_F16) rc = launch_dz<__half>(dy, z, d, out, dbias, st);
        else rc = launch_dz<__nv_bfloat16>(dy, z, d, out, dbias, st);
        if (rc) return rc;
        if (out) { dz = out; lddz = d.n; }
    }
    GemmOut o;
    o.alpha = 1.0f / dz_store_scale(d);
    if (dx && d.m > 0) {
        GemmIn in{dz, w, lddz, 1, 1, d.ldw, 0, 0, d.m, d.k, d.n};
        o.y = dx; o.ldy = d.ldx;
        if ((rc = launch_gemm(in, o, d.dtype, d.dtype, st))) return rc;
    }
    if (dw) {
        GemmIn in{dz, x, 1, lddz, 1, d.ldx, 0, 0, d.n, d.k, d.m};
        o.y = dw; o.ldy = d.ldw;
        if ((rc = launch_gemm(in, o, d.dtype, d.dtype, st))) return rc;
    }
    return EBS_OK;
}

}  // extern "C"
