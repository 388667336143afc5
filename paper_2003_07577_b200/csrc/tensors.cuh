// Host side of the real-valued operators: extents of a call's tensors, their checks, workspaces, copies of rows that no tensor copy can start on.
#pragma once

#include "gemm.cuh"

namespace ebs {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }
inline long long round8(long long v) { return (v + 7) & ~7LL; }

// One tensor of a call: `rows` rows of `cols` elements, `ld` elements apart.
struct Rows {
    const void* p;
    long long rows, cols, ld;
    bool out;
};

// Whether two tensors share an element.  Rows of the same stride may interleave (column ranges of one buffer).
inline bool overlap(const Rows& a, const Rows& b, size_t size) {
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
inline int check_tensors(const Rows* t, int count, size_t size, const Rows* same_a, const Rows* same_b) {
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

// The descriptor of a linear layer with its strides filled in, or an error (linear.cu).
int complete_linear(const ebs_linear_desc* in, ebs_linear_desc* d);

// Takes buffers out of the workspace one behind the other; without a base it only counts.
struct Carver {
    char* base;
    size_t used = 0;
    template <typename T> T* take(size_t count) {
        char* p = base ? base + used : nullptr;
        used += round256(count * sizeof(T));
        return reinterpret_cast<T*>(p);
    }
};

// Copies of 16-bit rows whose stride is a multiple of 16 bytes: up to three matrices in one launch (linear.cu).
struct CopyJobs {
    const uint16_t* src[3];
    uint16_t* dst[3];
    long long ld[3], ldd[3], first[3], pieces;                // first: pieces of the matrices before
    int cols[3], across[3], count;
};
void add_copy_rows(CopyJobs* j, const void* src, void* dst, long long rows, int cols, long long ld, long long ldd);
int launch_copies(const CopyJobs& j, cudaStream_t st);

// A half-precision dz is kept halved where a slope may exceed one: the steepest (1.13) times the type's largest value would not fit.  That costs
// dz below 2^-13 its last bit (multiples of 2^-23 instead of 2^-24); a rectified one is dy itself or zero and keeps all of them.
inline float dz_store_scale(const ebs_linear_desc& d) { return d.dtype == EBS_F16 && d.act > EBS_ACT_RELU ? 0.5f : 1.0f; }

}  // namespace ebs
