// Host interface of the tile kernel (gemm_tile.cu).
#pragma once

#include "gemm_umma.cuh"

namespace ebs {

struct TileArgs {
    int red, out_rows, out_cols, batch;
    int tiles_a, tiles_b, blocks, split, stages;      // tile kernel: tiles along the lanes and the columns, thread blocks
    int a_mn, b_mn, bf16, packs, symmetric, chunk;
    unsigned wait_limit;
    int test_flags;
};

// D (rows x cols) = sum over red of A (rows x red) and B (cols x red); out is what becomes of it.
int launch_gemm_tile(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const GemmOut& out, int dtype, cudaStream_t st);
// Two products that do not depend on each other, in one launch where their tiles have the same form.
struct TileTask {
    GemmOperand a, b;
    GemmShape s;
};
int launch_gemm_tiles(const TileTask (&t)[2], const GemmOut (&out)[2], int dtype, cudaStream_t st);
int launch_gemm_tile(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const PlanesOut& out, cudaStream_t st);
int launch_gemm_tile(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const FinalOut& out, int dtype, cudaStream_t st);

// How a product is run: the pair kernel on tiles of 256 x tn, with its reduction in `split` parts that meet in `scratch` bytes of memory, or the tile kernel.
struct GemmRoute {
    bool pair = false;
    int tn = 256, split = 1;                // columns of a tile, parts
    size_t scratch = 0;
};
GemmRoute gemm_route(const GemmShape& s, int planes);
int launch_gemm_pair(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const GemmRoute& r, float* scratch, const GemmOut& out, int dtype, cudaStream_t st);
int launch_gemm_pair(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const GemmRoute& r, float* scratch, const PlanesOut& out, cudaStream_t st);
int launch_gemm_pair(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const GemmRoute& r, float* scratch, const FinalOut& out, int dtype, cudaStream_t st);

// y = x W^T for one row of x of 16-bit values, or up to four of fp32; all operands as they are.
int launch_gemm_rows(const void* x, long long ldx, const void* w, long long ldw, int m, int n, int k, const GemmOut& o, int dtype, cudaStream_t st);

// scratch: gemm_route(s, planes).scratch bytes.
template <class... A>
inline int launch_gemm(const GemmOperand& a, const GemmOperand& b, const GemmShape& s, float* scratch, const A&... rest) {
    const GemmRoute r = gemm_route(s, a.planes);
    return r.pair ? launch_gemm_pair(a, b, s, r, scratch, rest...) : launch_gemm_tile(a, b, s, rest...);
}

}  // namespace ebs
