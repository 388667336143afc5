// Host interface of the tile kernel (gemm_tile.cu).
#pragma once

#include "gemm_umma.cuh"

namespace ebs {

constexpr int GEMM_CHUNK = 4;                 // stages (of 64 reduction elements) summed in the tensor core at a time, split products

struct TileArgs {
    int red, out_rows, out_cols;
    int split, stages;
    int a_mn, b_mn, bf16, packs;
    unsigned wait_limit;
    int test_flags;
};

// D (rows x cols) = sum over red of A (rows x red) and B (cols x red); out is what becomes of it.
int launch_gemm_tile(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const GemmOut& out, int dtype, cudaStream_t st);
int launch_gemm_tile(const GemmOperand& A, const GemmOperand& B, const GemmShape& s, const PlanesOut& out, cudaStream_t st);
unsigned long long gemm_tile_timeouts();

}  // namespace ebs
