// What the two forms of the orthogonalisation share.
#pragma once

#include "gemm_tile.cuh"

namespace ebs {

constexpr int ORTHO_MAX_STEPS = 64;

// Factors of a step's three products, with the powers of two its matrices are kept with: A = gram * sum, b I + c A = linear * sum +
// linear_diag I, Q = square * sum + square_diag I, X = next * sum; or from A's planes themselves, Q = quadratic * sum + direct * A + square_diag I.
struct OrthoFactors {
    float gram[ORTHO_MAX_STEPS], linear[ORTHO_MAX_STEPS], linear_diag[ORTHO_MAX_STEPS], square[ORTHO_MAX_STEPS], square_diag[ORTHO_MAX_STEPS], next[ORTHO_MAX_STEPS];
    float quadratic[ORTHO_MAX_STEPS], direct[ORTHO_MAX_STEPS];
};

// Matrices whose planes fit in the shared memory of a cluster of thread blocks (short side at most 128).
bool ortho_small_fits(int rows, int cols);
// first: power of two of the first X; last: scale of the result over the last product (steps = 0: over X).
int launch_ortho_small(const void* g, void* out, int batch, int rows, int cols, int dtype, int steps, float eps, float first, float last, const OrthoFactors& f, cudaStream_t st);

}  // namespace ebs
