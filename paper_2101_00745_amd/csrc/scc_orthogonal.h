// Orthogonalised momentum update of weight matrices: declarations shared by its kernels and entry points.
//
//   m <- mu m + g;   u = g + mu m (Nesterov) or m;   w <- (1 - lr wd) w - lr sqrt(max(1, rows/cols)) O(u)
// O(u): x = u / (||u||_F + eps), taken as its transpose where it has more rows than columns, then `steps` times
//   p = x x^T,   q = b p + c p p,   x <- a x + q x,
// which moves every singular value by the odd polynomial a s + b s^3 + c s^5 and leaves the singular vectors.
#pragma once
#include "scc_common.h"

namespace scc {
namespace orthogonal {

constexpr int kBatch = 40;      // matrices of one launch: their descriptions are kernel arguments (4 KB at most)
constexpr int kTile = 32;

struct Matrix {
    const void* g;
    float* m;           // null: u = g
    void* w;            // weights, or where O(u) goes
    int rows, cols;
    int s, l;           // tiles of 32 along the shorter and the longer side
    size_t at;          // of this matrix in the workspace
};

// The parts of a matrix's workspace.  x is kept in the operand layout of the matrix instruction, once with its own rows and once
// with its columns as rows; both twice, read from one and written to the other; p and q, which are symmetric, once.
struct Parts {
    size_t x[2], xt[2], p, q, sums, bytes;
};

__host__ __device__ inline size_t panel_bytes(int row_tiles, int k_tiles) { return (size_t)row_tiles * k_tiles * kTile * kTile * 6; }

__host__ __device__ inline Parts parts_of(int s, int l)
{
    Parts o;
    const size_t x = panel_bytes(s, l), p = panel_bytes(s, s);
    o.x[0] = 0;
    o.x[1] = x;
    o.xt[0] = 2 * x;
    o.xt[1] = 3 * x;
    o.p = 4 * x;
    o.q = o.p + p;
    o.sums = o.q + p;
    o.bytes = o.sums + ((size_t)s * l * 8 + 255) / 256 * 256;
    return o;
}

struct Batch {
    Matrix mat[kBatch];
    int count;
};

struct Options {
    float lr, momentum, decay, a, b, c, eps;
    int nesterov, steps;
};

// update: w is read and moved; else O(u) is written over it
template <typename T>
hipError_t launch_orthogonal(const Batch& batch, const Options& o, bool update, char* workspace, hipStream_t st);

}  // namespace orthogonal
}  // namespace scc
