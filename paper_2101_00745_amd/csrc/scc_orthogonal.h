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

// What a workgroup of a product needs to know, one load from the workspace: the first launch writes these for the others.
struct Block {
    uint32_t at;            // of the matrix in the workspace, in units of 256 bytes
    int s, l;               // tiles of the matrix
    int bi, bj;             // the block
    int matrix;             // in the list
    int unused[2];
};

// A batch's workspace: the matrices' descriptions, the blocks of both kinds of products (at most a tile each), then the matrices' parts.
struct Layout {
    size_t half, whole, matrices;
};

inline Layout layout_of(size_t half_tiles, size_t tiles)
{
    Layout o;
    o.half = (kBatch * sizeof(Matrix) + 255) / 256 * 256;
    o.whole = o.half + (half_tiles * sizeof(Block) + 255) / 256 * 256;
    o.matrices = o.whole + (tiles * sizeof(Block) + 255) / 256 * 256;
    return o;
}

struct Options {
    float lr, momentum, decay, a, b, c, eps;
    int nesterov, steps;
};

// update: w is read and moved; else O(u) is written over it.  The workspace begins with the batch's layout_of.
template <typename T>
hipError_t launch_orthogonal(const Batch& batch, const Options& o, bool update, char* workspace, hipStream_t st);

}  // namespace orthogonal
}  // namespace scc
