// Orthogonalised momentum update: Newton-Schulz products of a list of matrices (see scc_orthogonal.h).
//
// Every launch runs one stage of all matrices of the list, a workgroup per block of 1, 2 x 2 or 4 x 4 tiles of 32 x 32 of a result.  Products are binary32 products by the
// exact three-way cut of both factors (six of nine partial products on v_mfma_f32_32x32x16_bf16, see split3): rounded to bfloat16, the usual
// form of this iteration, an error of the first steps is multiplied by up to a^steps = 484 in the directions of small singular
// values.  All factors lie in the workspace cut and in operand layout, so that a product's loop is 1 KB loads straight into
// registers (blocks of 4 x 4 tiles: through LDS) and matrix instructions: panel [row tile][K step of 16][piece][lane][8 bf16], row tiles of 32, padding zero.
// Wavefronts of small blocks take the K steps in turn and add up through LDS in a fixed order.
//
// What bounds it: three dependent launches a step and, of small lists, their latencies (256 x 64: 17 launches and 72 us; the thirteen layers
// 64x16 to 1024x512: 243 us, p 15, q 9, x 22 us a step against 8 us of matrix work); of large ones the matrix pipes (six of 1000 x 1024:
// 0.98 ms, 124 TFLOP/s of binary32 products where six matrix instructions each allow 218).
#include "scc_orthogonal.h"

#include <type_traits>

namespace scc {
namespace orthogonal {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kPitch = kTile + 1;

// first workgroup of every matrix of a launch
struct Starts {
    int at[kBatch + 1];
};

// The matrix of this workgroup, and which of its blocks; -1: no work.  Consecutive workgroups go to consecutive XCDs; each XCD takes an eighth
// of the list's blocks in a row, so that a matrix is read through one L2 or two instead of eight (its panels were written all over the
// chip by the launch before, so every L2 has to fetch what it reads).
__device__ __forceinline__ int matrix_of(const Starts& s, int count, int& block)
{
    const int each = ((int)gridDim.x + 7) / 8;
    block = ((int)blockIdx.x & 7) * each + ((int)blockIdx.x >> 3);
    if (block >= s.at[count]) return -1;
    int lo = 0, hi = count;         // the last matrix that starts at or before the block
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (s.at[mid] <= block) lo = mid;
        else hi = mid;
    }
    block -= s.at[lo];
    return lo;
}

// element (i, j) of x: of u, or of its transpose where u has more rows than columns
__device__ __forceinline__ size_t place(const Matrix& m, int i, int j)
{
    return m.rows > m.cols ? (size_t)j * m.cols + i : (size_t)i * m.cols + j;
}

__device__ __forceinline__ bool inside(const Matrix& m, int i, int j)
{
    return m.rows > m.cols ? j < m.rows && i < m.cols : i < m.rows && j < m.cols;
}

__device__ __forceinline__ f32x16 mfma(const u32x4& a, const u32x4& b, f32x16 c)
{
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// the six partial products of a cut product, smallest first: piece of the left and of the right factor
constexpr int kLeft[6] = {2, 0, 1, 1, 0, 0}, kRight[6] = {0, 2, 1, 0, 1, 0};

// Address of a panel's K step: rows of tile r, K step k of 2 * k_tiles.
__device__ __forceinline__ const char* step_of(const char* panel, int r, int k_tiles, int k)
{
    return panel + ((size_t)r * 2 * k_tiles + k) * 3072;
}

// Four consecutive K values k0 + 8*q + 4*h .. + 3 of row f: where they lie in a panel's row tile r and K tile
__device__ __forceinline__ size_t quad_at(int r, int k_tiles, int k_tile, int q, int f, int h)
{
    return ((size_t)r * 2 * k_tiles + 2 * k_tile + (q >> 1)) * 3072 + (f + 32 * (q & 1)) * 16 + 8 * h;
}

__device__ __forceinline__ void store_quad(char* at, const float (&v)[4])
{
    uint32_t hi[2], mid[2], lo[2];
    split3<4>([&](int e) { return v[e]; }, hi, mid, lo);
    *(u32x2*)at = u32x2{hi[0], hi[1]};
    *(u32x2*)(at + 1024) = u32x2{mid[0], mid[1]};
    *(u32x2*)(at + 2048) = u32x2{lo[0], lo[1]};
}

// the values that store_quad cut, exactly
__device__ __forceinline__ void load_quad(const char* at, float (&v)[4])
{
    const u32x2 hi = *(const u32x2*)at, mid = *(const u32x2*)(at + 1024), lo = *(const u32x2*)(at + 2048);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int w = e >> 1;
        auto part = [&](const u32x2& p) { return __uint_as_float(e & 1 ? p[w] & 0xffff0000u : p[w] << 16); };
        v[e] = part(hi) + (part(mid) + part(lo));
    }
}

// A 32 x 32 tile in LDS, tile[row][column], into a panel with its rows as rows: row tile r, K tile kt.
__device__ __forceinline__ void store_rows(char* panel, int r, int k_tiles, int kt, const float* tile, int tid)
{
    if (tid >= 128) return;
    const int step = tid >> 6, lane = tid & 63, f = lane & 31, h = lane >> 5;
    uint32_t hi[4], mid[4], lo[4];
    const float* const from = tile + f * kPitch + 16 * step + 8 * h;
    split3<8>([&](int e) { return from[e]; }, hi, mid, lo);
    char* const to = panel + ((size_t)r * 2 * k_tiles + 2 * kt + step) * 3072 + lane * 16;
    *(u32x4*)to = u32x4{hi[0], hi[1], hi[2], hi[3]};
    *(u32x4*)(to + 1024) = u32x4{mid[0], mid[1], mid[2], mid[3]};
    *(u32x4*)(to + 2048) = u32x4{lo[0], lo[1], lo[2], lo[3]};
}

// u at an element, from the gradient and the momentum as it is after its update
template <typename T>
__device__ __forceinline__ float update_of(const Matrix& m, const Options& o, size_t at, float momentum)
{
    const float g = to_f32(((const T*)m.g)[at]);
    return !m.m ? g : o.nesterov ? fmaf(o.momentum, momentum, g) : momentum;
}

// block-th pair (i, j), i <= j, of the upper triangle: column j holds j + 1 of them
__device__ __forceinline__ void triangle(int block, int& i, int& j)
{
    j = (int)((sqrtf(8.f * (float)block + 1.f) - 1.f) * 0.5f);
    while (j * (j + 1) / 2 > block) --j;
    while ((j + 1) * (j + 2) / 2 <= block) ++j;
    i = block - j * (j + 1) / 2;
}

__host__ __device__ inline int blocks_of(const Matrix& m, int side, bool half)
{
    const int bs = (m.s + side - 1) / side, bl = (m.l + side - 1) / side;
    return half ? bs * (bs + 1) / 2 : bs * bl;
}

// Blocks of `side` tiles of the symmetric results and of x, and where a matrix's begin in the list of all
struct Plan {
    int half_side, whole_side;
    Starts half, whole;
    Layout at;
};

// Momentum, and the sum of the squares of u over the tile (in 64 bits: squares of binary32 values neither overflow nor vanish).
template <typename T>
__global__ __launch_bounds__(256) void ns_momentum(Batch B, Starts S, Plan plan, Options o, char* ws)
{
    int block;
    const int which = matrix_of(S, B.count, block);
    if (which < 0) return;      // the whole workgroup
    const Matrix& m = B.mat[which];
    if (threadIdx.x == 0) {     // the tables of the later launches; a matrix has no more blocks than tiles
        Block b = {(uint32_t)(m.at / 256), m.s, m.l, 0, 0, which, {0, 0}};
        if (block == 0) ((Matrix*)ws)[which] = m;
        if (block < blocks_of(m, plan.half_side, true)) {
            triangle(block, b.bi, b.bj);
            ((Block*)(ws + plan.at.half))[plan.half.at[which] + block] = b;
        }
        if (block < blocks_of(m, plan.whole_side, false)) {
            const int across = (m.l + plan.whole_side - 1) / plan.whole_side;
            b.bi = block / across;
            b.bj = block - b.bi * across;
            ((Block*)(ws + plan.at.whole))[plan.whole.at[which] + block] = b;
        }
    }
    const int ti = block / m.l, tj = block - ti * m.l;
    const bool flip = m.rows > m.cols;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    double sum = 0;
    for (int r = y; r < kTile; r += 8) {
        const int i = ti * kTile + (flip ? x : r), j = tj * kTile + (flip ? r : x);      // x runs along u's rows in memory
        if (!inside(m, i, j)) continue;
        const size_t at = place(m, i, j);
        float momentum = 0.f;
        if (m.m) {
            momentum = fmaf(o.momentum, m.m[at], to_f32(((const T*)m.g)[at]));
            m.m[at] = momentum;
        }
        const float u = update_of<T>(m, o, at, momentum);
        sum += (double)u * u;
    }
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    __shared__ double part[4];
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) ((double*)(ws + m.at + parts_of(m.s, m.l).sums))[block] = (part[0] + part[1]) + (part[2] + part[3]);
}

// ||u|| + eps in binary32, times a power of two that u is to be multiplied by as well: binary32 values have norms that it does not hold, or holds
// with a few bits only.
struct Norm {
    float by, value;
};

__device__ __forceinline__ Norm norm_of(double squares, float eps)
{
    const double root = sqrt(squares);
    const float by = root > 0x1p120 ? 0x1p-64f : root < 0x1p-100 ? 0x1p64f : 1.f;
    return {by, (float)(root * by) + eps * by};
}

// u / (||u|| + eps), 0 where that is 0 / 0 (only u = 0 has a norm of 0; a NaN stays one)
__device__ __forceinline__ float normalised(float u, const Norm& n) { return n.value == 0.f ? 0.f : u * n.by / n.value; }

// x = u / (||u|| + eps) into both panels
template <typename T>
__global__ __launch_bounds__(256) void ns_normalise(Batch B, Starts S, Options o, char* ws)
{
    int block;
    const int which = matrix_of(S, B.count, block);
    if (which < 0) return;      // the whole workgroup
    const Matrix& m = B.mat[which];
    const Parts parts = parts_of(m.s, m.l);
    char* const base = ws + m.at;
    __shared__ double part[4];
    __shared__ float tile[kTile * kPitch];
    const int tid = threadIdx.x;
    double sum = 0;
    for (int i = tid; i < m.s * m.l; i += 256) sum += ((const double*)(base + parts.sums))[i];
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if ((tid & 63) == 0) part[tid >> 6] = sum;
    __syncthreads();
    const Norm norm = norm_of((part[0] + part[1]) + (part[2] + part[3]), o.eps);
    const int ti = block / m.l, tj = block - ti * m.l;
    const bool flip = m.rows > m.cols;
    const int x = tid & 31, y = tid >> 5;
    for (int r = y; r < kTile; r += 8) {
        const int ii = flip ? x : r, jj = flip ? r : x;
        const int i = ti * kTile + ii, j = tj * kTile + jj;
        float v = 0.f;
        if (inside(m, i, j)) {
            const size_t at = place(m, i, j);
            v = normalised(update_of<T>(m, o, at, m.m ? m.m[at] : 0.f), norm);
        }
        tile[ii * kPitch + jj] = v;
    }
    __syncthreads();
    store_rows(base + parts.x[0], ti, m.l, tj, tile, tid);
    const int lane = tid & 63, f = lane & 31, h = lane >> 5, q = tid >> 6;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = tile[(8 * q + 4 * h + e) * kPitch + f];
    store_quad(base + parts.xt[0] + quad_at(tj, m.s, ti, q, f, h), v);
}

enum { kGram, kPoly, kApply, kLast };

// Which panels a stage multiplies: rows of `left` by rows of `right`, over k_tiles
struct Factors {
    const char *left, *right;
    int k_tiles;
};

template <int STAGE>
__device__ __forceinline__ Factors factors_of(const Block& m, const Parts& parts, const char* base, int from)
{
    if constexpr (STAGE == kGram) return {base + parts.x[from], base + parts.x[from], m.l};
    else if constexpr (STAGE == kPoly) return {base + parts.p, base + parts.p, m.s};
    else return {base + parts.q, base + parts.xt[from], m.s};
}

// the value that a stage adds its sums to: of p, or of x
template <int STAGE>
__device__ __forceinline__ void old_quad(const Block& m, const Parts& parts, const char* base, int from, int ti, int tj, int q, int f, int h,
                                         float (&x)[4])
{
    if constexpr (STAGE != kGram) load_quad(base + (STAGE == kPoly ? parts.p : parts.xt[from]) + quad_at(tj, m.s, ti, q, f, h), x);
}

// Four sums of a tile's column f, rows 8 * q + 4 * h + e, to what the stage makes of them: into the panel that has columns as rows (or the
// weights); v is then what was stored.
template <typename T, int STAGE>
__device__ __forceinline__ void finish_quad(const Block& m, const Matrix* list, const Parts& parts, char* base, const Options& o, int from, int update, int ti,
                                            int tj, int q, int f, int h, const float (&x)[4], float (&v)[4])
{
    const size_t at = quad_at(tj, m.s, ti, q, f, h);
    if constexpr (STAGE != kGram) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = STAGE == kPoly ? fmaf(o.b, x[e], o.c * v[e]) : fmaf(o.a, x[e], v[e]);
    }
    if constexpr (STAGE == kLast) {
        const Matrix& t = list[m.matrix];
        const float scale = update ? o.lr * sqrtf(fmaxf(1.f, (float)t.rows / (float)t.cols)) : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = ti * kTile + 8 * q + 4 * h + e, j = tj * kTile + f;
            if (!inside(t, i, j)) continue;
            T* const w = (T*)t.w + place(t, i, j);
            *w = from_f32<T>(update ? to_f32(*w) * (1.f - o.lr * o.decay) - scale * v[e] : v[e]);
        }
    } else {
        store_quad(base + (STAGE == kGram ? parts.p : STAGE == kPoly ? parts.q : parts.xt[from ^ 1]) + at, v);
    }
}

// the panel that has a stage's rows as rows: the mirrored half of a symmetric result, or the other panel of x
template <int STAGE>
__device__ __forceinline__ char* rows_of(const Parts& parts, char* base, int from)
{
    return base + (STAGE == kGram ? parts.p : STAGE == kPoly ? parts.q : parts.x[from ^ 1]);
}

// The blocks of each XCD, in a row as matrix_of deals them, but of equal work: a block's is its K steps and a fixed part.
struct Shares {
    int begin[9], most;
};

// This workgroup's block; most * 8 of them are launched.
__device__ __forceinline__ bool take_block(const Block* blocks, const Shares& shares, Block& b)
{
    const int xcd = (int)blockIdx.x & 7, i = shares.begin[xcd] + ((int)blockIdx.x >> 3);
    if (i >= shares.begin[xcd + 1]) return false;
    b = blocks[i];
    return true;
}

// whether a tile of a block is to be stored: inside the result, on or above the diagonal of a symmetric one
template <int STAGE>
__device__ __forceinline__ bool wanted(const Block& m, int ti, int tj)
{
    if constexpr (STAGE == kGram || STAGE == kPoly) return tj < m.s && ti <= tj;
    else return ti < m.s && tj < m.l;
}

// One block of R x R tiles of p = x x^T (kGram) or q = b p + c p p (kPoly), on and above the diagonal and mirrored; or of a x + q x, into the other two
// panels (kApply) or the weights (kLast).  The wavefronts (eight for a tile alone, four for 2 x 2) take the K steps in turn, loads of several steps in flight each, straight
// from the panels into registers, and add up through LDS.
template <int R> constexpr int split_of = R == 1 ? 8 : 4;

template <typename T, int STAGE, int R>
__global__ __launch_bounds__(64 * split_of<R>, 2) void ns_product(const Block* blocks, Shares shares, Options o, int from, int update, char* ws)
{
    constexpr int kSplit = split_of<R>, kArea = kTile * kPitch, kParts = R == 1 ? kSplit : kSplit / 2;
    __shared__ float partial[kParts][R * R][kArea];
    Block m;
    if (!take_block(blocks, shares, m)) return;      // the whole workgroup
    const Parts parts = parts_of(m.s, m.l);
    char* const base = ws + (size_t)m.at * 256;
    const int bi = m.bi, bj = m.bj;
    const Factors F = factors_of<STAGE>(m, parts, base, from);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, f = lane & 31, h = lane >> 5;
    const int steps = 2 * F.k_tiles;
    const int rows_r = STAGE == kGram || STAGE == kPoly ? m.s : m.l;
    f32x16 acc[R][R], low[R][R];    // every other partial product on its own: two chains of dependent instructions
    const char *a0[R], *b0[R];      // tiles past the edge are the last one's again, and not stored
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int ti = bi * R + i, tj = bj * R + i;
        a0[i] = step_of(F.left, ti < m.s ? ti : m.s - 1, F.k_tiles, 0) + lane * 16;
        b0[i] = step_of(F.right, tj < rows_r ? tj : rows_r - 1, F.k_tiles, 0) + lane * 16;
#pragma unroll
        for (int j = 0; j < R; ++j) acc[i][j] = low[i][j] = f32x16{};
    }
    // a ring of steps whose loads are in flight
    constexpr int kAhead = R == 1 ? 4 : 2;
    u32x4 a[kAhead][R][3], b[kAhead][R][3];
    auto fetch = [&](int slot, int k) {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                a[slot][i][p] = *(const u32x4*)(a0[i] + (size_t)k * 3072 + p * 1024);
                b[slot][i][p] = *(const u32x4*)(b0[i] + (size_t)k * 3072 + p * 1024);
            }
    };
#pragma unroll
    for (int d = 0; d < kAhead; ++d)
        if (wave + d * kSplit < steps) fetch(d, wave + d * kSplit);
    // each wavefront finishes quads of rows of a tile: rows 8 * q + 4 * h + e, column f; what they are added to is under way
    constexpr int kQuads = R * R * 4, kRounds = (kQuads + kSplit - 1) / kSplit;
    float old[kRounds][4] = {};
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const int quad = i * kSplit + wave, t = quad / 4;
        const int ti = bi * R + t / R, tj = bj * R + t % R;
        if (quad < kQuads && wanted<STAGE>(m, ti, tj)) old_quad<STAGE>(m, parts, base, from, ti, tj, quad % 4, f, h, old[i]);
    }
    for (int k0 = wave; k0 < steps; k0 += kAhead * kSplit) {
#pragma unroll
        for (int d = 0; d < kAhead; ++d) {
            const int k = k0 + d * kSplit;
            if (k >= steps) break;
#pragma unroll
            for (int p = 0; p < 6; ++p)
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int j = 0; j < R; ++j) {
                        f32x16& to = p % 2 == 0 ? low[i][j] : acc[i][j];
                        to = mfma(a[d][i][kLeft[p]], b[d][j][kRight[p]], to);
                    }
            if (k + kAhead * kSplit < steps) fetch(d, k + kAhead * kSplit);
        }
    }
#pragma unroll
    for (int t = 0; t < R * R; ++t) acc[t / R][t % R] += low[t / R][t % R];
    auto give = [&](int to) {
#pragma unroll
        for (int t = 0; t < R * R; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) partial[to][t][((r & 3) + 8 * (r >> 2) + 4 * h) * kPitch + f] = acc[t / R][t % R][r];
    };
    if constexpr (R == 1) {
        give(wave);
    } else {        // the upper half of the wavefronts give their sums to the lower
        if (wave >= kParts) give(wave - kParts);
        __syncthreads();
        if (wave < kParts) {
#pragma unroll
            for (int t = 0; t < R * R; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[t / R][t % R][r] += partial[wave][t][((r & 3) + 8 * (r >> 2) + 4 * h) * kPitch + f];
            give(wave);     // each lane wrote the places that it read
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
        const int quad = i * kSplit + wave, t = quad / 4, q = quad % 4;
        const int ti = bi * R + t / R, tj = bj * R + t % R;
        if (quad >= kQuads || !wanted<STAGE>(m, ti, tj)) continue;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int at = (8 * q + 4 * h + e) * kPitch + f;
            // K steps w and w + 2 first, in either shape, so that short products come out the same in both
            if constexpr (R == 1) {
                v[e] = ((partial[0][t][at] + partial[2][t][at]) + (partial[1][t][at] + partial[3][t][at])) +
                       ((partial[4][t][at] + partial[6][t][at]) + (partial[5][t][at] + partial[7][t][at]));
            } else {
                v[e] = partial[0][t][at] + partial[1][t][at];
            }
        }
        finish_quad<T, STAGE>(m, (const Matrix*)ws, parts, base, o, from, update, ti, tj, q, f, h, old[i], v);
        if constexpr (STAGE != kLast) {
#pragma unroll
            for (int e = 0; e < 4; ++e) partial[0][t][(8 * q + 4 * h + e) * kPitch + f] = v[e];     // read by this lane alone until now
        }
    }
    if constexpr (STAGE != kLast) {
        __syncthreads();
        for (int t = tid / 128; t < R * R; t += kSplit / 2) {       // 128 threads a tile
            const int ti = bi * R + t / R, tj = bj * R + t % R;
            if (wanted<STAGE>(m, ti, tj) && (STAGE == kApply || ti != tj))
                store_rows(rows_of<STAGE>(parts, base, from), ti, STAGE == kApply ? m.l : m.s, tj, partial[0][t], tid % 128);
        }
    }
}

// N times a matrix instruction and one of the kind, in this order
template <int N, int KIND>
__device__ __forceinline__ void interleave()
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(KIND, 1, 0);
    }
}

// The same in blocks of 4 x 4 tiles, for lists with enough of them.  Four wavefronts of 2 x 2 tiles share a K step's 24 KB through LDS: while a
// step is multiplied from registers, the next one's operands come from LDS and the one's after that go there, in three buffers with
// one barrier a step; the global loads of the step behind it are in flight.
constexpr int kBlock = 4;

// AHEAD: steps whose loads are in flight, two where two workgroups share a CU's registers, four where a launch has one for each CU at
// most (p of six matrices of 1000 x 1024: 56 us with two, 46 with four; x, 384 workgroups: 93 and 100).
template <typename T, int STAGE, int AHEAD>
__global__ __launch_bounds__(256, AHEAD == 2 ? 2 : 1) void ns_product_wide(const Block* blocks, Shares shares, Options o, int from, int update, char* ws)
{
    constexpr int kBuffer = 2 * kBlock * 3072;
    __shared__ __attribute__((aligned(16))) char lds[3 * kBuffer];
    Block m;
    if (!take_block(blocks, shares, m)) return;      // the whole workgroup
    const Parts parts = parts_of(m.s, m.l);
    char* const base = ws + (size_t)m.at * 256;
    const int bi = m.bi, bj = m.bj;
    const Factors F = factors_of<STAGE>(m, parts, base, from);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, f = lane & 31, h = lane >> 5;
    const int steps = 2 * F.k_tiles;
    const int rows_r = STAGE == kGram || STAGE == kPoly ? m.s : m.l;

    // a wavefront fetches two of the eight tiles' steps; tiles past the edge are the last one's again, and not stored
    const char* src[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int tile = 2 * wave + i, r = tile < kBlock ? bi * kBlock + tile : bj * kBlock + tile - kBlock;
        src[i] = tile < kBlock ? step_of(F.left, r < m.s ? r : m.s - 1, F.k_tiles, 0) : step_of(F.right, r < rows_r ? r : rows_r - 1, F.k_tiles, 0);
        src[i] += lane * 16;
    }
    u32x4 next[AHEAD][6];
    auto fetch = [&](int set, int k) {
        k = k < steps ? k : steps - 1;
#pragma unroll
        for (int i = 0; i < 6; ++i) next[set][i] = *(const u32x4*)(src[i / 3] + (size_t)k * 3072 + i % 3 * 1024);
    };
    auto park = [&](int set, int buffer) {
#pragma unroll
        for (int i = 0; i < 6; ++i) *(u32x4*)(lds + buffer + (2 * wave + i / 3) * 3072 + i % 3 * 1024 + lane * 16) = next[set][i];
    };
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i >> 1][i & 1] = f32x16{};
    const int wi = wave >> 1, wj = wave & 1;
    u32x4 a[2][2][3], b[2][2][3];
    auto take = [&](int set, int buffer) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                a[set][i][p] = *(const u32x4*)(lds + buffer + (2 * wi + i) * 3072 + p * 1024 + lane * 16);
                b[set][i][p] = *(const u32x4*)(lds + buffer + (kBlock + 2 * wj + i) * 3072 + p * 1024 + lane * 16);
            }
    };
    // One chain of 6 * steps matrix instructions loses too much: five steps of six matrices of 1000 x 1024 were off by 5.1e-6 of the result's norm,
    // where plain binary32 products are off by 2.6e-6.  So the products below the first pieces' have sums of their own where there are registers for
    // them (8.4e-7); else a step's six add up from zero, and their sum goes to the steps' before on the vector unit (7.5e-7), which
    // another workgroup's matrix instructions hide (p: 46 us with the former in a workgroup a CU, 59 with the latter).
    constexpr bool kTwo = AHEAD == 4;
    f32x16 low[2][2];
    if constexpr (kTwo) {
#pragma unroll
        for (int i = 0; i < 4; ++i) low[i >> 1][i & 1] = f32x16{};
    }
    auto multiply = [&](int set) {
        if constexpr (kTwo) {
#pragma unroll
            for (int p = 0; p < 6; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        f32x16& to = p < 5 ? low[i][j] : acc[i][j];
                        to = mfma(a[set][i][kLeft[p]], b[set][j][kRight[p]], to);
                    }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f32x16 sum[2] = {};
#pragma unroll
                for (int p = 0; p < 6; ++p)
#pragma unroll
                    for (int j = 0; j < 2; ++j) sum[j] = mfma(a[set][i][kLeft[p]], b[set][j][kRight[p]], sum[j]);
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] += sum[j];
            }
        }
    };
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) fetch(d, d);
    park(0, 0);
    fetch(0, AHEAD);
    park(1, kBuffer);
    __syncthreads();
    take(0, 0);
    int now = kBuffer;              // the buffer of the step after this one
    for (int k0 = 0; k0 < steps; k0 += AHEAD) {
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            const int k = k0 + d, after = now == 2 * kBuffer ? 0 : now + kBuffer;
            if (k >= steps) break;
            fetch((d + 1) % AHEAD, k + 1 + AHEAD);
            take(1 - d % 2, now);       // step k + 1
            multiply(d % 2);
            park((d + 2) % AHEAD, after);         // step k + 2: its buffer was last read before the last barrier
            now = after;
            // One wavefront per SIMD issues in order: 24 memory instructions in a row would hold up the matrix pipe for as long as it works.
            interleave<12, 0x100>();    // LDS reads
            interleave<6, 0x020>();     // global loads
            interleave<6, 0x200>();     // LDS writes
            __syncthreads();
        }
    }
    if constexpr (kTwo) {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i >> 1][i & 1] += low[i >> 1][i & 1];
    }
    float* const tile = (float*)lds + wave * kTile * kPitch;       // a wavefront's own
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int ti = bi * kBlock + 2 * wi + i, tj = bj * kBlock + 2 * wj + j;
            if (!wanted<STAGE>(m, ti, tj)) continue;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e];
                float x[4] = {};
                old_quad<STAGE>(m, parts, base, from, ti, tj, q, f, h, x);
                finish_quad<T, STAGE>(m, (const Matrix*)ws, parts, base, o, from, update, ti, tj, q, f, h, x, v);
                if constexpr (STAGE != kLast) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) tile[(8 * q + 4 * h + e) * kPitch + f] = v[e];
                }
            }
            if (STAGE == kLast || (STAGE != kApply && ti == tj)) continue;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            char* const to = rows_of<STAGE>(parts, base, from);
            store_rows(to, ti, STAGE == kApply ? m.l : m.s, tj, tile, lane);
            store_rows(to, ti, STAGE == kApply ? m.l : m.s, tj, tile, lane + 64);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
}

// ---- small matrices: a workgroup each and all steps in one launch, x, p and q in LDS in binary32 and cut when they are read ----
//
// A launch of its own for every stage takes 3 to 4 us whatever the size: each hands its panels on through memory, three accesses of some 0.7 us
// one behind the other, and so does one workgroup that keeps them there (20 x 20, five steps: 55 us in 17 launches, 70 in one).  In LDS a stage is
// below 1 us.

constexpr int kAlone = 16;          // wavefronts

__host__ __device__ inline int alone_pitch(int tiles) { return tiles * kTile + 4; }      // rows 16 bytes apart in their banks

__host__ __device__ inline int alone_floats(int s, int l) { return s * kTile * (alone_pitch(l) + 2 * alone_pitch(s)); }

constexpr int kSlotFloats = kTile * kPitch;             // a partial tile, one for each wavefront
constexpr int kAloneFloats = 35000;                     // of LDS: what alone_preferred lets in, at most 15 tiles of x

struct Operand {
    u32x4 p[3];
};

__device__ __forceinline__ Operand cut(const float (&v)[8])
{
    uint32_t hi[4], mid[4], lo[4];
    split3<8>([&](int e) { return v[e]; }, hi, mid, lo);
    return {{u32x4{hi[0], hi[1], hi[2], hi[3]}, u32x4{mid[0], mid[1], mid[2], mid[3]}, u32x4{lo[0], lo[1], lo[2], lo[3]}}};
}

// a K step's operand: this lane's row, 8 consecutive values; or this lane's column, 8 values below one another
__device__ __forceinline__ Operand of_row(const float* at)
{
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    const f32x4 lo = *(const f32x4*)at, hi = *(const f32x4*)(at + 4);
    const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return cut(v);
}

__device__ __forceinline__ Operand of_column(const float* at, int pitch)
{
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = at[e * pitch];
    return cut(v);
}

__device__ __forceinline__ void step_product(const Operand& a, const Operand& b, f32x16& acc, f32x16& low)
{
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        low = mfma(a.p[kLeft[i]], b.p[kRight[i]], low);
        acc = mfma(a.p[kLeft[i + 3]], b.p[kRight[i + 3]], acc);
    }
}

// from x x^T: to = x x^T over k columns of x; with p: to = b p + c p p.  Several wavefronts take a tile's K steps in turn.
template <bool POLY>
__device__ __forceinline__ void alone_square(const float* x, int pitch, int k, float* to, int to_pitch, int s, const Options& o,
                                             float (*partial)[kSlotFloats])
{
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, f = lane & 31, h = lane >> 5;
    const int steps = k / 16, tiles = s * (s + 1) / 2;
    const int most = kAlone / tiles, shares = most < steps ? most : steps, share = wave / tiles;
    if (share < shares) {
        int ti, tj;
        triangle(wave % tiles, ti, tj);
        f32x16 acc = {}, low = {};
#pragma unroll 2
        for (int i = share; i < steps; i += shares) {
            const Operand a = of_row(x + (ti * kTile + f) * pitch + 16 * i + 8 * h);
            const Operand b = of_row(x + (tj * kTile + f) * pitch + 16 * i + 8 * h);
            step_product(a, b, acc, low);
        }
        acc += low;
#pragma unroll
        for (int r = 0; r < 16; ++r) partial[wave][((r & 3) + 8 * (r >> 2) + 4 * h) * kPitch + f] = acc[r];
    }
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {       // a thread an element
        static_assert(64 * kAlone == kTile * kTile, "a tile at a time");
        const int row = tid / kTile, column = tid % kTile;
        int ti, tj;
        triangle(t, ti, tj);
        float v = 0.f;
        for (int w = t; w < tiles * shares; w += tiles) v += partial[w][row * kPitch + column];
        const int i = ti * kTile + row, j = tj * kTile + column;
        if constexpr (POLY) v = fmaf(o.b, x[i * pitch + j], o.c * v);
        to[i * to_pitch + j] = v;
        if (ti != tj) to[j * to_pitch + i] = v;
    }
    __syncthreads();
}

template <typename T>
__global__ __launch_bounds__(64 * kAlone) void ns_alone(Batch B, Options o, int update)
{
    extern __shared__ __attribute__((aligned(16))) float small[];
    __shared__ double sums[kAlone];
    const Matrix& t = B.mat[blockIdx.x];
    const int s = t.s, l = t.l, xp = alone_pitch(l), pp = alone_pitch(s);
    float* const x = small;
    float* const p = x + s * kTile * xp;
    float* const q = p + s * kTile * pp;
    float(*const partial)[kSlotFloats] = (float(*)[kSlotFloats])(q + s * kTile * pp);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, f = lane & 31, h = lane >> 5;

    // u, with its padding; along u's rows in memory
    const bool flip = t.rows > t.cols;
    const int across = (flip ? s : l) * kTile, down = (flip ? l : s) * kTile;
    double sum = 0;
    for (int e = tid; e < across * down; e += 64 * kAlone) {
        const int r = e / across, c = e - r * across;
        float u = 0.f;
        if (r < t.rows && c < t.cols) {
            const size_t at = (size_t)r * t.cols + c;
            float momentum = 0.f;
            if (t.m) {
                momentum = fmaf(o.momentum, t.m[at], to_f32(((const T*)t.g)[at]));
                t.m[at] = momentum;
            }
            u = update_of<T>(t, o, at, momentum);
        }
        x[flip ? c * xp + r : r * xp + c] = u;
        sum += (double)u * u;
    }
    for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = 0;
    for (int i = 0; i < kAlone; ++i) sum += sums[i];
    const Norm norm = norm_of(sum, o.eps);
    for (int e = tid; e < s * kTile * l * kTile; e += 64 * kAlone) {
        const int i = e / (l * kTile), j = e - i * (l * kTile);
        x[i * xp + j] = normalised(x[i * xp + j], norm);
    }
    __syncthreads();

    const int tiles = s * l;
    for (int step = 0; step < o.steps; ++step) {
        alone_square<false>(x, xp, l * kTile, p, pp, s, o, partial);
        alone_square<true>(p, pp, s * kTile, q, pp, s, o, partial);
        // a x + q x: a wavefront's tile stays in registers until all have read x
        f32x16 acc = {}, low = {};
        const int ti = wave / l, tj = wave - ti * l;
        float* const tile = x + (ti * kTile + 4 * h) * xp + tj * kTile + f;
        if (wave < tiles) {
#pragma unroll 2
            for (int i = 0; i < 2 * s; ++i)
                step_product(of_row(q + (ti * kTile + f) * pp + 16 * i + 8 * h), of_column(x + (16 * i + 8 * h) * xp + tj * kTile + f, xp), acc, low);
            acc += low;
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] = fmaf(o.a, tile[((r & 3) + 8 * (r >> 2)) * xp], acc[r]);
        }
        __syncthreads();
        if (wave < tiles) {
#pragma unroll
            for (int r = 0; r < 16; ++r) tile[((r & 3) + 8 * (r >> 2)) * xp] = acc[r];
        }
        __syncthreads();
    }
    const float scale = update ? o.lr * sqrtf(fmaxf(1.f, (float)t.rows / (float)t.cols)) : 0.f;
    for (int e = tid; e < across * down; e += 64 * kAlone) {
        const int r = e / across, c = e - r * across;
        if (r < t.rows && c < t.cols) {
            T* const w = (T*)t.w + (size_t)r * t.cols + c;
            const float v = x[flip ? c * xp + r : r * xp + c];
            *w = from_f32<T>(update ? to_f32(*w) * (1.f - o.lr * o.decay) - scale * v : v);
        }
    }
}

// Lists of small matrices only, at most 15 tiles of x and 3 of p.  us for a step, all stages as launches and in one: 20 x 20 55 and 21, 86 x 29 60 and 25, 64 x 64 64 and 40 (40 K steps of
// tiles); 56 x 197 70 and 69 (78), 256 x 64 71 and 73 (124), 96 x 96 68 and 83 (126).
bool alone_preferred(const Batch& b)
{
    for (int i = 0; i < b.count; ++i) {
        const long long s = b.mat[i].s, l = b.mat[i].l;
        if (s * (s + 1) * (s + l) + 2 * s * s * l > 64) return false;
        if (s * l > kAlone || alone_floats((int)s, (int)l) + kAlone * kSlotFloats > kAloneFloats) return false;
    }
    return true;
}

// whole eighths: matrix_of
dim3 grid_of(int blocks) { return dim3((unsigned)((blocks + 7) / 8 * 8)); }

template <typename F>
int starts_of(const Batch& b, Starts* s, F&& tiles)
{
    int at = 0;
    for (int i = 0; i < b.count; ++i) {
        s->at[i] = at;
        at += tiles(b.mat[i]);
    }
    s->at[b.count] = at;
    return at;
}

}  // namespace

template <typename T>
hipError_t launch_orthogonal(const Batch& batch, const Options& o, bool update, char* ws, hipStream_t st)
{
    if (alone_preferred(batch)) {
        constexpr int lds = kAloneFloats * 4;
        static const hipError_t allowed = hipFuncSetAttribute((const void*)ns_alone<T>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (allowed != hipSuccess) return allowed;
        ns_alone<T><<<dim3((unsigned)batch.count), dim3(64 * kAlone), lds, st>>>(batch, o, update ? 1 : 0);
        return hipGetLastError();
    }
    Starts all;
    Plan plan;
    const int n = starts_of(batch, &all, [](const Matrix& m) { return m.s * m.l; });
    size_t half_tiles = 0;
    for (int i = 0; i < batch.count; ++i) half_tiles += blocks_of(batch.mat[i], 1, true);
    plan.at = layout_of(half_tiles, n);
    // Tiles of a block's side: the widest that gives enough of the CUs a workgroup, 192 of 4 x 4 tiles (they share a K step's operands among
    // four wavefronts) or more than 128 of 2 x 2.  us of a whole update.  x, sides 1 and 2: 512 x 512 (64 blocks of side 2) 117 and 146, twice (128) 175 and
    // 179, 704 x 768 (132) 188 and 168, 1000 x 1024 (256) 437 and 339, the thirteen layers (385) 284 and 242; sides 2 and 4: two of 1000 x 1024 (128 of
    // side 4) 521 and 588, three (192) equal, six (384) 1028 and 994.  p and q, sides 1 and 2: the thirteen layers (106) 242 and 260, 960 x 1024 (120)
    // equal, 1000 x 1024 (136) 340 and 287, six of 512 x 512 (216) 308 and 255; sides 2 and 4: three of 1000 x 1024 (108) 616 and 718, six (216) 1070 and 992.
    auto choose = [&](bool half, int* side, Starts* s) {
        for (*side = kBlock;; *side /= 2) {
            const int count = starts_of(batch, s, [&](const Matrix& m) { return blocks_of(m, *side, half); });
            if (*side == 1 || (*side == kBlock ? count >= 192 : count > 128)) return;
        }
    };
    choose(true, &plan.half_side, &plan.half);
    choose(false, &plan.whole_side, &plan.whole);
    // work in K steps; a block's other launches' worth of latency counts as four
    auto share = [&](const Starts& s, bool gram) {
        auto each = [&](int i) { return (long long)(gram ? batch.mat[i].l : batch.mat[i].s) + 4; };
        long long total = 0, done = 0;
        for (int i = 0; i < batch.count; ++i) total += each(i) * (s.at[i + 1] - s.at[i]);
        Shares r;
        r.most = 0;
        int i = 0;
        for (int x = 0; x < 9; ++x) {
            const long long goal = (total * x + 7) / 8;
            while (i < batch.count && done + each(i) * (s.at[i + 1] - s.at[i]) <= goal) {
                done += each(i) * (s.at[i + 1] - s.at[i]);
                ++i;
            }
            r.begin[x] = i == batch.count ? s.at[i] : s.at[i] + (int)((goal - done + each(i) - 1) / each(i));
            if (x > 0 && r.begin[x] - r.begin[x - 1] > r.most) r.most = r.begin[x] - r.begin[x - 1];
        }
        return r;
    };
    const Shares gram = share(plan.half, true), poly = share(plan.half, false), apply = share(plan.whole, false);
    ns_momentum<T><<<grid_of(n), dim3(256), 0, st>>>(batch, all, plan, o, ws);
    ns_normalise<T><<<grid_of(n), dim3(256), 0, st>>>(batch, all, o, ws);
    auto run = [&](auto stage, int from) {
        constexpr int STAGE = decltype(stage)::value;
        constexpr bool kHalf = STAGE == kGram || STAGE == kPoly;
        const int up = update ? 1 : 0, side = kHalf ? plan.half_side : plan.whole_side;
        const Block* const blocks = (const Block*)(ws + (kHalf ? plan.at.half : plan.at.whole));
        const Shares& sh = STAGE == kGram ? gram : STAGE == kPoly ? poly : apply;
        const dim3 grid(8u * (unsigned)sh.most);
        if (side == kBlock && grid.x <= 256) ns_product_wide<T, STAGE, 4><<<grid, dim3(256), 0, st>>>(blocks, sh, o, from, up, ws);
        else if (side == kBlock) ns_product_wide<T, STAGE, 2><<<grid, dim3(256), 0, st>>>(blocks, sh, o, from, up, ws);
        else if (side == 2) ns_product<T, STAGE, 2><<<grid, dim3(64 * split_of<2>), 0, st>>>(blocks, sh, o, from, up, ws);
        else ns_product<T, STAGE, 1><<<grid, dim3(64 * split_of<1>), 0, st>>>(blocks, sh, o, from, up, ws);
    };
    for (int i = 0; i < o.steps; ++i) {
        run(std::integral_constant<int, kGram>(), i & 1);
        run(std::integral_constant<int, kPoly>(), i & 1);
        if (i + 1 < o.steps) run(std::integral_constant<int, kApply>(), i & 1);
        else run(std::integral_constant<int, kLast>(), i & 1);
    }
    return hipGetLastError();
}

template hipError_t launch_orthogonal<float>(const Batch&, const Options&, bool, char*, hipStream_t);
template hipError_t launch_orthogonal<bf16_t>(const Batch&, const Options&, bool, char*, hipStream_t);

}  // namespace orthogonal
}  // namespace scc
