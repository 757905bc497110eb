// Orthogonalised momentum update: Newton-Schulz products of a list of matrices (see scc_orthogonal.h).
//
// Every launch runs one stage of all matrices of the list, a workgroup per 32 x 32 tile of a result.  Products are binary32 products by the
// exact three-way cut of both factors (six of nine partial products on v_mfma_f32_32x32x16_bf16, see split3): rounded to bfloat16, the usual
// form of this iteration, an error of the first steps is multiplied by up to a^steps = 484 in the directions of small singular
// values.  All factors lie in the workspace cut and in operand layout, so that a product's loop is 1 KB loads straight into
// registers and matrix instructions: panel [row tile][K step of 16][piece][lane][8 bf16], row tiles of 32, padding zero.  The tile's
// four wavefronts take the K steps in turn and add up through LDS in a fixed order.
#include "scc_orthogonal.h"

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

__device__ __forceinline__ int matrix_of(const Starts& s, int count, int& block)
{
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

__device__ __forceinline__ f32x16 product(const u32x4 (&a)[3], const u32x4 (&b)[3], f32x16 c)
{
    c = mfma(a[2], b[0], c);
    c = mfma(a[0], b[2], c);
    c = mfma(a[1], b[1], c);
    c = mfma(a[1], b[0], c);
    c = mfma(a[0], b[1], c);
    return mfma(a[0], b[0], c);
}

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

// Momentum, and the sum of the squares of u over the tile (in 64 bits: squares of binary32 values neither overflow nor vanish).
template <typename T>
__global__ __launch_bounds__(256) void ns_momentum(Batch B, Starts S, Options o, char* ws)
{
    int block = (int)blockIdx.x;
    const Matrix& m = B.mat[matrix_of(S, B.count, block)];
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

// x = u / (||u|| + eps) into both panels
template <typename T>
__global__ __launch_bounds__(256) void ns_normalise(Batch B, Starts S, Options o, char* ws)
{
    int block = (int)blockIdx.x;
    const Matrix& m = B.mat[matrix_of(S, B.count, block)];
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
    const float norm = (float)sqrt((part[0] + part[1]) + (part[2] + part[3])) + o.eps;
    const int ti = block / m.l, tj = block - ti * m.l;
    const bool flip = m.rows > m.cols;
    const int x = tid & 31, y = tid >> 5;
    for (int r = y; r < kTile; r += 8) {
        const int ii = flip ? x : r, jj = flip ? r : x;
        const int i = ti * kTile + ii, j = tj * kTile + jj;
        float v = 0.f;
        if (inside(m, i, j)) {
            const size_t at = place(m, i, j);
            v = update_of<T>(m, o, at, m.m ? m.m[at] : 0.f) / norm;
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

// One tile of p = x x^T (kGram) or q = b p + c p p (kPoly), on and above the diagonal and mirrored; or of a x + q x, into the other two panels
// (kApply) or the weights (kLast).
template <typename T, int STAGE>
__global__ __launch_bounds__(256) void ns_product(Batch B, Starts S, Options o, int from, int update, char* ws)
{
    int block = (int)blockIdx.x;
    const Matrix& m = B.mat[matrix_of(S, B.count, block)];
    const Parts parts = parts_of(m.s, m.l);
    char* const base = ws + m.at;
    int ti, tj, k_tiles;
    const char *left, *right;
    if constexpr (STAGE == kGram || STAGE == kPoly) {
        // column tj of the upper triangle holds tj + 1 tiles
        tj = (int)((sqrtf(8.f * (float)block + 1.f) - 1.f) * 0.5f);
        while (tj * (tj + 1) / 2 > block) --tj;
        while ((tj + 1) * (tj + 2) / 2 <= block) ++tj;
        ti = block - tj * (tj + 1) / 2;
        k_tiles = STAGE == kGram ? m.l : m.s;
        left = right = base + (STAGE == kGram ? parts.x[from] : parts.p);
    } else {
        ti = block / m.l;
        tj = block - ti * m.l;
        k_tiles = m.s;
        left = base + parts.q;
        right = base + parts.xt[from];
    }
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, f = lane & 31, h = lane >> 5;
    const int steps = 2 * k_tiles;
    f32x16 acc = {};
    const char* const a0 = step_of(left, ti, k_tiles, 0) + lane * 16;
    const char* const b0 = step_of(right, tj, k_tiles, 0) + lane * 16;
#pragma unroll 2
    for (int k = wave; k < steps; k += 4) {
        u32x4 a[3], b[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            a[i] = *(const u32x4*)(a0 + (size_t)k * 3072 + i * 1024);
            b[i] = *(const u32x4*)(b0 + (size_t)k * 3072 + i * 1024);
        }
        acc = product(a, b, acc);
    }
    __shared__ float partial[4][kTile * kPitch];
#pragma unroll
    for (int r = 0; r < 16; ++r) partial[wave][((r & 3) + 8 * (r >> 2) + 4 * h) * kPitch + f] = acc[r];
    __syncthreads();
    // rows 8 * wave + 4 * h + e, column f, are this lane's from here
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int at = (8 * wave + 4 * h + e) * kPitch + f;
        v[e] = (partial[0][at] + partial[1][at]) + (partial[2][at] + partial[3][at]);
    }
    if constexpr (STAGE == kLast) {
        float x[4];
        load_quad(base + parts.xt[from] + quad_at(tj, m.s, ti, wave, f, h), x);
        const float scale = update ? o.lr * sqrtf(fmaxf(1.f, (float)m.rows / (float)m.cols)) : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = ti * kTile + 8 * wave + 4 * h + e, j = tj * kTile + f;
            if (!inside(m, i, j)) continue;
            T* const w = (T*)m.w + place(m, i, j);
            const float r = fmaf(o.a, x[e], v[e]);
            *w = from_f32<T>(update ? to_f32(*w) * (1.f - o.lr * o.decay) - scale * r : r);
        }
        return;
    }
    if constexpr (STAGE == kPoly || STAGE == kApply) {
        float x[4];
        load_quad(base + (STAGE == kPoly ? parts.p : parts.xt[from]) + quad_at(tj, m.s, ti, wave, f, h), x);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = STAGE == kPoly ? fmaf(o.b, x[e], o.c * v[e]) : fmaf(o.a, x[e], v[e]);
    }
    char* const to = base + (STAGE == kGram ? parts.p : STAGE == kPoly ? parts.q : parts.xt[from ^ 1]);
    store_quad(to + quad_at(tj, m.s, ti, wave, f, h), v);          // column f as a row
    if (STAGE != kApply && ti == tj) return;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) partial[0][(8 * wave + 4 * h + e) * kPitch + f] = v[e];
    __syncthreads();
    store_rows(STAGE == kApply ? base + parts.x[from ^ 1] : to, ti, STAGE == kApply ? m.l : m.s, tj, partial[0], tid);
}

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
    Starts all, half;
    const int n = starts_of(batch, &all, [](const Matrix& m) { return m.s * m.l; });
    const int nh = starts_of(batch, &half, [](const Matrix& m) { return m.s * (m.s + 1) / 2; });
    ns_momentum<T><<<dim3(n), dim3(256), 0, st>>>(batch, all, o, ws);
    ns_normalise<T><<<dim3(n), dim3(256), 0, st>>>(batch, all, o, ws);
    for (int i = 0; i < o.steps; ++i) {
        ns_product<T, kGram><<<dim3(nh), dim3(256), 0, st>>>(batch, half, o, i & 1, 0, ws);
        ns_product<T, kPoly><<<dim3(nh), dim3(256), 0, st>>>(batch, half, o, i & 1, 0, ws);
        if (i + 1 < o.steps) ns_product<T, kApply><<<dim3(n), dim3(256), 0, st>>>(batch, all, o, i & 1, 0, ws);
        else ns_product<T, kLast><<<dim3(n), dim3(256), 0, st>>>(batch, all, o, i & 1, update ? 1 : 0, ws);
    }
    return hipGetLastError();
}

template hipError_t launch_orthogonal<float>(const Batch&, const Options&, bool, char*, hipStream_t);
template hipError_t launch_orthogonal<bf16_t>(const Batch&, const Options&, bool, char*, hipStream_t);

}  // namespace orthogonal
}  // namespace scc
