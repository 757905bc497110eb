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

// Which panels a stage multiplies: rows of `left` by rows of `right`, over k_tiles
struct Factors {
    const char *left, *right;
    int k_tiles;
};

template <int STAGE>
__device__ __forceinline__ Factors factors_of(const Matrix& m, const Parts& parts, const char* base, int from)
{
    if constexpr (STAGE == kGram) return {base + parts.x[from], base + parts.x[from], m.l};
    else if constexpr (STAGE == kPoly) return {base + parts.p, base + parts.p, m.s};
    else return {base + parts.q, base + parts.xt[from], m.s};
}

// block-th pair (i, j), i <= j, of the upper triangle: column j holds j + 1 of them
__device__ __forceinline__ void triangle(int block, int& i, int& j)
{
    j = (int)((sqrtf(8.f * (float)block + 1.f) - 1.f) * 0.5f);
    while (j * (j + 1) / 2 > block) --j;
    while ((j + 1) * (j + 2) / 2 <= block) ++j;
    i = block - j * (j + 1) / 2;
}

// Four sums of a tile's column f, rows 8 * q + 4 * h + e, to what the stage makes of them: into the panel that has columns as rows (or the
// weights); v is then what was stored.
template <typename T, int STAGE>
__device__ __forceinline__ void finish_quad(const Matrix& m, const Parts& parts, char* base, const Options& o, int from, int update, int ti,
                                            int tj, int q, int f, int h, float (&v)[4])
{
    const size_t at = quad_at(tj, m.s, ti, q, f, h);
    if constexpr (STAGE != kGram) {
        float x[4];
        load_quad(base + (STAGE == kPoly ? parts.p : parts.xt[from]) + at, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = STAGE == kPoly ? fmaf(o.b, x[e], o.c * v[e]) : fmaf(o.a, x[e], v[e]);
    }
    if constexpr (STAGE == kLast) {
        const float scale = update ? o.lr * sqrtf(fmaxf(1.f, (float)m.rows / (float)m.cols)) : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = ti * kTile + 8 * q + 4 * h + e, j = tj * kTile + f;
            if (!inside(m, i, j)) continue;
            T* const w = (T*)m.w + place(m, i, j);
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

// One 32 x 32 tile of p = x x^T (kGram) or q = b p + c p p (kPoly), on and above the diagonal and mirrored; or of a x + q x, into the other two
// panels (kApply) or the weights (kLast).  The wavefronts take the K steps in turn, four steps' loads in flight each.
constexpr int kSplit = 8;

template <typename T, int STAGE>
__global__ __launch_bounds__(64 * kSplit) void ns_product(Batch B, Starts S, Options o, int from, int update, char* ws)
{
    int block = (int)blockIdx.x;
    const Matrix& m = B.mat[matrix_of(S, B.count, block)];
    const Parts parts = parts_of(m.s, m.l);
    char* const base = ws + m.at;
    int ti, tj;
    if constexpr (STAGE == kGram || STAGE == kPoly) {
        triangle(block, ti, tj);
    } else {
        ti = block / m.l;
        tj = block - ti * m.l;
    }
    const Factors F = factors_of<STAGE>(m, parts, base, from);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, f = lane & 31, h = lane >> 5;
    const int steps = 2 * F.k_tiles;
    f32x16 acc = {};
    const char* const a0 = step_of(F.left, ti, F.k_tiles, 0) + lane * 16;
    const char* const b0 = step_of(F.right, tj, F.k_tiles, 0) + lane * 16;
#pragma unroll 4
    for (int k = wave; k < steps; k += kSplit) {
        u32x4 a[3], b[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            a[i] = *(const u32x4*)(a0 + (size_t)k * 3072 + i * 1024);
            b[i] = *(const u32x4*)(b0 + (size_t)k * 3072 + i * 1024);
        }
        acc = product(a, b, acc);
    }
    __shared__ float partial[kSplit][kTile * kPitch];
#pragma unroll
    for (int r = 0; r < 16; ++r) partial[wave][((r & 3) + 8 * (r >> 2) + 4 * h) * kPitch + f] = acc[r];
    __syncthreads();
    // the first four wavefronts' lanes: rows 8 * wave + 4 * h + e, column f
    float v[4];
    if (wave < 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int at = (8 * wave + 4 * h + e) * kPitch + f;
            v[e] = 0.f;
#pragma unroll
            for (int i = 0; i < kSplit; ++i) v[e] += partial[i][at];
        }
        finish_quad<T, STAGE>(m, parts, base, o, from, update, ti, tj, wave, f, h, v);
    }
    if (STAGE == kLast || (STAGE != kApply && ti == tj)) return;
    __syncthreads();
    if (wave < 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) partial[0][(8 * wave + 4 * h + e) * kPitch + f] = v[e];
    }
    __syncthreads();
    store_rows(rows_of<STAGE>(parts, base, from), ti, STAGE == kApply ? m.l : m.s, tj, partial[0], tid);
}

// The same in blocks of 4 x 4 tiles, for lists with enough of them: four wavefronts of 2 x 2 tiles share a K step's 24 KB through LDS, two
// buffers, one barrier a step; the loads of the step after the next are in flight meanwhile.
constexpr int kBlock = 4;

template <typename T, int STAGE>
__global__ __launch_bounds__(256, 2) void ns_product_wide(Batch B, Starts S, Options o, int from, int update, char* ws)
{
    __shared__ __attribute__((aligned(16))) char lds[2][2 * kBlock * 3072];
    int block = (int)blockIdx.x;
    const Matrix& m = B.mat[matrix_of(S, B.count, block)];
    const Parts parts = parts_of(m.s, m.l);
    char* const base = ws + m.at;
    int bi, bj;
    if constexpr (STAGE == kGram || STAGE == kPoly) {
        triangle(block, bi, bj);
    } else {
        const int across = (m.l + kBlock - 1) / kBlock;
        bi = block / across;
        bj = block - bi * across;
    }
    const Factors F = factors_of<STAGE>(m, parts, base, from);
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, f = lane & 31, h = lane >> 5;
    const int steps = 2 * F.k_tiles;
    const int rows_l = m.s, rows_r = STAGE == kGram || STAGE == kPoly ? m.s : m.l;      // tiles of either factor

    // a wavefront fetches two of the eight tiles' steps; tiles past the edge are the last one's again, and not stored
    const char* src[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int which = 2 * wave + i, r = (which < kBlock ? bi * kBlock + which : bj * kBlock + which - kBlock);
        src[i] = which < kBlock ? step_of(F.left, r < rows_l ? r : rows_l - 1, F.k_tiles, 0) : step_of(F.right, r < rows_r ? r : rows_r - 1, F.k_tiles, 0);
        src[i] += lane * 16;
    }
    u32x4 next[2][6];
    auto fetch = [&](int set, int k) {
        k = k < steps ? k : steps - 1;
#pragma unroll
        for (int i = 0; i < 6; ++i) next[set][i] = *(const u32x4*)(src[i / 3] + (size_t)k * 3072 + i % 3 * 1024);
    };
    auto park = [&](int set, int buffer) {
#pragma unroll
        for (int i = 0; i < 6; ++i) *(u32x4*)(lds[buffer] + (2 * wave + i / 3) * 3072 + i % 3 * 1024 + lane * 16) = next[set][i];
    };
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i >> 1][i & 1] = f32x16{};
    const int wi = wave >> 1, wj = wave & 1;
    auto multiply = [&](int buffer) {
        u32x4 a[2][3], b[2][3];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                a[i][p] = *(const u32x4*)(lds[buffer] + (2 * wi + i) * 3072 + p * 1024 + lane * 16);
                b[i][p] = *(const u32x4*)(lds[buffer] + (kBlock + 2 * wj + i) * 3072 + p * 1024 + lane * 16);
            }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = product(a[i], b[j], acc[i][j]);
    };
    fetch(0, 0);
    fetch(1, 1);
    park(0, 0);
    for (int k = 0; k < steps; k += 2) {        // steps is even
        __syncthreads();
        fetch(0, k + 2);
        multiply(0);
        park(1, 1);
        __syncthreads();
        fetch(1, k + 3);
        multiply(1);
        park(0, 0);
    }
    __syncthreads();
    float* const tile = (float*)lds + wave * kTile * kPitch;       // a wavefront's own
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int ti = bi * kBlock + 2 * wi + i, tj = bj * kBlock + 2 * wj + j;
            if (ti >= rows_l || tj >= rows_r || ((STAGE == kGram || STAGE == kPoly) && ti > tj)) continue;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e];
                finish_quad<T, STAGE>(m, parts, base, o, from, update, ti, tj, q, f, h, v);
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
    Starts all, half, wide_all, wide_half;
    const int n = starts_of(batch, &all, [](const Matrix& m) { return m.s * m.l; });
    const int nh = starts_of(batch, &half, [](const Matrix& m) { return m.s * (m.s + 1) / 2; });
    auto blocks = [](int tiles) { return (tiles + kBlock - 1) / kBlock; };
    const int nw = starts_of(batch, &wide_all, [&](const Matrix& m) { return blocks(m.s) * blocks(m.l); });
    const int nwh = starts_of(batch, &wide_half, [&](const Matrix& m) { return blocks(m.s) * (blocks(m.s) + 1) / 2; });
    const bool wide = nwh >= 96;
    ns_momentum<T><<<dim3(n), dim3(256), 0, st>>>(batch, all, o, ws);
    ns_normalise<T><<<dim3(n), dim3(256), 0, st>>>(batch, all, o, ws);
    for (int i = 0; i < o.steps; ++i) {
        const bool last = i + 1 == o.steps;
        const int from = i & 1, up = update ? 1 : 0;
        if (wide) {
            ns_product_wide<T, kGram><<<dim3(nwh), dim3(256), 0, st>>>(batch, wide_half, o, from, 0, ws);
            ns_product_wide<T, kPoly><<<dim3(nwh), dim3(256), 0, st>>>(batch, wide_half, o, from, 0, ws);
            if (last) ns_product_wide<T, kLast><<<dim3(nw), dim3(256), 0, st>>>(batch, wide_all, o, from, up, ws);
            else ns_product_wide<T, kApply><<<dim3(nw), dim3(256), 0, st>>>(batch, wide_all, o, from, 0, ws);
        } else {
            constexpr int threads = 64 * kSplit;
            ns_product<T, kGram><<<dim3(nh), dim3(threads), 0, st>>>(batch, half, o, from, 0, ws);
            ns_product<T, kPoly><<<dim3(nh), dim3(threads), 0, st>>>(batch, half, o, from, 0, ws);
            if (last) ns_product<T, kLast><<<dim3(n), dim3(threads), 0, st>>>(batch, all, o, from, up, ws);
            else ns_product<T, kApply><<<dim3(n), dim3(threads), 0, st>>>(batch, all, o, from, 0, ws);
        }
    }
    return hipGetLastError();
}

template hipError_t launch_orthogonal<float>(const Batch&, const Options&, bool, char*, hipStream_t);
template hipError_t launch_orthogonal<bf16_t>(const Batch&, const Options&, bool, char*, hipStream_t);

}  // namespace orthogonal
}  // namespace scc
