// Cross entropy over a vocabulary and its gradients, without the logits in memory.
//
// The loss: one product x W^T on the matrix cores, of which every tile leaves the maximum and the sum of exponentials of its rows of the
// vocabulary for each token; these are joined per token.  The gradients: the vocabulary in pieces; for each piece the product again, whose
// tiles leave p = exp(l - lse) - [target] in the workspace, and then both p W and p^T x in one launch.  Four products of 2 T C V operations,
// where keeping the logits would take three and T V values of memory.
//
// bf16 tensors: the logits' products are exact in binary32.  The gradients' products are of fp16 values: p, in [-1, 1], as 2^14 p, and x and w
// with a power of two for each channel, which leaves the sum over tokens (the vocabulary) as a factor.  fp16 keeps 3 bits more of p than bf16,
// so that the gradients are rounded once in effect, at their end; of x and w it keeps all bits from 2^-31 of a channel's largest value up.
// binary32 tensors: all factors are cut exactly into three bf16 pieces, and six of nine products are taken (as in scc_forward).
#include "scc_vocabulary.h"
#include "scc_vocabulary_product.h"

namespace scc {
namespace vocabulary {
namespace {

constexpr float kLog2E = 1.4426950408889634f;
constexpr float kRaise = 14.f;              // p is stored as 2^14 p in fp16

enum Reduction { NONE = 0, SUM = 1, MEAN = 2 };

__device__ __forceinline__ uint16_t half_of(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }

// v as three bf16 values whose sum it is
__device__ __forceinline__ void cut(float v, uint16_t (&piece)[3])
{
    const uint32_t b = __float_as_uint(v);
    piece[0] = (uint16_t)(b >> 16);
    const float r = v - __uint_as_float(b & 0xffff0000u);
    const uint32_t c = __float_as_uint(r);
    piece[1] = (uint16_t)(c >> 16);
    piece[2] = (uint16_t)(__float_as_uint(r - __uint_as_float(c & 0xffff0000u)) >> 16);
}

__device__ __forceinline__ float power(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// k of the 2^k that brings a channel's largest value into [2^14, 2^15), fp16's last binade but one
__device__ __forceinline__ int channel_exponent(uint32_t most)
{
    const float m = __uint_as_float(most);
    const int k = __builtin_amdgcn_frexp_expf(m) - 15;
    return m > 0.f && m <= 3.4028235e38f ? (k < -110 ? -110 : k > 110 ? 110 : k) : 0;
}

// The tokens that count, in their order; one workgroup.  lse: of the tokens of x, or null; none: losses of the others, or null.
__global__ __launch_bounds__(1024) void find_tokens(const long long* __restrict__ target, long long ignored, const float* __restrict__ lse, Tokens k,
                                                    float* none, float* none_lse, uint32_t* clear, int cleared, int T)
{
    __shared__ int sums[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0;
    for (int i = threadIdx.x; i < cleared; i += 1024) clear[i] = 0;
    for (int first = 0; first < T; first += 1024) {
        const int t = first + (int)threadIdx.x;
        const long long y = t < T ? target[t] : ignored;
        const bool counts = y != ignored;
        const unsigned long long there = __ballot(counts);
        if (lane == 0) sums[wave] = __popcll(there);
        __syncthreads();
        int at = before + __popcll(there & ((1ull << lane) - 1));
        for (int i = 0; i < 16; ++i) {
            if (i < wave) at += sums[i];
            before += sums[i];
        }
        __syncthreads();
        if (counts) {
            k.order[at] = t;
            k.target[at] = y;
            if (lse) k.lse[at] = lse[t];
        }
        if (t < T) {
            k.place[t] = counts ? at : -1;
            if (none && !counts) none[t] = 0.f;
            if (none_lse && !counts) none_lse[t] = 0.f;
        }
    }
    const int end = (int)padded(before);
    for (int i = before + threadIdx.x; i < end; i += 1024) {
        k.order[i] = -1;
        k.target[i] = -1;
        k.lse[i] = 0.f;
        k.known[i] = 0.f;
    }
    if (threadIdx.x == 0) *k.count = before;
}

// What a packed token's row (or a row of w: no order) is multiplied by
struct Factor {
    const float* dloss;             // null: 1
    const int *order, *count;
    int reduction;
    __device__ __forceinline__ float of(int i) const
    {
        if (!dloss) return 1.f;
        if (order && order[i] < 0) return 0.f;
        return reduction == NONE ? dloss[order[i]] : reduction == SUM ? dloss[0] : dloss[0] / (float)*count;
    }
};

// x seen as rows of C values, row i being token order[i] (no order: row i of a plain matrix)
template <typename T>
struct Rows {
    const T* x;
    const int *order, *count;
    long long rows, C, HW;
    __device__ __forceinline__ long long end() const { return order ? *count : rows; }
    // f(row, channel, value) over 64 rows and 64 channels with 256 threads; value 0 outside.  by_row: lanes along the rows (tokens as columns)
    __device__ __forceinline__ bool by_row() const { return HW > 1; }
    __device__ __forceinline__ float at(long long i, long long c, long long last) const
    {
        if (i >= last || c >= C) return 0.f;
        const long long t = order ? order[i] : i, n = HW > 1 ? t / HW : t;
        return to_f32(x[(n * C + c) * HW + (t - n * HW)]);
    }
};

// most[c] = largest |value| of channel c, as the bits of a binary32 value: non-negative ones are ordered as their bits are
template <typename T>
__global__ __launch_bounds__(256) void channel_maxima(Rows<T> x, Factor f, uint32_t* __restrict__ most)
{
    const long long first = (long long)blockIdx.y * 256, end = x.end();
    if (first >= end) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (x.by_row()) {
        for (int r = 0; r < 256; r += 64) {
            const long long i = first + r + lane;
            const float d = i < end ? f.of((int)i) : 0.f;
            for (int j = 0; j < 16; ++j) {
                const long long c = (long long)blockIdx.x * 64 + wave * 16 + j;
                float v = fabsf(x.at(i, c, end) * d);
                for (int m = 1; m < 64; m *= 2) v = fmaxf(v, __shfl_xor(v, m));
                if (lane == 0 && c < x.C) atomicMax(most + c, __float_as_uint(v));
            }
        }
    } else {
        const long long c = (long long)blockIdx.x * 64 + lane;
        float v = 0.f;
        for (int r = wave; r < 256 && first + r < end; r += 4) v = fmaxf(v, fabsf(x.at(first + r, c, end) * f.of((int)(first + r))));
        if (c < x.C) atomicMax(most + c, __float_as_uint(v));
    }
}

// Rows into operands: `whole`, ld values a row, the value itself (PLANES 1: as bf16, 3: cut), and `scaled`, times its row's factor and its channel's
// power of two, in fp16.  Rows up to the next multiple of `pad` and channels up to ld are zeros.
template <typename T, int PLANES>
__global__ __launch_bounds__(256) void pack(Rows<T> x, Factor f, uint16_t* __restrict__ whole, long long plane, uint16_t* __restrict__ scaled,
                                            const uint32_t* __restrict__ most, int ld, int pad)
{
    __shared__ float tile[64][65];
    const long long first = (long long)blockIdx.y * 64, end = x.end();
    if (first >= (end + pad - 1) / pad * pad) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long c0 = (long long)blockIdx.x * 64;
    if (x.by_row()) {
        for (int j = 0; j < 16; ++j) tile[lane][wave * 16 + j] = x.at(first + lane, c0 + wave * 16 + j, end);
    } else {
        for (int j = 0; j < 16; ++j) tile[wave * 16 + j][lane] = x.at(first + wave * 16 + j, c0 + lane, end);
    }
    __syncthreads();
    const long long c = c0 + lane;
    const float unit = scaled ? power(-channel_exponent(c < x.C ? most[c] : 0)) : 0.f;
    for (int j = 0; j < 16; ++j) {
        const long long i = first + wave * 16 + j;
        const float v = tile[wave * 16 + j][lane];
        if (whole) {
            uint16_t piece[3];
            cut(v, piece);
#pragma unroll
            for (int p = 0; p < PLANES; ++p) whole[p * plane + i * ld + c] = piece[p];
        }
        if (scaled) scaled[i * ld + c] = half_of(v == 0.f ? 0.f : v * f.of((int)i) * unit);
    }
}

// The target's logit of each packed token, a wavefront each; with `minus`, exp(known - lse) - 1 instead.  A target outside of the vocabulary: NaN.
template <typename T, int PLANES>
__global__ __launch_bounds__(256) void target_logits(const uint16_t* __restrict__ xp, long long plane, int ld, const T* __restrict__ w, Tokens k,
                                                     bool minus, int C, int V)
{
    const int i = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (i >= *k.count) return;
    const long long y = k.target[i];
    const bool valid = y >= 0 && y < V;
    const T* row = w + (valid ? y : 0) * C;
    float sum = 0.f;
    for (int c = lane; c < C; c += 64) {
        float v = 0.f;
#pragma unroll
        for (int p = PLANES - 1; p >= 0; --p) v += to_f32((bf16_t)xp[p * plane + (long long)i * ld + c]);
        sum = fmaf(v, to_f32(row[c]), sum);
    }
    for (int m = 1; m < 64; m *= 2) sum += __shfl_xor(sum, m);
    if (!valid) sum = __uint_as_float(0x7fc00000u);
    if (lane == 0) k.known[i] = minus ? expm1f(sum - k.lse[i]) : sum;
}

// Workgroup -> tile.  Workgroups go to the XCDs in turn, and each of these takes a run of tiles: bands of four tiles of rows, all columns of a band.
struct Grid {
    int rows, columns;
};

__device__ __forceinline__ void tile_of(int block, const Grid& g, int& row, int& column)
{
    const int total = g.rows * g.columns, each = (total + 7) / 8;
    const int id = (block & 7) * each + (block >> 3);
    if ((block >> 3) >= each || id >= total) {
        row = -1;
        return;
    }
    const int band = id / (4 * g.columns), in = id - band * 4 * g.columns;
    const int high = g.rows - band * 4 < 4 ? g.rows - band * 4 : 4;
    column = in / high;
    row = band * 4 + in - column * high;
}

int blocks_of(const Grid& g) { return ((long long)g.rows * g.columns + 7) / 8 * 8; }

// Logits of a tile: rows of the vocabulary, columns are tokens.  part[tile row][token] = (max, sum of exp(l - max))
template <typename P>
__global__ __launch_bounds__(256, 2) void loss_product(Operand w, Operand x, const int* __restrict__ count, float2* __restrict__ part, long long Tp,
                                                       int steps, int V, Grid g)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    int row, column;
    tile_of(blockIdx.x, g, row, column);
    if (row < 0 || column * P::kN >= *count) return;
    f32x16 acc[P::FM][P::FN];
    P::run(w, x, (long long)row * P::kM, (long long)column * P::kN, 0, steps, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
    const int v0 = row * P::kM + wm * 32 * P::FM + 4 * (lane >> 5);
    if (row * P::kM + P::kM > V)
#pragma unroll
        for (int m = 0; m < P::FM; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (v0 + m * 32 + 8 * (r / 4) + r % 4 >= V)
#pragma unroll
                    for (int n = 0; n < P::FN; ++n) acc[m][n][r] = -__builtin_inff();
    float* most = (float*)lds;                  // [2][kN], then sums likewise
    float* sums = most + 2 * P::kN;
    float high[P::FN];
#pragma unroll
    for (int n = 0; n < P::FN; ++n) {
        high[n] = -__builtin_inff();
#pragma unroll
        for (int m = 0; m < P::FM; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) high[n] = fmaxf(high[n], acc[m][n][r]);
        high[n] = fmaxf(high[n], __shfl_xor(high[n], 32));
        if (lane < 32) most[wm * P::kN + (wn * P::FN + n) * 32 + lane] = high[n];
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < P::FN; ++n) {
        const int at = (wn * P::FN + n) * 32 + (lane & 31);
        high[n] = fmaxf(most[at], most[P::kN + at]);
        const float shift = -high[n] * kLog2E;
        float sum = 0.f;
#pragma unroll
        for (int m = 0; m < P::FM; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(fmaf(acc[m][n][r], kLog2E, shift));
        sum += __shfl_xor(sum, 32);
        if (lane < 32) sums[wm * P::kN + at] = sum;
    }
    __syncthreads();
    if (threadIdx.x < P::kN) {
        const int at = threadIdx.x;
        part[row * Tp + column * P::kN + at] = make_float2(fmaxf(most[at], most[P::kN + at]), sums[at] + sums[P::kN + at]);
    }
}

// lse and loss of 64 packed tokens from the tiles' parts; losses: of the tokens of x
__global__ __launch_bounds__(256) void join_parts(const float2* __restrict__ part, long long Tp, int tiles, Tokens k, float* __restrict__ losses,
                                                  float* __restrict__ lse)
{
    __shared__ float2 lds[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * 64 + lane, count = *k.count;
    if (blockIdx.x * 64 >= count) return;
    float high = -__builtin_inff(), sum = 0.f;
    auto join = [&](float2 p) {
        const float to = fmaxf(high, p.x);
        // a part without a finite value (-inf, 0 or NaN) has no say in the maximum
        sum = (sum == 0.f ? 0.f : sum * exp2f((high - to) * kLog2E)) + (p.y == 0.f ? 0.f : p.y * exp2f((p.x - to) * kLog2E));
        high = to;
    };
    for (int t = wave; t < tiles; t += 4) join(part[t * Tp + i]);
    lds[wave][lane] = make_float2(high, sum);
    __syncthreads();
    if (wave || i >= count) return;
    for (int t = 1; t < 4; ++t)
        if (t < tiles) join(lds[t][lane]);
    const float rest = logf(sum), all = high + rest;
    const int at = k.order[i];
    // of a token that is sure of its target the loss is what is left of rest: high = known
    losses[at] = rest + (high - k.known[i]);
    lse[at] = isnan(k.known[i]) ? k.known[i] : all;       // also where the target is outside of the vocabulary
}

// The sum or mean of T losses; one workgroup, in a fixed order
__global__ __launch_bounds__(1024) void sum_losses(const float* __restrict__ losses, const int* __restrict__ count, bool mean, float* __restrict__ out, int T)
{
    __shared__ double lds[16];
    double sum = 0.0;
    for (int i = threadIdx.x; i < T; i += 1024) sum += (double)losses[i];
    for (int m = 1; m < 64; m *= 2) sum += __shfl_xor(sum, m);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 1; i < 16; ++i) sum += lds[i];
    *out = (float)(mean ? sum / (double)(*count > 0 ? *count : 1) : sum);
}

// p of a tile of a piece of the vocabulary: p[token][v - first]
template <typename P>
__global__ __launch_bounds__(256, 2) void share_product(Operand w, Operand x, Tokens k, Factor f, uint16_t* __restrict__ p, long long plane,
                                                        int piece, int steps, int first, int V, Grid g)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    constexpr bool kCut = P::kPlanes == 3;
    int row, column;
    tile_of(blockIdx.x, g, row, column);
    if (row < 0 || column * P::kN >= *k.count) return;
    f32x16 acc[P::FM][P::FN];
    P::run(w, x, (long long)first + row * P::kM, (long long)column * P::kN, 0, steps, lds, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
    const int v0 = row * P::kM + wm * 32 * P::FM + 4 * (lane >> 5);
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int n = 0; n < P::FN; ++n) {
        const long long t = (long long)column * P::kN + (wn * P::FN + n) * 32 + (lane & 31);
        const float shift = (kCut ? 0.f : kRaise) - k.lse[t] * kLog2E;
        const float d = kCut ? f.of((int)t) : 1.f;
#pragma unroll
        for (int m = 0; m < P::FM; ++m)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int v = v0 + m * 32 + 8 * q;
                u16x4 o[P::kPlanes];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float share = __builtin_amdgcn_exp2f(fmaf(acc[m][n][4 * q + e], kLog2E, shift));
                    if (first + v + e >= V) share = 0.f;
                    if constexpr (kCut) {
                        uint16_t c[3];
                        cut(share * d, c);
#pragma unroll
                        for (int i = 0; i < 3; ++i) o[i][e] = c[i];
                    } else {
                        o[0][e] = half_of(share);
                    }
                }
#pragma unroll
                for (int i = 0; i < P::kPlanes; ++i) *(u16x4*)(p + i * plane + t * piece + v) = o[i];
            }
    }
    // the target's own, from its logit: exp(l - lse) - 1
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x < P::kN) {
        const long long t = (long long)column * P::kN + threadIdx.x;
        const long long v = k.target[t] - first - row * P::kM;
        if (t < *k.count && v >= 0 && v < P::kM) {
            uint16_t* to = p + t * piece + row * P::kM + v;
            if constexpr (kCut) {
                uint16_t c[3];
                cut(k.known[t] * f.of((int)t), c);
#pragma unroll
                for (int i = 0; i < 3; ++i) to[i * plane] = c[i];
            } else {
                *to = half_of(k.known[t] * (float)(1 << (int)kRaise));
            }
        }
    }
}

struct Gradients {
    Operand w, x, p_tokens, p_rows;     // across: w, x, p as K x rows; along: p as rows of tokens
    const int* count;
    float* dx;                          // [split][token][ld]
    long long dx_plane;
    void* dw;
    const uint32_t *most_x;             // null: no powers of two
    int ld, C, V, first, piece;         // the piece begins at row `first` of the vocabulary
    int split, split_steps, steps;      // of K = piece
    bool wide, begins;                  // dw in binary32; the first piece
    Grid gx, gw;
    int blocks_x;                       // of the grid; the others are dw's
};

// p W: rows are channels, columns tokens, K a part of the piece; and p^T x: rows are channels, columns the piece's rows, K the tokens
template <typename PX, typename PW>
__global__ __launch_bounds__(256, 2) void gradient_products(Gradients a)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    if ((int)blockIdx.x < a.blocks_x) {
        Grid g = a.gx;
        const int each = a.blocks_x / a.split, part = blockIdx.x / each;
        int row, column;
        tile_of(blockIdx.x - part * each, g, row, column);
        if (row < 0 || column * PX::kN >= *a.count) return;
        const int from = part * a.split_steps, left = a.steps - from;
        f32x16 acc[PX::FM][PX::FN];
        PX::run(a.w, a.p_tokens, (long long)row * PX::kM, (long long)column * PX::kN, (long long)from * PX::kK,
                left < a.split_steps ? left : a.split_steps, lds, acc);
#pragma unroll
        for (int n = 0; n < PX::FN; ++n) {
            const long long t = (long long)column * PX::kN + (wn * PX::FN + n) * 32 + (lane & 31);
#pragma unroll
            for (int m = 0; m < PX::FM; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = row * PX::kM + (wm * PX::FM + m) * 32 + 4 * (lane >> 5) + 8 * q;
                    if (c >= a.ld) continue;
                    f32x4* to = (f32x4*)(a.dx + part * a.dx_plane + t * a.ld + c);
                    f32x4 v = {acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]};
                    if (!a.begins) v += *to;
                    *to = v;
                }
        }
        return;
    }
    int row, column;
    tile_of(blockIdx.x - a.blocks_x, a.gw, row, column);
    if (row < 0) return;
    f32x16 acc[PW::FM][PW::FN];
    PW::run(a.x, a.p_rows, (long long)row * PW::kM, (long long)column * PW::kN, 0, (*a.count + PW::kK - 1) / PW::kK, lds, acc);
#pragma unroll
    for (int m = 0; m < PW::FM; ++m)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = row * PW::kM + (wm * PW::FM + m) * 32 + 4 * (lane >> 5) + 8 * q;
            float unit[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                unit[e] = a.most_x && c + e < a.C ? power(channel_exponent(a.most_x[c + e]) - (int)kRaise) : 1.f;
#pragma unroll
            for (int n = 0; n < PW::FN; ++n) {
                const int in = column * PW::kN + (wn * PW::FN + n) * 32 + (lane & 31);
                const long long v = a.first + in;
                if (v >= a.V || in >= a.piece) continue;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (c + e >= a.C) continue;
                    const float s = acc[m][n][4 * q + e] * unit[e];
                    if (a.wide) ((float*)a.dw)[v * a.C + c + e] = s;
                    else ((bf16_t*)a.dw)[v * a.C + c + e] = from_f32<bf16_t>(s);
                }
            }
        }
}

// dx of 64 tokens of x and 64 channels from the parts of p W
template <typename T>
__global__ __launch_bounds__(256) void join_dx(const float* __restrict__ parts, long long plane, int split, int ld, Tokens k, Factor f,
                                               const uint32_t* __restrict__ most, T* __restrict__ dx, long long tokens, int C, long long HW)
{
    __shared__ float tile[64][65];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long first = (long long)blockIdx.y * 64, c = (long long)blockIdx.x * 64 + lane;
    const float unit = most ? power(channel_exponent(c < C ? most[c] : 0) - (int)kRaise) : 1.f;
    for (int j = 0; j < 16; ++j) {
        const long long t = first + wave * 16 + j;
        const int i = t < tokens ? k.place[t] : -1;
        float sum = 0.f;
        if (i >= 0 && c < C) {
            for (int s = 0; s < split; ++s) sum += parts[s * plane + (long long)i * ld + c];
            sum *= most ? f.of(i) * unit : 1.f;
        }
        if (HW > 1) tile[wave * 16 + j][lane] = sum;
        else if (t < tokens && c < C) dx[t * C + c] = from_f32<T>(sum);
    }
    if (HW == 1) return;
    __syncthreads();
    const long long t = first + lane, n = t / HW;
    if (t >= tokens) return;
    for (int j = 0; j < 16; ++j) {
        const long long channel = (long long)blockIdx.x * 64 + wave * 16 + j;
        if (channel < C) dx[(n * C + channel) * HW + (t - n * HW)] = from_f32<T>(tile[lane][wave * 16 + j]);
    }
}

// ---- sizes ----

constexpr int kRowsPad = 256;               // rows of the vocabulary in a workspace end at a multiple of this

long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }

template <typename T> constexpr int kPlanesOf = sizeof(T) == 4 ? 3 : 1;

template <typename T, int BM, int BN> using LossProduct = Product<BM, BN, (sizeof(T) == 4 && (BM > 64)) ? 16 : 32, kPlanesOf<T>, false, false, false>;
template <typename T, int BM, int BN> using DxProduct = Product<BM, BN, (sizeof(T) == 4 && (BM > 64)) ? 16 : 32, kPlanesOf<T>, sizeof(T) == 2, true, false>;
template <typename T, int BM, int BN> using DwProduct = Product<BM, BN, (sizeof(T) == 4 && (BM > 64)) ? 16 : 32, kPlanesOf<T>, sizeof(T) == 2, true, true>;

// f(BM, BN) as constants: tiles of the product; few tokens: small ones, so that there are enough
template <typename T, typename F>
auto with_tiles(long long tokens, F&& f)
{
    typedef std::integral_constant<int, 64> small;
    typedef std::integral_constant<int, 128> middle;
    typedef std::integral_constant<int, sizeof(T) == 4 ? 128 : 256> large;
    if (tokens <= 64) return f(small(), small());
    return f(large(), middle());
}

template <typename T> bool direct(const T* w, const Shape& s) { return sizeof(T) == 2 && s.C % 64 == 0 && ((uintptr_t)w & 15u) == 0; }

struct Common {
    Tokens k;
    uint16_t* xp;
    long long ld, Tp;
};

Common take_common(Room& room, const Shape& s, int planes)
{
    Common c;
    const long long T = s.T();
    c.Tp = padded(T);
    c.ld = round_up(s.C, 64);
    c.k.order = room.take<int>(c.Tp);
    c.k.place = room.take<int>(T);
    c.k.count = room.take<int>(1);
    c.k.target = room.take<long long>(c.Tp);
    c.k.known = room.take<float>(c.Tp);
    c.k.lse = room.take<float>(c.Tp);
    c.xp = room.take<uint16_t>(planes * c.Tp * c.ld);
    return c;
}

struct LossRoom {
    Common c;
    uint16_t* wp;
    float2* part;
    float* losses;
};

// direct: w is read where it is
LossRoom take_loss(Room& room, const Shape& s, int planes, bool direct_w, int reduction)
{
    LossRoom r;
    r.c = take_common(room, s, planes);
    r.wp = direct_w ? nullptr : room.take<uint16_t>(planes * round_up(s.V, kRowsPad) * r.c.ld);
    r.part = room.take<float2>(round_up(s.V, 64) / 64 * r.c.Tp);
    r.losses = reduction == NONE ? nullptr : room.take<float>(s.T());
    return r;
}

struct Pieces {
    long long piece;
    int count;
};

// Pieces of the vocabulary: at most so many values of p at a time (in the last-level cache with both of its uses), equally long
Pieces pieces_of(const Shape& s, int planes)
{
    const long long Tp = padded(s.T()), Vp = round_up(s.V, kRowsPad), most = planes == 3 ? 1ll << 25 : 1ll << 26;
    long long piece = most / Tp / kRowsPad * kRowsPad;
    if (piece < 2048) piece = 2048;
    const long long count = (Vp + piece - 1) / piece;
    return {round_up((Vp + count - 1) / count, kRowsPad), (int)count};
}

template <typename T>
int split_of(const Shape& s, long long piece, int BM, int BN)
{
    const long long ld = round_up(s.C, 64), Tp = padded(s.T());
    const long long tiles = ((ld + BM - 1) / BM) * ((Tp + BN - 1) / BN), others = ((ld + BM - 1) / BM) * (piece / BN);
    long long split = (piece + Tp - 1) / Tp;                // as many steps as the other product's
    while (tiles * split + others < 512 && piece / split > 1024) ++split;
    if (split > 16) split = 16;
    while (split > 1 && piece / split < 256) --split;
    return (int)split;
}

struct GradientRoom {
    Common c;
    uint16_t *wp, *ws, *xs, *p;
    uint32_t *most_x, *most_w;
    float* parts;
    Pieces pieces;
    int split;
};

template <typename T>
GradientRoom take_gradients(Room& room, const Shape& s, bool direct_w)
{
    constexpr int planes = kPlanesOf<T>;
    GradientRoom r = {};
    r.c = take_common(room, s, planes);
    const long long rows = round_up(s.V, kRowsPad);
    r.wp = direct_w ? nullptr : room.take<uint16_t>(planes * rows * r.c.ld);
    if (planes == 1) {
        r.ws = room.take<uint16_t>(rows * r.c.ld);
        r.xs = room.take<uint16_t>(r.c.Tp * r.c.ld);
        r.most_x = room.take<uint32_t>(2 * s.C);
        r.most_w = r.most_x + s.C;
    }
    r.pieces = pieces_of(s, planes);
    r.p = room.take<uint16_t>(planes * r.c.Tp * r.pieces.piece);
    r.split = with_tiles<T>(s.T(), [&](auto bm, auto bn) { return split_of<T>(s, r.pieces.piece, decltype(bm)::value, decltype(bn)::value); });
    r.parts = room.take<float>(r.split * r.c.Tp * r.c.ld);
    return r;
}

template <typename T>
Operand vocabulary_rows(const T* w, const uint16_t* wp, const Shape& s, long long ld)
{
    if (wp) return {wp, round_up(s.V, kRowsPad) * ld, ld, round_up(s.V, kRowsPad) - 1};
    return {(const uint16_t*)w, 0, s.C, (long long)s.V - 1};
}

template <typename K>
hipError_t allow(K* kernel, int bytes)
{
    return bytes > 65536 ? hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) : hipSuccess;
}

}  // namespace

size_t loss_workspace(const Shape& s, int es, bool aligned, int reduction)
{
    Room room = {nullptr};
    (void)take_loss(room, s, es == 4 ? 3 : 1, es == 2 && s.C % 64 == 0 && aligned, reduction);
    return room.used;
}

template <typename T>
hipError_t launch_loss(const T* x, const T* w, const long long* target, long long ignored, int reduction, float* loss, float* lse, const Shape& s,
                       char* workspace, hipStream_t st)
{
    constexpr int planes = kPlanesOf<T>;
    Room room = {workspace};
    const bool at_place = direct(w, s);
    const LossRoom r = take_loss(room, s, planes, at_place, reduction);
    const Tokens& k = r.c.k;
    const long long T_ = s.T(), ld = r.c.ld, Tp = r.c.Tp;
    float* losses = reduction == NONE ? loss : r.losses;
    find_tokens<<<1, 1024, 0, st>>>(target, ignored, nullptr, k, losses, lse, nullptr, 0, (int)T_);
    const Rows<T> rows = {x, k.order, k.count, T_, s.C, s.HW};
    pack<T, planes><<<dim3(ld / 64, Tp / 64), 256, 0, st>>>(rows, Factor{}, r.c.xp, Tp * ld, nullptr, nullptr, (int)ld, kPad);
    if (r.wp) {
        const long long Vp = round_up(s.V, kRowsPad);
        const Rows<T> all = {w, nullptr, nullptr, s.V, s.C, 1};
        pack<T, planes><<<dim3(ld / 64, Vp / 64), 256, 0, st>>>(all, Factor{}, r.wp, Vp * ld, nullptr, nullptr, (int)ld, kRowsPad);
    }
    target_logits<T, planes><<<(T_ + 3) / 4, 256, 0, st>>>(r.c.xp, Tp * ld, (int)ld, w, k, false, s.C, s.V);
    int tiles = 0;
    const hipError_t e = with_tiles<T>(T_, [&](auto bm, auto bn) {
        typedef LossProduct<T, decltype(bm)::value, decltype(bn)::value> P;
        const Grid g = {(int)((s.V + P::kM - 1) / P::kM), (int)((T_ + P::kN - 1) / P::kN)};
        tiles = g.rows;
        const hipError_t e = allow(loss_product<P>, P::kLds);
        if (e != hipSuccess) return e;
        const Operand b = {r.c.xp, Tp * ld, ld, Tp - 1};
        loss_product<P><<<blocks_of(g), 256, P::kLds, st>>>(vocabulary_rows(w, r.wp, s, ld), b, k.count, r.part, Tp, (int)(ld / P::kK), s.V, g);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    join_parts<<<(T_ + 63) / 64, 256, 0, st>>>(r.part, Tp, tiles, k, losses, lse);
    if (reduction != NONE) sum_losses<<<1, 1024, 0, st>>>(losses, k.count, reduction == MEAN, loss, (int)T_);
    return hipGetLastError();
}

size_t gradients_workspace(const Shape& s, int es)
{
    Room room = {nullptr};
    if (es == 4) (void)take_gradients<float>(room, s, false);
    else (void)take_gradients<bf16_t>(room, s, false);
    return room.used;
}

template <typename T>
hipError_t launch_gradients(const T* x, const T* w, const long long* target, long long ignored, int reduction, const float* lse, const float* dloss,
                            T* dx, void* dw, bool wide, const Shape& s, char* workspace, hipStream_t st)
{
    constexpr int planes = kPlanesOf<T>;
    Room room = {workspace};
    const GradientRoom r = take_gradients<T>(room, s, direct(w, s));
    const Tokens& k = r.c.k;
    const long long T_ = s.T(), ld = r.c.ld, Tp = r.c.Tp, Vp = round_up(s.V, kRowsPad), piece = r.pieces.piece;
    const Factor f = {dloss, k.order, k.count, reduction};
    find_tokens<<<1, 1024, 0, st>>>(target, ignored, lse, k, nullptr, nullptr, r.most_x, planes == 1 ? 2 * s.C : 0, (int)T_);
    const Rows<T> rows = {x, k.order, k.count, T_, s.C, s.HW}, all = {w, nullptr, nullptr, s.V, s.C, 1};
    if (planes == 1) {
        channel_maxima<T><<<dim3(ld / 64, (T_ + 255) / 256), 256, 0, st>>>(rows, f, r.most_x);
        channel_maxima<T><<<dim3(ld / 64, (s.V + 255) / 256), 256, 0, st>>>(all, Factor{}, r.most_w);
    }
    pack<T, planes><<<dim3(ld / 64, Tp / 64), 256, 0, st>>>(rows, f, r.c.xp, Tp * ld, r.xs, r.most_x, (int)ld, kPad);
    if (planes == 1 || r.wp)
        pack<T, planes><<<dim3(ld / 64, Vp / 64), 256, 0, st>>>(all, Factor{}, r.wp, Vp * ld, r.ws, r.most_w, (int)ld, kRowsPad);
    target_logits<T, planes><<<(T_ + 3) / 4, 256, 0, st>>>(r.c.xp, Tp * ld, (int)ld, w, k, true, s.C, s.V);
    int parts = 1;                          // of p W: the first piece, the longest, has the most
    const hipError_t e = with_tiles<T>(T_, [&](auto bm, auto bn) {
        constexpr int BM = decltype(bm)::value, BN = decltype(bn)::value;
        typedef LossProduct<T, BM, BN> P;
        typedef DxProduct<T, BM, BN> PX;
        typedef DwProduct<T, BM, BN> PW;
        hipError_t e = allow(share_product<P>, P::kLds);
        if (e == hipSuccess) e = allow(gradient_products<PX, PW>, PX::kLds);
        for (int i = 0; i < r.pieces.count && e == hipSuccess; ++i) {
            const long long first = i * piece, length = Vp - first < piece ? Vp - first : piece;
            if (length <= 0) break;
            const int columns = (int)((T_ + BN - 1) / BN);
            const Grid g = {(int)(length / BM), columns};
            const Operand b = {r.c.xp, Tp * ld, ld, Tp - 1};
            share_product<P><<<blocks_of(g), 256, P::kLds, st>>>(vocabulary_rows(w, r.wp, s, ld), b, k, f, r.p, Tp * piece, (int)piece,
                                                               (int)(ld / P::kK), (int)first, s.V, g);
            Gradients a = {};
            const uint16_t *ws = planes == 3 ? r.wp : r.ws, *xs = planes == 3 ? r.c.xp : r.xs;
            a.w = {ws + first * ld, Vp * ld, ld, ld - 8};
            a.x = {xs, Tp * ld, ld, ld - 8};
            a.p_tokens = {r.p, Tp * piece, piece, Tp - 1};
            a.p_rows = {r.p, Tp * piece, piece, piece - 8};
            a.count = k.count;
            a.dx = r.parts;
            a.dx_plane = Tp * ld;
            a.dw = dw;
            a.most_x = r.most_x;
            a.ld = (int)ld;
            a.C = s.C;
            a.V = s.V;
            a.first = (int)first;
            a.piece = (int)length;
            a.steps = (int)(length / PX::kK);
            a.split = r.split;
            a.split_steps = (a.steps + r.split - 1) / r.split;
            a.split = (a.steps + a.split_steps - 1) / a.split_steps;
            if (i == 0) parts = a.split;
            a.wide = wide;
            a.begins = i == 0;
            a.gx = {(int)((ld + BM - 1) / BM), columns};
            a.gw = {(int)((ld + BM - 1) / BM), (int)(length / BN)};
            a.blocks_x = blocks_of(a.gx) * a.split;
            gradient_products<PX, PW><<<a.blocks_x + blocks_of(a.gw), 256, PX::kLds, st>>>(a);
            e = hipGetLastError();
        }
        return e;
    });
    if (e != hipSuccess) return e;
    join_dx<T><<<dim3(ld / 64, (T_ + 63) / 64), 256, 0, st>>>(r.parts, Tp * ld, parts, (int)ld, k, f, r.most_w, dx, T_, s.C, s.HW);
    return hipGetLastError();
}

#define INSTANCE(T)                                                                                                                        \
    template hipError_t launch_loss<T>(const T*, const T*, const long long*, long long, int, float*, float*, const Shape&, char*,          \
                                       hipStream_t);                                                                                       \
    template hipError_t launch_gradients<T>(const T*, const T*, const long long*, long long, int, const float*, const float*, T*, void*,   \
                                            bool, const Shape&, char*, hipStream_t);
INSTANCE(float)
INSTANCE(bf16_t)

}  // namespace vocabulary
}  // namespace scc
