// Cross entropy over a vocabulary and its gradients, without the logits in memory.
//
// The loss: one product x W^T on the matrix cores, of which every tile leaves the maximum and the sum of exponentials of its rows of the
// vocabulary for each token; these are joined per token.  The gradients: the vocabulary in pieces; for each piece the product again, whose
// tiles leave p = exp(l - lse) - [target] in the workspace, and then both p W and p^T x in one launch.  Four products of 2 T C V operations,
// where keeping the logits would take three and T V values of memory.  Bound by the matrix instructions, of which our loop alone reaches 1.39 PFLOP/s in bf16: 16000 tokens x 1024
// x 64001 1.94 ms for the logits (1.08), 2.34 for p (0.89) and 3.74 for both gradients (1.12); 4096 x 512 x 32000, K of eight steps, 158, 205 and 271 us (0.85, 0.65, 0.99).
//
// bf16 tensors: the logits' products are exact in binary32.  The gradients' products are of fp16 values: p, in [-1, 1], as 2^14 p, and x and w
// with a power of two for each channel, which leaves the sum over tokens (the vocabulary) as a factor.  fp16 keeps 3 bits more of p than bf16 from 2^-28
// up (below that steps are of 2^-38: fewer bits than bf16's below 2^-31, nothing below 2^-39), so that bf16 gradients are rounded once in effect, at their
// end (16000 x 1024 x 64001, dw: 0.00168 in norm, with p and d x in binary32 0.00166); gradients asked for in binary32 are off by 2^-12 of their terms.  Of x and w
// fp16 keeps all bits from 2^-31 of a channel's largest value up.
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

// The tokens that count, in their order; one workgroup, of which a wavefront takes 512 tokens at a time.  lse: of the tokens of x, or null; none, none_lse:
// losses and lse of the others, or null.
__global__ __launch_bounds__(1024) void find_tokens(const long long* __restrict__ target, long long ignored, const float* __restrict__ lse, Tokens k,
                                                    float* none, float* none_lse, int T)
{
    constexpr int kEach = 8;
    __shared__ int sums[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int before = 0;
    for (int first = 0; first < T; first += 1024 * kEach) {
        const int t0 = first + wave * 64 * kEach + lane;
        long long y[kEach];
        float l[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int t = t0 + e * 64;
            y[e] = t < T ? target[t] : ignored;
            l[e] = lse && t < T ? lse[t] : 0.f;
        }
        int own = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) own += __popcll(__ballot(y[e] != ignored));
        if (lane == 0) sums[wave] = own;
        __syncthreads();
        int at = before;
        for (int i = 0; i < 16; ++i) {
            if (i < wave) at += sums[i];
            before += sums[i];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int t = t0 + e * 64;
            const unsigned long long there = __ballot(y[e] != ignored);
            const int place = at + __popcll(there & ((1ull << lane) - 1));
            at += __popcll(there);
            if (t >= T) continue;
            const bool counts = y[e] != ignored;
            k.place[t] = counts ? place : -1;
            if (counts) {
                k.order[place] = t;
                k.target[place] = y[e];
                k.known[place] = __uint_as_float(0x7fc00000u);          // until the target's tile writes it: never, if it is outside of the vocabulary
                if (lse) k.lse[place] = l[e];
            } else {
                if (none) none[t] = 0.f;
                if (none_lse) none_lse[t] = 0.f;
            }
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
    // where row i's channel 0 is; channels are HW apart
    __device__ __forceinline__ const T* row(long long i) const
    {
        const uint32_t t = order ? (uint32_t)order[i] : (uint32_t)i, n = HW > 1 ? t / (uint32_t)HW : t;
        return x + (long long)n * C * HW + (t - n * (uint32_t)HW);
    }
};

// Rows whose channels are consecutive, in vectors of 8
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ void read8(const float* p, float (&v)[8])
{
    const u32x8 t = *(const u32x8*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(t[e]);
}
__device__ __forceinline__ void read8(const bf16_t* p, float (&v)[8])
{
    const u32x4 t = *(const u32x4*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e % 2 ? t[e / 2] & 0xffff0000u : t[e / 2] << 16);
}
__device__ __forceinline__ void write8(uint16_t* p, const uint16_t (&v)[8])
{
    u32x4 t;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = (uint32_t)v[2 * e] | (uint32_t)v[2 * e + 1] << 16;
    *(u32x4*)p = t;
}

// parts[block][c] = largest |value| of channel c among 128 rows, as the bits of a binary32 value: non-negative ones are ordered as their bits are.  512 channels
// a workgroup, a wavefront's eight rows under way.  (Atomics instead of the parts, which cross the XCDs: 37 us for 32 MB instead of 10.)
constexpr int kMaximaRows = 128;
template <typename T>
__device__ __forceinline__ void maxima_wide(const Rows<T>& x, const Factor& f, uint32_t* __restrict__ parts, int ld, int block, int group, float* lds)
{
    constexpr int kWaves = 16;
    const long long first = (long long)block * kMaximaRows, end = x.end();
    if (first >= end) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long c = (long long)group * 512 + lane * 8;
    float high[8] = {}, v[8][8], d[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const long long row = first + i * kWaves + wave;
        d[i] = row < end ? f.of((int)row) : 0.f;
        read8(x.row(row < end ? row : end - 1) + (c < x.C ? c : 0), v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) high[e] = fmaxf(high[e], fabsf(v[i][e] * d[i]));
#pragma unroll
    for (int e = 0; e < 8; ++e) lds[wave * 512 + e * 64 + lane] = high[e];
    __syncthreads();
    if (threadIdx.x < 512) {
        const int at = (threadIdx.x & 7) * 64 + (threadIdx.x >> 3);
        const long long channel = (long long)group * 512 + threadIdx.x;
        float most = lds[at];
#pragma unroll
        for (int j = 1; j < kWaves; ++j) most = fmaxf(most, lds[j * 512 + at]);
        if (channel < ld) parts[(long long)block * ld + channel] = __float_as_uint(channel < x.C ? most : 0.f);
    }
}

// The same for any rows: 256 channels a workgroup, four wavefronts for each 64 of them, lanes along the rows where tokens are columns
template <typename T>
__device__ __forceinline__ void maxima_any(const Rows<T>& x, const Factor& f, uint32_t* __restrict__ parts, int ld, int block, int group, float* lds)
{
    const long long first = (long long)block * kMaximaRows, end = x.end(), c0 = (long long)group * 256 + (threadIdx.x >> 8) * 64;
    if (first >= end) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6 & 3;
    uint32_t* const to = parts + (long long)block * ld + c0;
    if (x.HW > 1) {
        if (c0 >= ld) return;
        const T* row[2];
        float d[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const long long i = first + r * 64 + lane;
            row[r] = x.row(i < end ? i : end - 1);
            d[r] = i < end ? f.of((int)i) : 0.f;
        }
#pragma unroll 4
        for (int j = 0; j < 16; ++j) {
            const long long c = c0 + wave * 16 + j, from = (c < x.C ? c : x.C - 1) * x.HW;
            float v = fmaxf(fabsf(to_f32(row[0][from]) * d[0]), fabsf(to_f32(row[1][from]) * d[1]));
            for (int m = 1; m < 64; m *= 2) v = fmaxf(v, __shfl_xor(v, m));
            if (lane == 0) to[wave * 16 + j] = __float_as_uint(c < x.C ? v : 0.f);
        }
    } else {
        const long long c = c0 + lane < x.C ? c0 + lane : x.C - 1;
        float v = 0.f;
#pragma unroll 4
        for (int r = wave; r < kMaximaRows; r += 4)
            if (first + r < end) v = fmaxf(v, fabsf(to_f32(x.row(first + r)[c]) * f.of((int)(first + r))));
        float* const own = lds + (threadIdx.x >> 8) * 256 + lane;
        own[wave * 64] = v;
        __syncthreads();
        if (wave == 0 && c0 < ld) to[lane] = __float_as_uint(c0 + lane < x.C ? fmaxf(fmaxf(own[0], own[64]), fmaxf(own[128], own[192])) : 0.f);
    }
}

// Of both matrices in one launch: workgroups from `blocks_x` on are the second's
template <typename T>
__global__ __launch_bounds__(1024) void channel_maxima(Rows<T> x, Factor f, uint32_t* __restrict__ parts_x, int blocks_x, bool wide_x, Rows<T> w,
                                                       uint32_t* __restrict__ parts_w, bool wide_w, int ld)
{
    __shared__ float lds[16 * 512];
    const bool first = (int)blockIdx.x < blocks_x, wide = first ? wide_x : wide_w;
    const int i = first ? blockIdx.x : blockIdx.x - blocks_x, groups = wide ? (ld + 511) / 512 : (ld + 255) / 256, block = i / groups, group = i % groups;
    const Rows<T> m = first ? x : w;
    const Factor own = first ? f : Factor{};
    uint32_t* const parts = first ? parts_x : parts_w;
    if (wide) maxima_wide(m, own, parts, ld, block, group, lds);
    else maxima_any(m, own, parts, ld, block, group, lds);
}

// most[c] of both matrices from their parts, 64 channels a workgroup
__global__ __launch_bounds__(1024) void join_maxima(const uint32_t* __restrict__ parts_x, const int* __restrict__ tokens, uint32_t* __restrict__ most_x,
                                                    const uint32_t* __restrict__ parts_w, int rows_w, uint32_t* __restrict__ most_w, int ld)
{
    __shared__ uint32_t lds[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    const uint32_t* parts = blockIdx.y ? parts_w : parts_x;
    const int rows = ((blockIdx.y ? rows_w : *tokens) + kMaximaRows - 1) / kMaximaRows;
    uint32_t most = 0;
    for (int i = wave; i < rows; i += 64) {
        uint32_t v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = i + j * 16 < rows ? parts[(long long)(i + j * 16) * ld + c] : 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) most = most > v[j] ? most : v[j];
    }
    lds[wave][lane] = most;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) most = most > lds[i][lane] ? most : lds[i][lane];
    (blockIdx.y ? most_w : most_x)[c] = most;
}

// What the two kernels below write of a value v of row i and channel c.  whole: the value itself (PLANES 1: as bf16, 3: cut), ld values a row.  scaled: times its
// row's factor and its channel's power of two, in fp16.  Rows up to the next multiple of `pad` and channels up to ld are zeros.
struct Packed {
    uint16_t *whole, *scaled;
    long long plane;
    const uint32_t* most;
    int ld, pad;
};

// the powers of two of 8 channels
__device__ __forceinline__ void units_of(const Packed& o, long long c, float (&unit)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) unit[e] = o.scaled ? power(-channel_exponent(o.most[c + e])) : 0.f;
}

template <int PLANES>
__device__ __forceinline__ void write_packed(const Packed& o, long long i, long long c, const float (&v)[8], const float (&unit)[8], float d)
{
    if (o.whole) {
        uint16_t piece[8][3], line[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) cut(v[e], piece[e]);
#pragma unroll
        for (int p = 0; p < PLANES; ++p) {
#pragma unroll
            for (int e = 0; e < 8; ++e) line[e] = piece[e][p];
            write8(o.whole + p * o.plane + i * o.ld + c, line);
        }
    }
    if (o.scaled) {
        uint16_t line[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) line[e] = half_of(v[e] == 0.f ? 0.f : v[e] * d * unit[e]);
        write8(o.scaled + i * o.ld + c, line);
    }
}

// Rows into operands, 8 channels a lane: 32 rows and 512 channels a workgroup
template <typename T, int PLANES>
__device__ __forceinline__ void pack_wide(const Rows<T>& x, const Factor& f, const Packed& o, int block, int group)
{
    const long long first = (long long)block * 32, end = x.end();
    if (first >= (end + o.pad - 1) / o.pad * o.pad) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long c = (long long)group * 512 + lane * 8;
    if (c >= o.ld) return;
    float unit[8];
    units_of(o, c, unit);
#pragma unroll
    for (int r = 0; r < 8; r += 4) {
        float v[4][8], d[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const long long i = first + (r + j) * 4 + wave;
            const bool there = i < end && c < x.C;
            read8(x.row(i < end ? i : 0) + (c < x.C ? c : 0), v[j]);
            d[j] = i < end ? f.of((int)i) : 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] = there ? v[j][e] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) write_packed<PLANES>(o, first + (r + j) * 4 + wave, c, v[j], unit, d[j]);
    }
}

// The same for any rows: 64 rows and 64 channels a workgroup through LDS, read with the lanes along the tokens where these are columns
template <typename T, int PLANES>
__device__ __forceinline__ void pack_any(const Rows<T>& x, const Factor& f, const Packed& o, int block, int group, float (&tile)[64][65])
{
    const long long first = (long long)block * 64, end = x.end();
    if (first >= (end + o.pad - 1) / o.pad * o.pad) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long c0 = (long long)group * 64;
    if (x.HW > 1) {
        const bool there = first + lane < end;
        const T* row = there ? x.row(first + lane) : nullptr;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const long long c = c0 + wave * 16 + j;
            tile[lane][wave * 16 + j] = there && c < x.C ? to_f32(row[c * x.HW]) : 0.f;
        }
    } else {
#pragma unroll 4
        for (int j = 0; j < 16; ++j) {
            const long long i = first + wave * 16 + j;
            tile[wave * 16 + j][lane] = i < end && c0 + lane < x.C ? to_f32(x.row(i)[c0 + lane]) : 0.f;
        }
    }
    __syncthreads();
    float unit[8];
    units_of(o, c0 + (threadIdx.x % 8) * 8, unit);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int line = j * 32 + threadIdx.x / 8, at = (threadIdx.x % 8) * 8;
        const long long i = first + line;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[line][at + e];
        write_packed<PLANES>(o, i, c0 + at, v, unit, i < end ? f.of((int)i) : 0.f);
    }
}

// Both matrices in one launch: workgroups from `blocks_x` on are the second's
template <typename T, int PLANES>
__global__ __launch_bounds__(256) void pack(Rows<T> x, Factor f, Packed to_x, int blocks_x, bool wide_x, Rows<T> w, Packed to_w, bool wide_w)
{
    __shared__ float tile[64][65];
    const bool first = (int)blockIdx.x < blocks_x, wide = first ? wide_x : wide_w;
    const Rows<T> m = first ? x : w;
    const Factor own = first ? f : Factor{};
    const Packed o = first ? to_x : to_w;
    const int i = first ? blockIdx.x : blockIdx.x - blocks_x, groups = wide ? (o.ld + 511) / 512 : o.ld / 64, block = i / groups, group = i % groups;
    if (wide) pack_wide<T, PLANES>(m, own, o, block, group);
    else pack_any<T, PLANES>(m, own, o, block, group, tile);
}

// find_tokens and pack for the loss of at most 64 tokens in one: a wavefront for each packed token, all of which look at the targets
template <typename T, int PLANES>
__global__ __launch_bounds__(256) void begin_few(Rows<T> x, const long long* __restrict__ target, long long ignored, Tokens k,
                                                 uint16_t* __restrict__ xp, long long plane, int ld, float* none, float* none_lse, bool wide)
{
    const int lane = threadIdx.x & 63, i = blockIdx.x * 4 + (threadIdx.x >> 6), T_ = (int)x.rows, C = (int)x.C;
    const long long y = lane < T_ ? target[lane] : ignored;
    const unsigned long long there = __ballot(y != ignored);
    const int count = __popcll(there), before = __popcll(there & ((1ull << lane) - 1));
    if (i == 0) {
        if (lane == 0) *k.count = count;
        if (lane < T_ && y == ignored) {
            if (none) none[lane] = 0.f;
            if (none_lse) none_lse[lane] = 0.f;
        }
    }
    uint16_t* const to = xp + (long long)i * ld;
    if (i >= count) {           // zeros behind the last one
        for (int c = lane * 8; c < ld; c += 512)
#pragma unroll
            for (int p = 0; p < PLANES; ++p) *(u32x4*)(to + p * plane + c) = u32x4{0, 0, 0, 0};
        return;
    }
    const uint32_t t = __ffsll(__ballot(y != ignored && before == i)) - 1, n = x.HW > 1 ? t / (uint32_t)x.HW : t;
    const long long v = __shfl(y, (int)t);
    const T* const from = x.x + (long long)n * C * x.HW + (t - n * (uint32_t)x.HW);
    for (int c = lane * 8; c < ld; c += 512) {
        float a[8] = {}, unit[8] = {};
        if (wide && c < C) read8(from + c, a);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!wide && c + e < C) a[e] = to_f32(from[(c + e) * x.HW]);
        write_packed<PLANES>({xp, nullptr, plane, nullptr, ld, 0}, i, c, a, unit, 1.f);
    }
    if (lane == 0) {
        k.order[i] = (int)t;
        k.target[i] = v;
        k.known[i] = __uint_as_float(0x7fc00000u);
    }
}

// Workgroup -> tiles.  Workgroups go to the XCDs in turn, and each of these takes a run of tiles: bands of four tiles of rows, all columns of a band.
struct Grid {
    int rows, columns;
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// The i'th tile of workgroup `block` of `blocks`, a multiple of 8; false if there is none
__device__ __forceinline__ bool tile_of(int block, int blocks, int i, const Grid& g, int& row, int& column)
{
    const int total = g.rows * g.columns, each = (total + 7) / 8;
    const int in_run = (block >> 3) + i * (blocks >> 3), id = (block & 7) * each + in_run;
    if (in_run >= each || id >= total) return false;
    const int band = id / (4 * g.columns), in = id - band * 4 * g.columns;
    const int high = g.rows - band * 4 < 4 ? g.rows - band * 4 : 4;
    column = in / high;
    row = band * 4 + in - column * high;
    return true;
}

int blocks_of(const Grid& g) { return ((long long)g.rows * g.columns + 7) / 8 * 8; }

// ... of a kernel whose workgroups walk over the tiles: as many as are resident, 256 CUs with 160 KB of LDS each
int walkers_of(const Grid& g, int lds)
{
    const int all = blocks_of(g), resident = 256 * (lds <= 80 * 1024 ? 2 : 1);
    return all < resident ? all : resident;
}

// f(m, n, r) for the accumulator that holds the target of the lane's token, in the lane that has it; first: row of the vocabulary with which the tile begins
template <typename P, typename F>
__device__ __forceinline__ void at_targets(const Tokens& k, int count, int V, long long first, long long column, int wm, int wn, F&& f)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int n = 0; n < P::FN; ++n) {
        const long long t = column + (wn * P::FN + n) * 32 + (lane & 31), y = k.target[t], v = y - first - wm * 32 * P::FM;
        const int in = t < count && y < V && v >= 0 && v < 32 * P::FM && ((int)v >> 2 & 1) == lane >> 5 ? (int)v & ~4 : -1;
        if (!__any(in >= 0)) continue;              // seldom: a token's target is in one of the vocabulary's many tiles
#pragma unroll
        for (int m = 0; m < P::FM; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (in == m * 32 + 8 * (r / 4) + r % 4) f(t, m, n, r);
    }
}

// Logits of a tile: rows of the vocabulary, columns are tokens.  part[tile row][token] = (max, sum of exp(l - max)); and the targets' own: the loss is a difference
// of the same sums
template <typename P>
__global__ __launch_bounds__(P::kThreads, P::kWavesPerSimd) void loss_product(Operand w, Operand x, Tokens k,
                                                                              float2* __restrict__ part, long long Tp, int steps, int V, int rows)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    constexpr int kHigh = P::kM / 32 / P::FM;   // wavefronts one above the other
    const int count = uniform(*k.count);
    const Grid g = {rows, (count + P::kN - 1) / P::kN};
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / (P::kN / 32 / P::FN), wn = wave % (P::kN / 32 / P::FN);
    float* most = (float*)(lds + P::kLds);      // [kHigh][kN], then sums likewise
    float* sums = most + kHigh * P::kN;
    P::walk(
        w, x, lds,
        [&](int i, typename P::Part& p) {
            int row, column;
            if (!tile_of(blockIdx.x, gridDim.x, i, g, row, column)) return false;
            p = {(long long)row * P::kM, (long long)column * P::kN, 0, steps};
            return true;
        },
        [&](const typename P::Part& p, f32x16 (&acc)[P::FM][P::FN]) {
            const int v0 = (int)p.row + wm * 32 * P::FM + 4 * (lane >> 5);
            at_targets<P>(k, count, V, p.row, p.column, wm, wn, [&](long long t, int m, int n, int r) { k.known[t] = acc[m][n][r]; });
            if (p.row + P::kM > V)
#pragma unroll
                for (int m = 0; m < P::FM; ++m)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (v0 + m * 32 + 8 * (r / 4) + r % 4 >= V)
#pragma unroll
                            for (int n = 0; n < P::FN; ++n) acc[m][n][r] = -__builtin_inff();
#pragma unroll
            for (int n = 0; n < P::FN; ++n) {
                float high = -__builtin_inff();
#pragma unroll
                for (int m = 0; m < P::FM; ++m)
#pragma unroll
                    for (int r = 0; r < 16; ++r) high = fmaxf(high, acc[m][n][r]);
                high = fmaxf(high, __shfl_xor(high, 32));
                if (lane < 32) most[wm * P::kN + (wn * P::FN + n) * 32 + lane] = high;
            }
            lds_barrier();
#pragma unroll
            for (int n = 0; n < P::FN; ++n) {
                const int at = (wn * P::FN + n) * 32 + (lane & 31);
                float high = most[at];
#pragma unroll
                for (int i = 1; i < kHigh; ++i) high = fmaxf(high, most[i * P::kN + at]);
                // the difference first, which is exact near the maximum: the largest term is 1, and the loss of a token that is sure of its target 0 or more.  (With
                // high log2(e) rounded beforehand all terms were off by up to 2^-24 of that: losses of +-5e-6 at logits of 100.)
                float sum = 0.f;
#pragma unroll
                for (int m = 0; m < P::FM; ++m)
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f((acc[m][n][r] - high) * kLog2E);
                sum += __shfl_xor(sum, 32);
                if (lane < 32) sums[wm * P::kN + at] = sum;
            }
            lds_barrier();
            if (threadIdx.x < P::kN) {
                const int at = threadIdx.x;
                float high = most[at], sum = sums[at];
#pragma unroll
                for (int i = 1; i < kHigh; ++i) {
                    high = fmaxf(high, most[i * P::kN + at]);
                    sum += sums[i * P::kN + at];
                }
                part[p.row / P::kM * Tp + p.column + at] = make_float2(high, sum);
            }
            lds_barrier();                      // most is written again
        });
}
template <typename P> constexpr int kLossLds = P::kLds + 2 * (P::kM / 32 / P::FM) * P::kN * 4;

// lse and loss of 16 packed tokens from the tiles' parts, which 64 groups of lanes take in turn; losses: of the tokens of x.  (64 tokens and 16 groups: 6.1 us
// instead of 3.6 for 48 tokens and 500 parts each, 7.9 instead of 10.1 for 16000 and 251.)
__global__ __launch_bounds__(1024) void join_parts(const float2* __restrict__ part, long long Tp, int tiles, Tokens k, float* __restrict__ losses,
                                                   float* __restrict__ lse)
{
    constexpr int TOKENS = 16, kWaves = 16, kAhead = 8, kSets = 1024 / TOKENS;
    __shared__ float2 lds[kWaves][TOKENS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = blockIdx.x * TOKENS + lane % TOKENS, count = *k.count;
    if ((int)blockIdx.x * TOKENS >= count) return;
    float high = -__builtin_inff(), sum = 0.f;
    // several parts at once, so that their exponentials wait for nothing but the maximum; a part of sum 0 has no values
    auto join = [&](const float2* p, int n) {
        float to = high;
#pragma unroll
        for (int e = 0; e < n; ++e) to = fmaxf(to, p[e].x);
        sum = sum == 0.f ? 0.f : sum * __builtin_amdgcn_exp2f((high - to) * kLog2E);
#pragma unroll
        for (int e = 0; e < n; ++e) sum += p[e].y == 0.f ? 0.f : p[e].y * __builtin_amdgcn_exp2f((p[e].x - to) * kLog2E);
        high = to;
    };
    for (int t = threadIdx.x / TOKENS; t < tiles; t += kSets * kAhead) {
        float2 p[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int at = t + e * kSets;
            p[e] = at < tiles ? part[at * Tp + i] : make_float2(-__builtin_inff(), 0.f);
        }
        join(p, kAhead);
    }
#pragma unroll
    for (int m = TOKENS; m < 64; m *= 2) {
        const float2 other = make_float2(__shfl_xor(high, m), __shfl_xor(sum, m));
        join(&other, 1);
    }
    if (lane < TOKENS) lds[wave][lane] = make_float2(high, sum);
    __syncthreads();
    if (wave || lane >= TOKENS || i >= count) return;
    float2 p[kWaves];
#pragma unroll
    for (int t = 0; t < kWaves; ++t) p[t] = lds[t][lane];
    high = -__builtin_inff();
    sum = 0.f;
    join(p, kWaves);
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

// p of a tile of a piece of the vocabulary: p[token][v - first].  Three planes: workgroups walk over the tiles, and a tile's values leave through 16 KB beside
// the operands' buffers while the next tile's are loaded (177 -> 162 us a launch of 2000 tokens x 512 x 16000).  One plane: a tile a workgroup, whose
// values leave through all of the buffers' room in one go (4096 x 512 x 32000: 193 us, walking 230: eight pieces, and no registers left).
template <typename P> constexpr bool kWalks = P::kPlanes == 3;
template <typename P> constexpr bool kTwoRooms = P::kLds + 2 * Lines<P>::kPiece <= 160 * 1024;
template <typename P> constexpr int kShareLds = P::kLds + (kWalks<P> ? (kTwoRooms<P> ? 2 : 1) * Lines<P>::kPiece : 0);

template <typename P>
__global__ __launch_bounds__(P::kThreads, P::kWavesPerSimd) void share_product(Operand w, Operand x, Tokens k, Factor f, uint16_t* __restrict__ p,
                                                                               long long plane, int piece, int steps, int first, int V, int rows)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    constexpr bool kCut = P::kPlanes == 3;
    const int count = uniform(*k.count);
    const Grid g = {rows, (count + P::kN - 1) / P::kN};
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / (P::kN / 32 / P::FN), wn = wave % (P::kN / 32 / P::FN);
    auto at = [&](int i, typename P::Part& part) {
        int row, column;
        if (!tile_of(blockIdx.x, gridDim.x, i, g, row, column)) return false;
        part = {(long long)first + row * P::kM, (long long)column * P::kN, 0, steps};
        return true;
    };
    // logits into p, which a token's gradient is part of where it is cut
    auto shares = [&](const typename P::Part& part, f32x16 (&acc)[P::FM][P::FN]) {
        const int v0 = (int)part.row + wm * 32 * P::FM + 4 * (lane >> 5);
        const bool ends = part.row + P::kM > V;
#pragma unroll
        for (int n = 0; n < P::FN; ++n) {
            const long long t = part.column + (wn * P::FN + n) * 32 + (lane & 31);
            // lse off first, as in loss_product: what p is off by as a whole is half a step of lse (2^-24 of it) and, raised, of 14 (3e-7)
            const float lse = k.lse[t];
            const float d = kCut ? f.of((int)t) : 1.f;
#pragma unroll
            for (int m = 0; m < P::FM; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float share = __builtin_amdgcn_exp2f(fmaf(acc[m][n][r] - lse, kLog2E, kCut ? 0.f : kRaise));
                    if (ends && v0 + m * 32 + 8 * (r / 4) + r % 4 >= V) share = 0.f;
                    acc[m][n][r] = kCut ? share * d : share;
                }
        }
        at_targets<P>(k, count, V, part.row, part.column, wm, wn,
                      [&](long long t, int m, int n, int r) { acc[m][n][r] -= kCut ? f.of((int)t) : (float)(1 << (int)kRaise); });
    };
    if constexpr (kWalks<P>) {
        P::walk(w, x, lds, at, [&](const typename P::Part& part, f32x16 (&acc)[P::FM][P::FN]) {
            shares(part, acc);
#pragma unroll
            for (int plane_at = 0; plane_at < P::kPlanes; ++plane_at) {
                auto piece_of = [&](float v) {
                    uint16_t c[3];
                    cut(v, c);
                    return c[plane_at];
                };
                Lines<P>::template stream<kTwoRooms<P>>(
                    lds + P::kLds, wm, wn, [&](int m, int n, int r) { return piece_of(acc[m][n][r]); },
                    [&](int line, int at, u32x4 v) { *(u32x4*)(p + plane_at * plane + (part.column + line) * piece + (part.row - first) + at) = v; });
            }
        });
    } else {
        typename P::Part part;
        if (!at(0, part)) return;
        f32x16 acc[P::FM][P::FN];
        P::run(w, x, part, lds, acc);
        shares(part, acc);
        Lines<P>::store(
            lds, wm, wn, [&](int m, int n, int r) { return half_of(acc[m][n][r]); },
            [&](int line, int at, u32x4 v) { *(u32x4*)(p + (part.column + line) * piece + (part.row - first) + at) = v; });
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
    int blocks_x, blocks_w;             // of the grid, the longer ones first
    bool w_first;
    int split_w;                        // of K = tokens; more than one: sums to dw_parts, [split][row of the piece][ld]
    float* dw_parts;
    long long dw_plane;
};

// p W: rows are channels, columns tokens, K a part of the piece; and p^T x: rows are channels, columns the piece's rows, K the tokens
template <typename PX, typename PW>
__global__ __launch_bounds__(PX::kThreads, PX::kWavesPerSimd) void gradient_products(Gradients a)
{
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    constexpr int kWide = PX::kN / 32 / PX::FN;     // wavefronts side by side
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / kWide, wn = wave % kWide;
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    const int of_x = a.w_first ? (int)blockIdx.x - a.blocks_w : (int)blockIdx.x, of_w = a.w_first ? (int)blockIdx.x : (int)blockIdx.x - a.blocks_x;
    if (of_x >= 0 && of_x < a.blocks_x) {
        const int each = a.blocks_x / a.split, part = of_x / each;
        int row, column;
        if (!tile_of(of_x - part * each, each, 0, {a.gx.rows, (uniform(*a.count) + PX::kN - 1) / PX::kN}, row, column)) return;
        const int from = part * a.split_steps, left = a.steps - from;
        f32x16 acc[PX::FM][PX::FN];
        PX::run(a.w, a.p_tokens, {(long long)row * PX::kM, (long long)column * PX::kN, (long long)from * PX::kK, left < a.split_steps ? left : a.split_steps}, lds,
                acc);
#pragma unroll
        for (int n = 0; n < PX::FN; ++n) {
            const long long t = (long long)column * PX::kN + (wn * PX::FN + n) * 32 + (lane & 31);
            float* const to = a.dx + part * a.dx_plane + t * a.ld;
            f32x4 before[PX::FM][4];
#pragma unroll
            for (int m = 0; m < PX::FM; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = row * PX::kM + (wm * PX::FM + m) * 32 + 4 * (lane >> 5) + 8 * q;
                    before[m][q] = f32x4{0.f, 0.f, 0.f, 0.f};
                    if (!a.begins && c < a.ld) before[m][q] = *(const f32x4*)(to + c);
                }
#pragma unroll
            for (int m = 0; m < PX::FM; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = row * PX::kM + (wm * PX::FM + m) * 32 + 4 * (lane >> 5) + 8 * q;
                    const f32x4 v = {acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]};
                    if (c < a.ld) *(f32x4*)(to + c) = before[m][q] + v;
                }
        }
        return;
    }
    const int each = a.blocks_w / a.split_w, part = of_w / each;
    int row, column;
    if (!tile_of(of_w - part * each, each, 0, a.gw, row, column)) return;
    const int steps = (uniform(*a.count) + PW::kK - 1) / PW::kK, own = (steps + a.split_w - 1) / a.split_w, from = part * own;
    f32x16 acc[PW::FM][PW::FN];
    PW::run(a.x, a.p_rows,
            {(long long)row * PW::kM, (long long)column * PW::kN, (long long)from * PW::kK, steps - from < own ? (steps > from ? steps - from : 0) : own}, lds, acc);
#pragma unroll
    for (int m = 0; m < PW::FM; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int c = row * PW::kM + (wm * PW::FM + m) * 32 + 4 * (lane >> 5) + 8 * (r / 4) + r % 4;
            const float unit = a.most_x && c < a.C ? power(channel_exponent(a.most_x[c]) - (int)kRaise) : 1.f;
#pragma unroll
            for (int n = 0; n < PW::FN; ++n) acc[m][n][r] *= unit;
        }
    if (a.split_w > 1) {
#pragma unroll
        for (int n = 0; n < PW::FN; ++n) {
            const long long in = column * PW::kN + (wn * PW::FN + n) * 32 + (lane & 31);
            float* const to = a.dw_parts + part * a.dw_plane + in * a.ld;
#pragma unroll
            for (int m = 0; m < PW::FM; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = row * PW::kM + (wm * PW::FM + m) * 32 + 4 * (lane >> 5) + 8 * q;
                    if (c < a.ld && in < a.piece)
                        *(f32x4*)(to + c) = f32x4{acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]};
                }
        }
        return;
    }
    if (a.wide) {
#pragma unroll
        for (int n = 0; n < PW::FN; ++n) {
            const int in = column * PW::kN + (wn * PW::FN + n) * 32 + (lane & 31);
            const long long v = a.first + in;
            if (v >= a.V || in >= a.piece) continue;
            float* const to = (float*)a.dw + v * a.C;
#pragma unroll
            for (int m = 0; m < PW::FM; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = row * PW::kM + (wm * PW::FM + m) * 32 + 4 * (lane >> 5) + 8 * q;
                    typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
                    if (c + 3 < a.C) {
                        *(f32x4u*)(to + c) = f32x4u{acc[m][n][4 * q], acc[m][n][4 * q + 1], acc[m][n][4 * q + 2], acc[m][n][4 * q + 3]};
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (c + e < a.C) to[c + e] = acc[m][n][4 * q + e];
                    }
                }
        }
        return;
    }
    Lines<PW>::store(
        lds, wm, wn, [&](int m, int n, int r) { return from_f32<bf16_t>(acc[m][n][r]); },
        [&](int line, int at, u32x4 v) {
            const int in = column * PW::kN + line, c = row * PW::kM + at;
            const long long place = a.first + in;
            if (place >= a.V || in >= a.piece) return;
            bf16_t* const to = (bf16_t*)a.dw + place * a.C + c;
            typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));
            if (c + 7 < a.C) {
                *(u32x4u*)to = v;
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c + e < a.C) to[e] = (bf16_t)(v[e / 2] >> 16 * (e % 2));
            }
        });
}

// dx of 64 tokens of x and 64 channels from the parts of p W, four channels a lane; through LDS where tokens are columns
template <typename T>
__global__ __launch_bounds__(256) void join_dx(const float* __restrict__ parts, long long plane, int split, int ld, Tokens k, Factor f,
                                               const uint32_t* __restrict__ most, T* __restrict__ dx, long long tokens, int C, long long HW)
{
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    __shared__ float tile[64][65];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in = (threadIdx.x % 16) * 4;
    const long long first = (long long)blockIdx.x * 64, c = (long long)blockIdx.y * 64 + in;
    float unit[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) unit[e] = most ? power(channel_exponent(c + e < C ? most[c + e] : 0) - (int)kRaise) : 1.f;
    f32x4 sum[4];
    const float* from[4];
    int place[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const long long t = first + threadIdx.x / 16 + j * 16;
        place[j] = t < tokens ? k.place[t] : -1;
        from[j] = parts + (long long)(place[j] < 0 ? 0 : place[j]) * ld + c;
        sum[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (place[0] >= 0 || place[1] >= 0 || place[2] >= 0 || place[3] >= 0)
#pragma unroll 4
        for (int s = 0; s < split; ++s)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] += *(const f32x4*)(from[j] + s * plane);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const long long t = first + threadIdx.x / 16 + j * 16;
        const float d = place[j] < 0 ? 0.f : most ? f.of(place[j]) : 1.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[j][e] = place[j] < 0 ? 0.f : sum[j][e] * (most ? d * unit[e] : 1.f);
        if (HW > 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) tile[threadIdx.x / 16 + j * 16][in + e] = sum[j][e];
        } else if (t < tokens) {
            typedef T out __attribute__((ext_vector_type(4), aligned(sizeof(T))));
            if (c + 3 < C) {
                out o;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = from_f32<T>(sum[j][e]);
                *(out*)(dx + t * C + c) = o;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < C) dx[t * C + c + e] = from_f32<T>(sum[j][e]);
            }
        }
    }
    if (HW == 1) return;
    __syncthreads();
    const uint32_t t = (uint32_t)first + lane, n = t / (uint32_t)HW;
    if (t >= tokens) return;
    T* const to = dx + (long long)n * C * HW + (t - n * (uint32_t)HW);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const long long channel = (long long)blockIdx.y * 64 + wave * 16 + j;
        if (channel < C) to[channel * HW] = from_f32<T>(tile[lane][wave * 16 + j]);
    }
}

// dw of a piece from the parts of p^T x, four channels a thread
__global__ __launch_bounds__(256) void join_dw(const float* __restrict__ parts, long long plane, int split, int ld, void* __restrict__ dw, bool wide, int rows, int C)
{
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, v = at / (ld / 4);
    const int c = (int)(at - v * (ld / 4)) * 4;
    if (v >= rows || c >= C) return;
    f32x4 sum = *(const f32x4*)(parts + v * ld + c);
    for (int s = 1; s < split; ++s) sum += *(const f32x4*)(parts + s * plane + v * ld + c);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (c + e < C) {
            if (wide) ((float*)dw)[v * C + c + e] = sum[e];
            else ((bf16_t*)dw)[v * C + c + e] = from_f32<bf16_t>(sum[e]);
        }
}

// ---- sizes ----

constexpr int kRowsPad = 256;               // rows of the vocabulary in a workspace end at a multiple of this

long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }

template <typename T> constexpr int kPlanesOf = sizeof(T) == 4 ? 3 : 1;

// Tiles of the products.  bf16: 128 bytes of a line at a time (K = 64), a full line of the L2; three planes: 64 bytes of each.
template <typename T> struct Forms {
    typedef Form<256, 256, 2, 4, 64, 2, 1> Large;
    typedef Form<128, 128, 2, 2, 64, 2, 1> Middle;
    typedef Form<64, 64, 2, 2, 64, 4, 1> Small;
    typedef Form<64, 64, 2, 2, 64, 2, 1> Few;
};
template <> struct Forms<float> {
    typedef Form<256, 128, 4, 2, 32, 2, 3> Large;
    typedef Form<128, 128, 2, 2, 32, 3, 3> Middle;
    typedef Form<64, 64, 2, 2, 32, 3, 3> Small;
    typedef Form<64, 64, 2, 2, 32, 2, 3> Few;
};

template <typename T, typename F> using LossProduct = Product<F, false, false, false>;
template <typename T, typename F> using DxProduct = Product<F, sizeof(T) == 2, true, false>;
template <typename T, typename F> using DwProduct = Product<F, sizeof(T) == 2, true, true>;

// f(form) for a product of so many rows and columns: the largest tiles of which there are enough.  Losses of C = 512 bf16: 300 x 16000 (126 large tiles) 32.3 us in the large form,
// 26.6 in the middle one; 1000 x 16000 (252) 36, 39; 4096 x 32000 166, 193; 100 x 16000 (125 middle tiles) 23.3 in the middle form, 21.1 in the small one
template <typename T, typename F>
auto with_form(long long rows, long long columns, F&& f)
{
    typedef typename Forms<T>::Large L;
    typedef typename Forms<T>::Middle M;
    auto tiles = [&](int bm, int bn) { return ((rows + bm - 1) / bm) * ((columns + bn - 1) / bn); };
    if (columns > M::BN && rows > M::BM && tiles(L::BM, L::BN) >= 200) return f(L());
    if (columns > 64 && rows > 64 && tiles(M::BM, M::BN) >= 200) return f(M());
    return f(typename Forms<T>::Small());
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
template <typename T>
LossRoom take_loss(Room& room, const Shape& s, bool direct_w, int reduction)
{
    constexpr int planes = kPlanesOf<T>;
    LossRoom r;
    r.c = take_common(room, s, planes);
    r.wp = direct_w ? nullptr : room.take<uint16_t>(planes * round_up(s.V, kRowsPad) * r.c.ld);
    r.part = room.take<float2>(with_form<T>(s.V, s.T(), [&](auto form) { return (s.V + decltype(form)::BM - 1) / decltype(form)::BM; }) * r.c.Tp);
    r.losses = reduction == NONE ? nullptr : room.take<float>(s.T());
    return r;
}

struct Pieces {
    long long piece;
    int count;
};

// Pieces of the vocabulary, equally long: at most 2^28 values of p at a time, 2^26 of three planes, some 0.5 GB, or 2048 rows of the vocabulary where that is more (beyond 131072
// tokens in bf16 and 32768 in binary32: 262144 tokens keep 1.1 or 3.2 GB); a piece costs a round of dx's sums and the ends of three launches.  16000 x 1024 x
// 64001 bf16, gradients: 2^26 7.1 ms, 2^27 6.5, 2^28 6.2, 2^29 6.1; 1340 x 512 x 32000 binary32: 2^24 934 us, 2^25 916, 2^26 834, 2^27 858
Pieces pieces_of(const Shape& s, int planes)
{
    const long long Tp = padded(s.T()), Vp = round_up(s.V, kRowsPad), most = planes == 3 ? 1ll << 26 : 1ll << 28;
    long long piece = most / Tp / kRowsPad * kRowsPad;
    if (piece < 2048) piece = 2048;
    const long long count = (Vp + piece - 1) / piece;
    return {round_up((Vp + count - 1) / count, kRowsPad), (int)count};
}

// The form of both gradients' products: rows are channels, columns tokens and the piece's rows.  Gradients of 512 x 32000 bf16: 512 tokens (282 blocks) 172 us in the large
// form, 156 in the middle one; 1000 (314) 222, 212; 2000 (378) 321, 357; 4096 (506) 543, 697.
// Few tokens make most tiles one or two steps long: two buffers, so that more of them share a CU; 48 tokens 98 us, in the small form 112, 100 tokens 109, in the middle one 113; 200
// tokens 135 and 122; 4096 x 64 x 32000 302, in the small form 252
template <typename T, typename F>
auto with_gradient_form(const Shape& s, long long piece, F&& f)
{
    typedef typename Forms<T>::Large L;
    typedef typename Forms<T>::Middle M;
    const long long ld = round_up(s.C, 64), T_ = s.T();
    // K of the first product can be split
    auto blocks = [&](int bm, int bn) { return ((ld + bm - 1) / bm) * (piece / bn + (T_ + bn - 1) / bn * 8); };
    if (ld > 128 && T_ > 128 && blocks(L::BM, L::BN) >= 350) return f(L());
    if (T_ <= 128) return f(typename Forms<T>::Few());
    if (ld > 64) return f(M());
    return f(typename Forms<T>::Small());
}

// Parts of K of p W and of p^T x: so many that none takes longer than a CU's share of both products, and none of fewer than 512 values of K (in one part each the gradients
// of 48 tokens x 512 x 32000 take 186 us instead of 119, of 4096 tokens 985 instead of 543)
struct Splits {
    int x, w;
};

template <typename T>
Splits splits_of(const Shape& s, long long piece)
{
    return with_gradient_form<T>(s, piece, [&](auto form) {
        typedef decltype(form) F;
        const long long ld = round_up(s.C, 64), T_ = s.T(), high = (ld + F::BM - 1) / F::BM;
        const long long tiles_x = high * ((T_ + F::BN - 1) / F::BN), tiles_w = high * (piece / F::BN);
        const long long steps_x = piece / F::BK, steps_w = (T_ + F::BK - 1) / F::BK;
        const long long share = (tiles_x * steps_x + tiles_w * steps_w + 255) / 256;
        auto split = [&](long long steps, long long k) {
            long long n = (steps + share - 1) / share;
            n = n > 16 ? 16 : n;
            return (int)(n > k / 512 ? (k / 512 > 1 ? k / 512 : 1) : n);
        };
        return Splits{split(steps_x, piece), split(steps_w, T_)};
    });
}

struct GradientRoom {
    Common c;
    uint16_t *wp, *ws, *xs, *p;
    uint32_t *most_x, *most_w, *parts_x, *parts_w;
    float* parts;
    Pieces pieces;
    Splits split;
    float* dw_parts;
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
        r.most_x = room.take<uint32_t>(r.c.ld);
        r.most_w = room.take<uint32_t>(r.c.ld);
        r.parts_x = room.take<uint32_t>((s.T() + kMaximaRows - 1) / kMaximaRows * r.c.ld);
        r.parts_w = room.take<uint32_t>((s.V + kMaximaRows - 1) / kMaximaRows * r.c.ld);
    }
    r.pieces = pieces_of(s, planes);
    r.p = room.take<uint16_t>(planes * r.c.Tp * r.pieces.piece);
    r.split = splits_of<T>(s, r.pieces.piece);
    r.parts = room.take<float>(r.split.x * r.c.Tp * r.c.ld);
    r.dw_parts = r.split.w > 1 ? room.take<float>(r.split.w * r.pieces.piece * r.c.ld) : nullptr;
    return r;
}

template <typename T>
Operand vocabulary_rows(const T* w, const uint16_t* wp, const Shape& s, long long ld)
{
    if (wp) return {wp, round_up(s.V, kRowsPad) * ld, ld, round_up(s.V, kRowsPad) - 1};
    return {(const uint16_t*)w, 0, s.C, (long long)s.V - 1};
}

template <typename T> bool wide_rows(const T* p, long long C) { return C % 8 == 0 && ((uintptr_t)p & (8 * sizeof(T) - 1)) == 0; }

template <typename T> bool wide(const Rows<T>& m) { return m.HW == 1 && wide_rows(m.x, m.C); }

template <typename T>
void launch_maxima(const Rows<T>& x, const Factor& f, uint32_t* parts_x, const Rows<T>& w, uint32_t* parts_w, int ld, hipStream_t st)
{
    auto blocks = [&](const Rows<T>& m) { return (int)((m.rows + kMaximaRows - 1) / kMaximaRows) * (wide(m) ? (ld + 511) / 512 : (ld + 255) / 256); };
    channel_maxima<T><<<blocks(x) + blocks(w), 1024, 0, st>>>(x, f, parts_x, blocks(x), wide(x), w, parts_w, wide(w), ld);
}

// rows: padded, 0 for a matrix that is not packed
template <typename T>
void launch_pack(const Rows<T>& x, const Factor& f, const Packed& to_x, long long rows_x, const Rows<T>& w, const Packed& to_w, long long rows_w, hipStream_t st)
{
    auto blocks = [&](const Rows<T>& m, const Packed& o, long long rows) { return (int)(wide(m) ? rows / 32 * ((o.ld + 511) / 512) : rows / 64 * (o.ld / 64)); };
    const int of_x = blocks(x, to_x, rows_x), all = of_x + blocks(w, to_w, rows_w);
    if (all) pack<T, kPlanesOf<T>><<<all, 256, 0, st>>>(x, f, to_x, of_x, wide(x), w, to_w, wide(w));
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
    if (es == 4) (void)take_loss<float>(room, s, false, reduction);
    else (void)take_loss<bf16_t>(room, s, s.C % 64 == 0 && aligned, reduction);
    return room.used;
}

template <typename T>
hipError_t launch_loss(const T* x, const T* w, const long long* target, long long ignored, int reduction, float* loss, float* lse, const Shape& s,
                       char* workspace, hipStream_t st)
{
    constexpr int planes = kPlanesOf<T>;
    Room room = {workspace};
    const bool at_place = direct(w, s);
    const LossRoom r = take_loss<T>(room, s, at_place, reduction);
    const Tokens& k = r.c.k;
    const long long T_ = s.T(), ld = r.c.ld, Tp = r.c.Tp;
    float* losses = reduction == NONE ? loss : r.losses;
    const Rows<T> rows = {x, k.order, k.count, T_, s.C, s.HW};
    const bool few = T_ <= 64;
    const long long Vp = round_up(s.V, kRowsPad);
    if (few)
        begin_few<T, planes><<<16, 256, 0, st>>>(rows, target, ignored, k, r.c.xp, Tp * ld, (int)ld, losses, lse, wide(rows));
    else
        find_tokens<<<1, 1024, 0, st>>>(target, ignored, nullptr, k, losses, lse, (int)T_);
    launch_pack<T>(rows, {}, {r.c.xp, nullptr, Tp * ld, nullptr, (int)ld, kPad}, few ? 0 : Tp, {w, nullptr, nullptr, s.V, s.C, 1},
                   {r.wp, nullptr, Vp * ld, nullptr, (int)ld, kRowsPad}, r.wp ? Vp : 0, st);
    int tiles = 0;
    const hipError_t e = with_form<T>(s.V, T_, [&](auto form) {
        typedef LossProduct<T, decltype(form)> P;
        const Grid g = {(int)((s.V + P::kM - 1) / P::kM), (int)((T_ + P::kN - 1) / P::kN)};
        tiles = g.rows;
        const hipError_t e = allow(loss_product<P>, kLossLds<P>);
        if (e != hipSuccess) return e;
        const Operand b = {r.c.xp, Tp * ld, ld, Tp - 1};
        loss_product<P><<<walkers_of(g, kLossLds<P>), P::kThreads, kLossLds<P>, st>>>(vocabulary_rows(w, r.wp, s, ld), b, k, r.part, Tp,
                                                                                      (int)(ld / P::kK), s.V, g.rows);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    join_parts<<<(T_ + 15) / 16, 1024, 0, st>>>(r.part, Tp, tiles, k, losses, lse);
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
    find_tokens<<<1, 1024, 0, st>>>(target, ignored, lse, k, nullptr, nullptr, (int)T_);
    const Rows<T> rows = {x, k.order, k.count, T_, s.C, s.HW}, all = {w, nullptr, nullptr, s.V, s.C, 1};
    if constexpr (planes == 1) {
        launch_maxima(rows, f, r.parts_x, all, r.parts_w, (int)ld, st);
        join_maxima<<<dim3(ld / 64, 2), 1024, 0, st>>>(r.parts_x, k.count, r.most_x, r.parts_w, s.V, r.most_w, (int)ld);
    }
    launch_pack(rows, f, {r.c.xp, r.xs, Tp * ld, r.most_x, (int)ld, kPad}, Tp, all, {r.wp, r.ws, Vp * ld, r.most_w, (int)ld, kRowsPad},
                planes == 1 || r.wp ? Vp : 0, st);
    int parts = 1;                          // of p W: the first piece, the longest, has the most
    hipError_t e = hipSuccess;
    for (int i = 0; i < r.pieces.count && e == hipSuccess; ++i) {
        const long long first = i * piece, length = Vp - first < piece ? Vp - first : piece;
        if (length <= 0) break;
        e = with_form<T>(length, T_, [&](auto form) {
            typedef LossProduct<T, decltype(form)> P;
            const Grid g = {(int)(length / P::kM), (int)((T_ + P::kN - 1) / P::kN)};
            const hipError_t e = allow(share_product<P>, kShareLds<P>);
            if (e != hipSuccess) return e;
            const Operand b = {r.c.xp, Tp * ld, ld, Tp - 1};
            share_product<P><<<kWalks<P> ? walkers_of(g, kShareLds<P>) : blocks_of(g), P::kThreads, kShareLds<P>, st>>>(vocabulary_rows(w, r.wp, s, ld), b, k, f, r.p, Tp * piece,
                                                                                            (int)piece, (int)(ld / P::kK), (int)first, s.V, g.rows);
            return hipGetLastError();
        });
        if (e != hipSuccess) break;
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
        a.wide = wide;
        a.begins = i == 0;
        e = with_gradient_form<T>(s, piece, [&](auto form) {
            typedef decltype(form) F;
            typedef DxProduct<T, F> PX;
            typedef DwProduct<T, F> PW;
            const hipError_t e = allow(gradient_products<PX, PW>, PX::kLds);
            if (e != hipSuccess) return e;
            a.steps = (int)(length / F::BK);
            a.split_steps = (int)((piece / F::BK + r.split.x - 1) / r.split.x);     // of a whole piece, so that no later one has more parts than the first
            a.split = (a.steps + a.split_steps - 1) / a.split_steps;
            if (i == 0) parts = a.split;
            const int high = (int)((ld + F::BM - 1) / F::BM);
            a.gx = {high, (int)((T_ + F::BN - 1) / F::BN)};
            a.gw = {high, (int)(length / F::BN)};
            a.blocks_x = blocks_of(a.gx) * a.split;
            a.split_w = r.split.w;
            a.dw_parts = r.dw_parts;
            a.dw_plane = piece * ld;
            a.blocks_w = blocks_of(a.gw) * a.split_w;
            a.w_first = T_ / F::BK / a.split_w > a.split_steps;
            gradient_products<PX, PW><<<a.blocks_x + a.blocks_w, PX::kThreads, PX::kLds, st>>>(a);
            if (a.split_w > 1) {
                const long long rows = s.V - first < length ? s.V - first : length;
                void* const to = (char*)dw + first * s.C * (wide ? 4 : 2);
                if (rows > 0) join_dw<<<(rows * (ld / 4) + 255) / 256, 256, 0, st>>>(r.dw_parts, piece * ld, a.split_w, (int)ld, to, wide, (int)rows, s.C);
            }
            return hipGetLastError();
        });
    }
    if (e != hipSuccess) return e;
    join_dx<T><<<dim3((T_ + 63) / 64, ld / 64), 256, 0, st>>>(r.parts, Tp * ld, parts, (int)ld, k, f, r.most_w, dx, T_, s.C, s.HW);
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
