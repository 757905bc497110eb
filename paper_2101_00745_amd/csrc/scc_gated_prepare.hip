// What the gated layer's products need done before and after (see scc_gated.h): each a single launch, its workgroups dealt out over the
// jobs, since a job of its own costs a launch's 3 us and is itself below one.
#include "scc_gated.h"

namespace scc {
namespace gated {

namespace {

// a stored value in another storage type
template <typename To, typename From>
__device__ __forceinline__ To as(From v)
{
    if constexpr (sizeof(To) == sizeof(From)) return v;
    else return from_f32<To>(to_f32(v));
}

// filter of a row: -1 past the rows; from Cout on it is a hole
__device__ __forceinline__ int filter_of(const Plan& t, int row)
{
    if (row >= t.rows) return -1;
    if (t.whole) return row;
    const int m = row / t.b.F, i = row - m * t.b.F;
    return (int)(((uint32_t)m * (uint32_t)t.b.inv) % (uint32_t)t.b.P) + t.b.P * i;
}

// The weights of both projections for every tile of 32 filters and K step of 16 channels, in the operand layout of v_mfma_f32_32x32x16_bf16 (64 lanes
// x 8 values, binary32 weights cut into their three bfloat16 pieces), zero where a channel is outside a filter's window; and the table of
// the rows' filters.  One wavefront per (tile, K step, projection).
template <typename From, typename T>
__device__ __forceinline__ void pack(const From* __restrict__ w, char* __restrict__ ws, const Problem& P, const Plan& t, int block)
{
    const int unit = block * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (unit >= t.tiles * t.steps * 2) return;
    const int half = unit & 1, step = unit / 2 % t.steps, tile = unit / 2 / t.steps;
    const int lane = threadIdx.x & 63, f = lane & 31, h = lane >> 5;
    int q0, count;
    walk_of(P, t, tile, q0, count);
    const int k = filter_of(t, tile * kRows + f);
    if (step == 0 && half == 0 && h == 0) ((int*)ws)[tile * kRows + f] = k;

    const int e = 2 * step + h;
    int q = q0 + e;
    q -= q >= t.chunks ? t.chunks : 0;
    const bool real = (e < count) & (k >= 0) & (k < P.Cout);
    const int s = real ? (int)((long long)k * P.stride % P.Cin) : 0;
    const From* const row = w + (size_t)half * P.Cout * P.L + (size_t)(real ? k : 0) * P.L;
    T v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = 8 * q + i;
        int j = c - s;
        j += j < 0 ? P.Cin : 0;
        const bool in = real & (c < P.Cin) & (j < P.L);
        const T x = as<T>(row[in ? j : 0]);
        v[i] = in ? x : T(0);
    }
    u32x4 o[pieces<T>];
    cut8(v, o);
    char* const to = ws + t.a_at + (size_t)((tile * t.steps + step) * 2 + half) * pieces<T> * 1024 + lane * 16;
#pragma unroll
    for (int i = 0; i < pieces<T>; ++i) *(u32x4*)(to + i * 1024) = o[i];
}


// 64 columns x 64 channels through LDS.  TO_PLANES: from samples, to[channel][column], zeros from the last column to `width`; else back.
template <typename From, typename To, bool TO_PLANES>
__device__ __forceinline__ void turn(const Planes& a, const Problem& P, long long width, unsigned block, char* lds)
{
    constexpr int kPitch = 65;
    To* const tile = (To*)lds;                             // [channel][column]
    const unsigned across = (unsigned)((a.channels + 63) / 64);
    const long long q0 = (long long)(block / across) * 64;
    const int c0 = (int)(block % across) * 64, tid = threadIdx.x;
    const From* const from = (const From*)a.from;
    To* const to = (To*)a.to;
    // rows of channels are read and written along the channels, planes along the columns
    auto sample_at = [&](long long q, int c) {
        const long long n = P.HW == 1 ? q : q / P.HW;
        return ((size_t)n * a.channels + c) * P.HW + (P.HW == 1 ? 0 : q - n * P.HW);
    };
    const int lo = tid & 63, hi = tid >> 6;
    From v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int q = TO_PLANES ? hi + 4 * i : lo, c = TO_PLANES ? lo : hi + 4 * i;
        const bool there = q0 + q < P.NQ && c0 + c < a.channels;
        const size_t at = !there ? 0 : TO_PLANES ? sample_at(q0 + q, c0 + c) : (size_t)(c0 + c) * width + q0 + q;
        v[i] = from[at];
        if (!there) v[i] = From(0);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int q = TO_PLANES ? hi + 4 * i : lo, c = TO_PLANES ? lo : hi + 4 * i;
        tile[c * kPitch + q] = as<To>(v[i]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int q = TO_PLANES ? lo : hi + 4 * i, c = TO_PLANES ? hi + 4 * i : lo;
        if (c0 + c >= a.channels || q0 + q >= (TO_PLANES ? width : P.NQ)) continue;
        to[TO_PLANES ? (size_t)(c0 + c) * width + q0 + q : sample_at(q0 + q, c0 + c)] = tile[c * kPitch + q];
    }
}

unsigned blocks_of(long long n, int each) { return (unsigned)((n + each - 1) / each); }

constexpr int kEach = 1024;     // values of a workgroup's share of the weights

template <typename From, typename To>
__global__ __launch_bounds__(256) void gated_prepare(Prepare a, Problem P, Plan t, unsigned planes0, unsigned planes1, unsigned wide)
{
    __shared__ char lds[64 * 65 * sizeof(To)];
    unsigned block = blockIdx.x;
    if (block < planes0) return turn<From, To, true>(a.planes[0], P, a.width, block, lds);
    block -= planes0;
    if (block < planes1) return turn<From, To, true>(a.planes[1], P, a.width, block, lds);
    block -= planes1;
    if (block >= wide) return pack<From, To>((const From*)a.w, a.packed, P, t, (int)(block - wide));
    const long long count = 2ll * a.padded * P.L;
#pragma unroll
    for (int i = 0; i < kEach / 256; ++i) {
        const long long e = (long long)block * kEach + i * 256 + threadIdx.x;
        if (e >= count) return;
        const long long row = e / P.L, j = e - row * P.L, half = row >= a.padded, k = row - half * a.padded;
        ((To*)a.wide)[e] = k < P.Cout ? as<To>(((const From*)a.w)[(half * P.Cout + k) * P.L + j]) : To(0);
    }
}

template <typename From, typename To, typename Grad>
__global__ __launch_bounds__(256) void gated_finish(Finish a, Problem P, unsigned turns)
{
    __shared__ char lds[64 * 65 * sizeof(To)];
    unsigned block = blockIdx.x;
    if (block < turns) return turn<From, To, false>(a.dx, P, a.width, block, lds);
    block -= turns;
    const long long e = (long long)block * 256 + threadIdx.x;
    if (e >= 2ll * P.Cout * P.L) return;
    const long long row = e / P.L, j = e - row * P.L, half = row >= P.Cout, k = row - half * P.Cout;
    const float* const part = a.sum.part + (half * a.padded + k) * P.L + j;
    float v = 0.f;
#pragma unroll 4
    for (int s = 0; s < a.sum.slices; ++s) v += part[(size_t)s * a.sum.count];
    ((Grad*)a.dw)[e] = from_f32<Grad>(v);
}

}  // namespace

template <typename From, typename To>
hipError_t launch_prepare(const Prepare& a, const Problem& p, const Plan& t, hipStream_t st)
{
    auto turns = [&](const Planes& v) { return v.from ? blocks_of(a.width, 64) * blocks_of(v.channels, 64) : 0u; };
    const unsigned n0 = turns(a.planes[0]), n1 = turns(a.planes[1]);
    const unsigned nw = a.wide ? blocks_of(2ll * a.padded * p.L, kEach) : 0u;
    const unsigned np = a.packed ? blocks_of((long long)t.tiles * t.steps * 2, 4) : 0u;
    if (n0 + n1 + nw + np == 0) return hipSuccess;
    gated_prepare<From, To><<<dim3(n0 + n1 + nw + np), dim3(256), 0, st>>>(a, p, t, n0, n1, nw);
    return hipGetLastError();
}

template <typename From, typename To, typename Grad>
hipError_t launch_finish(const Finish& a, const Problem& p, hipStream_t st)
{
    const unsigned turns = a.dx.from ? blocks_of(p.NQ, 64) * blocks_of(a.dx.channels, 64) : 0u;
    const unsigned sums = a.dw ? blocks_of(2ll * p.Cout * p.L, 256) : 0u;
    if (turns + sums == 0) return hipSuccess;
    gated_finish<From, To, Grad><<<dim3(turns + sums), dim3(256), 0, st>>>(a, p, turns);
    return hipGetLastError();
}

template hipError_t launch_prepare<float, float>(const Prepare&, const Problem&, const Plan&, hipStream_t);
template hipError_t launch_prepare<bf16_t, bf16_t>(const Prepare&, const Problem&, const Plan&, hipStream_t);
template hipError_t launch_prepare<bf16_t, float>(const Prepare&, const Problem&, const Plan&, hipStream_t);
template hipError_t launch_finish<float, float, float>(const Finish&, const Problem&, hipStream_t);
template hipError_t launch_finish<float, float, bf16_t>(const Finish&, const Problem&, hipStream_t);
template hipError_t launch_finish<bf16_t, bf16_t, float>(const Finish&, const Problem&, hipStream_t);
template hipError_t launch_finish<bf16_t, bf16_t, bf16_t>(const Finish&, const Problem&, hipStream_t);
template hipError_t launch_finish<float, bf16_t, float>(const Finish&, const Problem&, hipStream_t);
template hipError_t launch_finish<float, bf16_t, bf16_t>(const Finish&, const Problem&, hipStream_t);

}  // namespace gated
}  // namespace scc
