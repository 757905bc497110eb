// The gated layer beside the matrix cores' product: any shape, and one column.
#include "scc_gated.h"

namespace scc {
namespace gated {

namespace {

// Any shape: lanes are columns, a filter at a time, plain binary32 multiply-adds (a vector ALU's worth: for layers whose channels do
// not fit LDS).  Of a gradient, rows from Cout to the padded count are holes.
template <typename T, bool GRAD>
__global__ __launch_bounds__(256) void gated_any(const T* __restrict__ x, const T* __restrict__ w, const T* __restrict__ dy,
                                                 T* __restrict__ out, int w_rows, int padded, Problem P, int act)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const long long q = (long long)blockIdx.x * 64 + lane;
    const bool live = q < P.NQ;
    const long long qc = live ? q : 0;
    const long long n = qc / P.HW, p = qc % P.HW;
    const T* const col = x + (size_t)n * P.Cin * P.HW + p;
    const int filters = GRAD ? padded : P.Cout;
    for (long long k = (long long)blockIdx.y * 4 + wave; k < filters; k += (long long)gridDim.y * 4) {
        const bool there = k < P.Cout;
        float g = 0.f, u = 0.f;
        if (there) {
            int c = (int)(k * P.stride % P.Cin);
            const T* const wg = w + k * P.L;
            const T* const wu = w + ((long long)w_rows + k) * P.L;
#pragma unroll 4
            for (int j = 0; j < P.L; ++j) {
                const float v = to_f32(col[(size_t)c * P.HW]);
                g = fmaf(to_f32(wg[j]), v, g);
                u = fmaf(to_f32(wu[j]), v, u);
                c = c + 1 == P.Cin ? 0 : c + 1;
            }
        }
        float a, slope;
        activate(act, g, a, slope);
        if (!live) continue;
        if constexpr (GRAD) {
            const float up = there ? to_f32(dy[((size_t)n * P.Cout + k) * P.HW + p]) : 0.f;
            T* const to = out + ((size_t)n * 2 * padded + k) * P.HW + p;
            to[0] = from_f32<T>(there ? up * u * slope : 0.f);
            to[(size_t)padded * P.HW] = from_f32<T>(there ? up * a : 0.f);
        } else {
            out[((size_t)n * P.Cout + k) * P.HW + p] = from_f32<T>(a * u);
        }
    }
}

// One column, a single token: the weights are what has to be read.  Half a wavefront per projection of a filter, lanes along the window; the
// column's channels lie in LDS as binary32, the circle continued by a window so that no index wraps.  512 -> 1024, cg 2, bf16, a megabyte of
// weights: 3.2 us, of which a launch alone is 2.3; 1024 -> 1024 dense, f32 4.8 (the matrix cores' kernel for few columns 8.7).
template <typename T>
__global__ __launch_bounds__(256) void gated_one(const T* __restrict__ x, const T* __restrict__ w, T* __restrict__ y, Problem P, int act)
{
    extern __shared__ __attribute__((aligned(16))) float circle[];     // Cin + L
    const int lane = threadIdx.x & 63, f = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int k = (int)blockIdx.x * 4 + wave;
    for (int e = threadIdx.x; e < P.Cin + P.L; e += 256) circle[e] = to_f32(x[e >= P.Cin ? e - P.Cin : e]);
    __syncthreads();
    if (k >= P.Cout) return;
    const int s = (int)((long long)k * P.stride % P.Cin);
    const T* const row = w + ((size_t)h * P.Cout + k) * P.L;
    const float* const window = circle + s;
    float sum = 0.f;
    typedef T vec __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    const int full = P.L & ~7;
    for (int j = 8 * f; j < full; j += 256) {
        const vec v = *(const vec*)(row + j);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(to_f32((T)v[e]), window[j + e], sum);
    }
    if (full + f < P.L) sum = fmaf(to_f32(row[full + f]), window[full + f], sum);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    const float u = __shfl_xor(sum, 32, 64);
    float a, slope;
    activate(act, sum, a, slope);
    if (lane == 0) y[k] = from_f32<T>(a * u);
}

unsigned blocks_of(long long n, int each) { return (unsigned)((n + each - 1) / each); }

}  // namespace

template <typename T>
hipError_t launch_any(const T* x, const T* w, int w_rows, const T* dy, T* out, int padded, const Problem& p, int act, hipStream_t st)
{
    const long long shares = ((dy ? (long long)padded : p.Cout) + 15) / 16;
    const dim3 grid(blocks_of(p.NQ, 64), (unsigned)(shares < 65535 ? shares : 65535));
    if (dy) gated_any<T, true><<<grid, dim3(256), 0, st>>>(x, w, dy, out, w_rows, padded, p, act);
    else gated_any<T, false><<<grid, dim3(256), 0, st>>>(x, w, dy, out, w_rows, padded, p, act);
    return hipGetLastError();
}

bool one_preferred(const Problem& p) { return p.NQ == 1 && (p.Cin + p.L) * 4ll <= 64 << 10; }

template <typename T>
hipError_t launch_one(const T* x, const T* w, T* y, const Problem& p, int act, hipStream_t st)
{
    gated_one<T><<<dim3(blocks_of(p.Cout, 4)), dim3(256), (p.Cin + p.L) * 4, st>>>(x, w, y, p, act);
    return hipGetLastError();
}

#define INSTANCES(T)                                                                                        \
    template hipError_t launch_any(const T*, const T*, int, const T*, T*, int, const Problem&, int, hipStream_t); \
    template hipError_t launch_one(const T*, const T*, T*, const Problem&, int, hipStream_t);
INSTANCES(float)
INSTANCES(bf16_t)

}  // namespace gated
}  // namespace scc
