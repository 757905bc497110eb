// The gated layer beside the matrix cores' kernel: any shape, few columns, and the movements of data around the gradient.
#include "scc_gated.h"

namespace scc {
namespace gated {

namespace {

// Any shape: lanes are columns, a filter at a time, plain binary32 multiply-adds (a vector ALU's worth: for layers whose channels do
// not fit LDS).  Rows from Cout to the padded count are holes.
template <typename T, bool GRAD>
__global__ __launch_bounds__(256) void gated_any(const T* __restrict__ x, const T* __restrict__ w, const T* __restrict__ dy,
                                                 T* __restrict__ out, GradOut o, Problem P, int act)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const long long q = (long long)blockIdx.x * 64 + lane;
    const bool real = q < P.NQ, live = GRAD ? real || (P.HW == 1 && q < o.columns) : real;
    const long long qc = real ? q : 0;
    const long long n = qc / P.HW, p = qc % P.HW;
    const long long to_n = P.HW == 1 ? q : n;
    const T* const col = x + (size_t)n * P.Cin * P.HW + p;
    const int filters = GRAD ? o.padded : P.Cout;
    for (long long k = (long long)blockIdx.y * 4 + wave; k < filters; k += (long long)gridDim.y * 4) {
        const bool there = k < P.Cout;
        float g = 0.f, u = 0.f;
        if (there) {
            int c = (int)(k * P.stride % P.Cin);
            const T* const wg = w + k * P.L;
            const T* const wu = w + ((long long)P.Cout + k) * P.L;
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
        if constexpr (GRAD) {
            const bool zero = !there || !real;
            const float up = zero ? 0.f : to_f32(dy[((size_t)n * P.Cout + k) * P.HW + p]);
            T* const to = out + (size_t)to_n * o.n_stride + (size_t)k * o.k_stride + p;
            if (live) {
                to[0] = from_f32<T>(zero ? 0.f : up * u * slope);
                to[(size_t)o.padded * o.k_stride] = from_f32<T>(zero ? 0.f : up * a);
            }
        } else {
            if (live) out[((size_t)n * P.Cout + k) * P.HW + p] = from_f32<T>(a * u);
        }
    }
}

// Few columns: the weights are what has to be read.  Half a wavefront per projection of a filter, lanes along the window; the
// columns' channels lie in LDS as binary32, the circle continued by a window so that no index wraps.
constexpr int kFew = 4;      // columns at most

template <typename T, int Q>
__global__ __launch_bounds__(256) void gated_few(const T* __restrict__ x, const T* __restrict__ w, T* __restrict__ y, Problem P, int act)
{
    extern __shared__ __attribute__((aligned(16))) float circle[];     // [column][Cin + L]
    const int lane = threadIdx.x & 63, f = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int k = (int)blockIdx.x * 4 + wave;
    const int width = P.Cin + P.L;
    for (int i = threadIdx.x; i < Q * width; i += 256) {
        const int q = i / width, e = i - q * width;
        const int c = e >= P.Cin ? e - P.Cin : e;
        const int n = q / P.HW, p = q - n * P.HW;
        circle[i] = to_f32(x[((size_t)n * P.Cin + c) * P.HW + p]);
    }
    __syncthreads();
    if (k >= P.Cout) return;
    const int s = (int)((long long)k * P.stride % P.Cin);
    const T* const row = w + ((size_t)h * P.Cout + k) * P.L;
    float sum[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) sum[q] = 0.f;
    typedef T vec __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    const int full = P.L & ~7;
    for (int j = 8 * f; j < full; j += 256) {
        const vec v = *(const vec*)(row + j);
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[q] = fmaf(to_f32((T)v[e]), circle[q * width + s + j + e], sum[q]);
    }
    if (full + f < P.L) {
        const float v = to_f32(row[full + f]);
#pragma unroll
        for (int q = 0; q < Q; ++q) sum[q] = fmaf(v, circle[q * width + s + full + f], sum[q]);
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) sum[q] += __shfl_xor(sum[q], off, 64);
        const float u = __shfl_xor(sum[q], 32, 64);
        float a, slope;
        activate(act, sum[q], a, slope);
        if (lane == 0) {
            const int n = q / P.HW, p = q - n * P.HW;
            y[((size_t)n * P.Cout + k) * P.HW + p] = from_f32<T>(a * u);
        }
    }
}

// 64 x 64 values through LDS, four of a row with one access where rows begin on whole groups of four.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(256) void transpose(const T* __restrict__ in, T* __restrict__ out, long long rows, int cols,
                                                 long long in_pitch, long long out_pitch, long long width)
{
    typedef T vec __attribute__((ext_vector_type(4)));
    __shared__ T tile[64][68];
    const unsigned across = (unsigned)((cols + 63) / 64);
    const long long r0 = (long long)(blockIdx.x / across) * 64;
    const int c0 = (int)(blockIdx.x % across) * 64, x = (threadIdx.x & 15) * 4, y = threadIdx.x >> 4;
    vec v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const long long r = r0 + y + 16 * k;
        v[k] = vec{};
        if (r < rows) {
            const T* const from = in + r * in_pitch + c0 + x;
            if (WHOLE) {
                if (c0 + x < cols) v[k] = *(const vec*)from;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c0 + x + e < cols) v[k][e] = from[e];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) tile[x + e][y + 16 * k] = v[k][e];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int c = y + 16 * k;
        if (c0 + c >= cols) continue;
        T* const to = out + (long long)(c0 + c) * out_pitch + r0 + x;
        if (WHOLE) {
            if (r0 + x < width) *(vec*)to = *(const vec*)&tile[c][x];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (r0 + x + e < width) to[e] = tile[c][x + e];
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void spread(const T* __restrict__ w, T* __restrict__ wide, long long filters, long long padded, int L)
{
    const long long e = (long long)blockIdx.x * 256 + threadIdx.x;
    if (e >= 2 * padded * L) return;
    const long long row = e / L, j = e - row * L, half = row >= padded, k = row - half * padded;
    wide[e] = k < filters ? w[(half * filters + k) * L + j] : T(0);
}

template <typename T>
__global__ __launch_bounds__(256) void gather(const float* __restrict__ wide, T* __restrict__ dw, long long filters, long long padded, int L)
{
    const long long e = (long long)blockIdx.x * 256 + threadIdx.x;
    if (e >= 2 * filters * L) return;
    const long long row = e / L, j = e - row * L, half = row >= filters, k = row - half * filters;
    dw[e] = from_f32<T>(wide[(half * padded + k) * L + j]);
}

struct Three {
    const bf16_t* from[3];
    float* to[3];
    int count[3];
};

__global__ __launch_bounds__(256) void widen(Three a)
{
    const int i = (int)blockIdx.y;
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < a.count[i]; e += (long long)gridDim.x * 256) a.to[i][e] = to_f32(a.from[i][e]);
}

__global__ __launch_bounds__(256) void narrow(const float* __restrict__ from, bf16_t* __restrict__ to, int count)
{
    const long long e = (long long)blockIdx.x * 256 + threadIdx.x;
    if (e < count) to[e] = from_f32<bf16_t>(from[e]);
}

unsigned blocks_of(long long n, int each) { return (unsigned)((n + each - 1) / each); }

}  // namespace

template <typename T>
hipError_t launch_any(const T* x, const T* w, const T* dy, T* out, const GradOut& o, const Problem& p, int act, hipStream_t st)
{
    const long long shares = ((dy ? (long long)o.padded : p.Cout) + 15) / 16;
    const dim3 grid(blocks_of(dy && o.columns > p.NQ ? o.columns : p.NQ, 64), (unsigned)(shares < 65535 ? shares : 65535));
    if (dy) gated_any<T, true><<<grid, dim3(256), 0, st>>>(x, w, dy, out, o, p, act);
    else gated_any<T, false><<<grid, dim3(256), 0, st>>>(x, w, dy, out, o, p, act);
    return hipGetLastError();
}

bool few_preferred(const Problem& p) { return p.NQ <= kFew && p.NQ * (long long)(p.Cin + p.L) * 4 <= 64 << 10; }

template <typename T>
hipError_t launch_few(const T* x, const T* w, T* y, const Problem& p, int act, hipStream_t st)
{
    const dim3 grid(blocks_of(p.Cout, 4));
    const int lds = (int)p.NQ * (p.Cin + p.L) * 4;
    switch (p.NQ) {
        case 1: gated_few<T, 1><<<grid, dim3(256), lds, st>>>(x, w, y, p, act); break;
        case 2: gated_few<T, 2><<<grid, dim3(256), lds, st>>>(x, w, y, p, act); break;
        case 3: gated_few<T, 3><<<grid, dim3(256), lds, st>>>(x, w, y, p, act); break;
        default: gated_few<T, 4><<<grid, dim3(256), lds, st>>>(x, w, y, p, act); break;
    }
    return hipGetLastError();
}

template <typename T>
hipError_t launch_transpose(const T* in, T* out, long long rows, int cols, long long in_pitch, long long out_pitch, long long width,
                            hipStream_t st)
{
    const bool whole = cols % 4 == 0 && in_pitch % 4 == 0 && out_pitch % 4 == 0 && width % 4 == 0 &&
                       (((uintptr_t)in | (uintptr_t)out) & (4 * sizeof(T) - 1)) == 0;
    const dim3 grid(blocks_of(width, 64) * blocks_of(cols, 64));
    if (whole) transpose<T, true><<<grid, dim3(256), 0, st>>>(in, out, rows, cols, in_pitch, out_pitch, width);
    else transpose<T, false><<<grid, dim3(256), 0, st>>>(in, out, rows, cols, in_pitch, out_pitch, width);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_spread(const T* w, T* wide, const Problem& p, int padded, hipStream_t st)
{
    spread<T><<<dim3(blocks_of(2ll * padded * p.L, 256)), dim3(256), 0, st>>>(w, wide, p.Cout, padded, p.L);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_gather(const float* wide, T* dw, const Problem& p, int padded, hipStream_t st)
{
    gather<T><<<dim3(blocks_of(2ll * p.Cout * p.L, 256)), dim3(256), 0, st>>>(wide, dw, p.Cout, padded, p.L);
    return hipGetLastError();
}

hipError_t launch_widen(const bf16_t* const (&from)[3], float* const (&to)[3], const int (&count)[3], hipStream_t st)
{
    Three a;
    int most = 0;
    for (int i = 0; i < 3; ++i) {
        a.from[i] = from[i];
        a.to[i] = to[i];
        a.count[i] = count[i];
        most = count[i] > most ? count[i] : most;
    }
    const unsigned blocks = blocks_of(most, 1024);
    widen<<<dim3(blocks, 3), dim3(256), 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_narrow(const float* from, bf16_t* to, int count, hipStream_t st)
{
    narrow<<<dim3(blocks_of(count, 256)), dim3(256), 0, st>>>(from, to, count);
    return hipGetLastError();
}

#define INSTANCES(T)                                                                                                         \
    template hipError_t launch_any(const T*, const T*, const T*, T*, const GradOut&, const Problem&, int, hipStream_t);      \
    template hipError_t launch_few(const T*, const T*, T*, const Problem&, int, hipStream_t);                                \
    template hipError_t launch_transpose(const T*, T*, long long, int, long long, long long, long long, hipStream_t);        \
    template hipError_t launch_spread(const T*, T*, const Problem&, int, hipStream_t);                                       \
    template hipError_t launch_gather(const float*, T*, const Problem&, int, hipStream_t);
INSTANCES(float)
INSTANCES(bf16_t)

}  // namespace gated
}  // namespace scc
