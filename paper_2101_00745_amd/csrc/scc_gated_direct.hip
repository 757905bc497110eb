// The gated layer of few columns, a batch of single tokens say, in one launch: operands straight from the tensors into registers.
//
// A workgroup takes 16 filters that lie next to each other in the order of their windows' starts, and up to 64 columns; its four wavefronts take the K steps
// of 32 channels of the filters' common stretch of the circle in turn, with v_mfma_f32_16x16x32_bf16 for both projections, and add up
// through LDS.  A lane's 8 channels of a step, and its filter's weights for them, lie one behind the other in memory, and come with one
// load each but where a window begins or ends among them (and on maps, whose pixels are fetched one by one).  What bounds it is latency: a
// launch, the first loads, LDS.  Against the product with weights packed by a launch of their own see direct_preferred.
#include "scc_gated.h"

namespace scc {
namespace gated {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kFilters = 16, kStep = 32, kWaves = 4;

__device__ __forceinline__ f32x4 mfma(const u32x4& a, const u32x4& b, f32x4 c)
{
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <int NP>
__device__ __forceinline__ f32x4 product(const u32x4 (&a)[NP], const u32x4 (&b)[NP], f32x4 c)
{
    if constexpr (NP == 3) {
        c = mfma(a[2], b[0], c);
        c = mfma(a[0], b[2], c);
        c = mfma(a[1], b[1], c);
        c = mfma(a[1], b[0], c);
        c = mfma(a[0], b[1], c);
    }
    return mfma(a[0], b[0], c);
}

template <typename T>
__device__ __forceinline__ void load8(const T* at, T (&v)[8])
{
    typedef T vec __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    const vec r = *(const vec*)at;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = r[e];
}

// The rows that tiles are cut from: filters in the order of their windows (Band), or in their own where there are far fewer than windows.
struct Order {
    Band b;
    int whole, rows;
};

// filter of a row (from Cout on it is a hole) and its window's start; false: past the rows.  Of at most 65536 windows (direct_preferred).
__device__ __forceinline__ bool filter_of(const Order& o, const Problem& P, int row, int& k, int& start)
{
    if (o.whole) {
        k = row;
        start = (int)((long long)row * P.stride % P.Cin);
    } else {
        const int m = row / o.b.F, i = row - m * o.b.F;
        k = (int)(((uint32_t)m * (uint32_t)o.b.inv) % (uint32_t)o.b.P) + o.b.P * i;
        start = m < o.b.P ? o.b.g * m % P.Cin : 0;
    }
    return row < o.rows;
}

// Where results go: y, or with dy dh, both in planes of `width` columns of one sample (zeros past the last) or, width 0, as y.
template <typename T, typename To>
struct Results {
    const T* dy;
    To* out;
    int padded;         // dh only: filters of either half
    long long width;
};

// Q: groups of 16 columns
template <typename T, typename To, int Q, bool GRAD>
__global__ __launch_bounds__(64 * kWaves) void gated_direct(const T* __restrict__ x, const T* __restrict__ w, Results<T, To> R, Problem P,
                                                            Order o, int act)
{
    constexpr int NP = pieces<T>;
    __shared__ float partial[kWaves][2][Q][16][17];         // [projection][columns][filter][column]
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = tid & 15, h = (tid & 63) >> 4;
    const int row0 = (int)blockIdx.x * kFilters;
    const long long c0 = (long long)blockIdx.y * 16 * Q;

    int first = 0, span = P.Cin;
    if (!o.whole) {
        const int last = (row0 + kFilters < o.rows ? row0 + kFilters : o.rows) - 1;
        const long long all = P.L + (long long)o.b.g * (last / o.b.F - row0 / o.b.F);
        first = o.b.g * (row0 / o.b.F) % P.Cin;
        span = all < P.Cin ? (int)all : P.Cin;
    }
    // this lane's filter, of both projections, and its columns; where there is none the first one's, which is not stored
    int k, start;
    const bool real = filter_of(o, P, row0 + r, k, start) & (k < P.Cout);
    const T* const row = w + (size_t)(real ? k : 0) * P.L;
    const T* const second = row + (size_t)P.Cout * P.L;
    const T* column[Q];
#pragma unroll
    for (int c = 0; c < Q; ++c) {
        const long long q = c0 + 16 * c + r, at = q < P.NQ ? q : 0, n = at / P.HW;
        column[c] = x + (size_t)n * P.Cin * P.HW + (at - n * P.HW);
    }
    f32x4 acc[2][Q];
#pragma unroll
    for (int c = 0; c < Q; ++c) acc[0][c] = acc[1][c] = f32x4{};
#pragma unroll 2
    for (int p0 = wave * kStep; p0 < span; p0 += kWaves * kStep) {
        const int pos = p0 + 8 * h;
        int ch = first + (pos < span ? pos : 0);
        ch -= ch >= P.Cin ? P.Cin : 0;
        int j = ch - start;                                 // of the lane's filter, at its first channel
        j += j < 0 ? P.Cin : 0;
        T va[2][8], vb[Q][8];
        if (real & (j + 8 <= P.L) & (pos + 8 <= span)) {
            load8(row + j, va[0]);
            load8(second + j, va[1]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                int at = j + e;
                at -= at >= P.Cin ? P.Cin : 0;
                const bool in = real & (at < P.L) & (pos + e < span);
                const T v0 = row[in ? at : 0], v1 = second[in ? at : 0];
                va[0][e] = in ? v0 : T(0);
                va[1][e] = in ? v1 : T(0);
            }
        }
#pragma unroll
        for (int c = 0; c < Q; ++c) {
            if ((P.HW == 1) & (ch + 8 <= P.Cin)) {
                load8(column[c] + ch, vb[c]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    int at = ch + e;
                    while (at >= P.Cin) at -= P.Cin;        // more than once where there are fewer than 8 channels
                    vb[c][e] = column[c][(size_t)at * P.HW];
                }
            }
        }
        u32x4 a[2][NP];
        cut8(va[0], a[0]);
        cut8(va[1], a[1]);
#pragma unroll
        for (int c = 0; c < Q; ++c) {
            u32x4 o[NP];
            cut8(vb[c], o);
            acc[0][c] = product<NP>(a[0], o, acc[0][c]);
            acc[1][c] = product<NP>(a[1], o, acc[1][c]);
        }
    }
    // acc[.][c][e]: filter 4 * h + e, column 16 * c + r
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int c = 0; c < Q; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) partial[wave][i][c][4 * h + e][r] = acc[i][c][e];
    __syncthreads();
    // Sixteen lanes in a row take what lies in a row: y's filters of a token, dh's columns of a plane.
    const int f = GRAD ? tid >> 4 : r, at = GRAD ? r : tid >> 4;
    if constexpr (GRAD) {
        if (!filter_of(o, P, row0 + f, k, start)) return;
    } else {
        if (!real) return;
    }
#pragma unroll
    for (int c = 0; c < Q; ++c) {
        const long long q = c0 + 16 * c + at;
        if (q >= (GRAD && R.width ? R.width : P.NQ)) continue;
        float g = 0.f, u = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
            g += partial[v][0][c][f][at];
            u += partial[v][1][c][f][at];
        }
        float a, slope;
        activate(act, g, a, slope);
        const long long n = q / P.HW, pixel = q - n * P.HW;
        if constexpr (!GRAD) {
            R.out[((size_t)n * P.Cout + k) * P.HW + pixel] = from_f32<To>(a * u);
        } else {
            const bool there = (k < P.Cout) & (q < P.NQ);
            const float d = there ? to_f32(R.dy[((size_t)n * P.Cout + k) * P.HW + pixel]) : 0.f;
            To* const to = R.out + (R.width ? (size_t)k * R.width + q : ((size_t)n * 2 * R.padded + k) * P.HW + pixel);
            to[0] = from_f32<To>(there ? d * u * slope : 0.f);
            to[(size_t)R.padded * (R.width ? R.width : P.HW)] = from_f32<To>(there ? d * a : 0.f);
        }
    }
}

}  // namespace

namespace {

// rows and channels of a tile
long long channels_of(const Problem& p, const Band& b, bool whole)
{
    const long long span = p.L + (long long)b.g * ((kFilters + b.F - 2) / b.F);
    return whole || span > p.Cin ? p.Cin : span;
}

Order make_order(const Problem& p, bool grad)
{
    Order o;
    o.b = make_band(p);
    const long long grid = (long long)o.b.P * o.b.F, own = grad ? grid : p.Cout;
    auto tiles = [](long long rows) { return (rows + kFilters - 1) / kFilters; };
    o.whole = tiles(own) * p.Cin < tiles(grid) * channels_of(p, o.b, false);
    o.rows = (int)(o.whole ? own : grid);
    return o;
}

template <typename T, typename To, bool GRAD>
hipError_t start(const T* x, const T* w, const Results<T, To>& r, const Problem& p, int act, hipStream_t st)
{
    const Order o = make_order(p, GRAD);
    const unsigned tiles = (unsigned)((o.rows + kFilters - 1) / kFilters);
    const long long columns = r.width ? r.width : p.NQ;
    auto grid = [&](int q) { return dim3(tiles, (unsigned)((columns + 16 * q - 1) / (16 * q))); };
    if (columns <= 16) gated_direct<T, To, 1, GRAD><<<grid(1), dim3(64 * kWaves), 0, st>>>(x, w, r, p, o, act);
    else if (columns <= 32) gated_direct<T, To, 2, GRAD><<<grid(2), dim3(64 * kWaves), 0, st>>>(x, w, r, p, o, act);
    else if (columns <= 48) gated_direct<T, To, 3, GRAD><<<grid(3), dim3(64 * kWaves), 0, st>>>(x, w, r, p, o, act);
    else gated_direct<T, To, 4, GRAD><<<grid(4), dim3(64 * kWaves), 0, st>>>(x, w, r, p, o, act);
    return hipGetLastError();
}

}  // namespace

// Lines in products of one projection, zeros of the tiles among them.  us, packed -> direct.  bf16: 48 tokens 512 -> 1024, cg 2 13.8 -> 5.0, 1024 of them 14.6 -> 10.0,
// 2048 (5e8) 15.9 -> 16.4; 256 tokens 510 -> 1021, co 0.33 (1.3e8) 17.3 -> 13.0, 1024 (5e8) 19.3 -> 24.7; 16 x 256 -> 256 on 16x16, cg 4 (7e7) 10.0 -> 8.4, 64 (3e8)
// 11.7 -> 25.8.  f32: 2048 tokens 31.8 -> 27.0, dense (1e9) 66 -> 63, 4096 dense (2e9) 67 -> 90; 256 x 256 -> 512 on 4x4, cg 2 (3e8) 17.4 -> 18.8.
// All gradients: bf16 256 tokens 512 -> 1024, cg 2 29.5 -> 24.5, 1024 (3e8) 36.9 -> 36.8, 256 x 510 -> 509, co 0.33 32.6 -> 32.9; f32 1024 of these (1.3e8)
// 59 -> 56, 4096 256 -> 512, cg 2 (3e8) 59 -> 66; maps: 64 x 256 -> 512 on 4x4, cg 2 (7e7) bf16 22.7 -> 18.8, f32 29.0 -> 21.3, 64 x 264 -> 512 on 7x7, co 0.25 (2e8)
// 42 -> 51, 50 -> 58.
bool direct_preferred(const Problem& p, int es, bool grad)
{
    const Order o = make_order(p, grad);
    const double products = (double)p.NQ * ((o.rows + kFilters - 1) / kFilters * kFilters) * channels_of(p, o.b, o.whole);
    const bool whole = p.Cin % 8 == 0 && p.L % 8 == 0 && o.b.g % 8 == 0;    // loads of 8 channels
    if (p.NQ > 1 << 20) return false;                                       // grid.y
    if (!o.whole && o.b.P > 65536) return false;                            // filter_of: m * inv is below P^2, and has 32 bits
    const double token = grad ? (es == 4 ? 2e8 : whole ? 1.5e8 : 5e7) : es == 4 ? 1e9 : whole ? 5e8 : 2.5e8;
    const double map = grad || es == 2 ? 1e8 : 2e8;
    return products <= (p.HW > 1 ? map : token);
}

template <typename T>
hipError_t launch_direct(const T* x, const T* w, T* y, const Problem& p, int act, hipStream_t st)
{
    return start<T, T, false>(x, w, Results<T, T>{nullptr, y, 0, 0}, p, act, st);
}

template <typename T, typename To>
hipError_t launch_direct_grad(const T* x, const T* w, const T* dy, To* dh, int padded, long long width, const Problem& p, int act, hipStream_t st)
{
    return start<T, To, true>(x, w, Results<T, To>{dy, dh, padded, width}, p, act, st);
}

#define GRAD_INSTANCE(T, To) \
    template hipError_t launch_direct_grad(const T*, const T*, const T*, To*, int, long long, const Problem&, int, hipStream_t)
GRAD_INSTANCE(float, float);
GRAD_INSTANCE(bf16_t, bf16_t);
GRAD_INSTANCE(bf16_t, float);
template hipError_t launch_direct(const float*, const float*, float*, const Problem&, int, hipStream_t);
template hipError_t launch_direct(const bf16_t*, const bf16_t*, bf16_t*, const Problem&, int, hipStream_t);

}  // namespace gated
}  // namespace scc
