// Gated sliding-channel layer, the opening of a gated feed-forward block: two sliding-channel convolutions of the same input and
// windows, the first through an activation, multiplied:
//   g[n,k,p] = sum_j w[0][k,j] x[n,(s_k+j) mod Cin,p],   u[n,k,p] the same with w[1],   y = act(g) u.
// Declarations shared by its kernels and entry points.
#pragma once
#include "scc_band.h"
#include "scc_common.h"

namespace scc {
namespace gated {

enum { kSilu = 0, kGelu = 1 };

constexpr int kRows = 32;               // filters of a tile: one operand of v_mfma_f32_32x32x16_bf16
constexpr int kLds = 160 << 10;         // bytes of LDS of a CU

// How the filters are cut into tiles.  Rows are filters in the order of their windows' starts (scc_band.h), so a tile's 32 windows
// lie in one short stretch of the channel circle; the circle is held in chunks of 8 channels, the last one filled up with zeros.
// A layer with far fewer filters than windows has its rows in the order of the filters, each tile on the whole circle.
struct Plan {
    Band b;
    int whole;          // rows are filters in their own order
    int rows;           // rows with a filter, or with a hole, where a gradient has to be zero
    int tiles;          // of 32 rows
    int chunks;         // of 8 channels
    int steps;          // K steps of 16 channels of the longest tile
    uint32_t a_at;      // byte offset of the packed weights in the workspace, behind the table of filters
    size_t bytes;       // of both
};

// Filters, rounded up so that a second set of as many behind the first starts on the first window again.
inline long long padded_filters(const Problem& p) { return (long long)(p.Cout + p.period - 1) / p.period * p.period; }

__host__ __device__ inline void walk_of(const Problem& p, const Plan& t, int tile, int& q0, int& count)
{
    q0 = 0;
    count = t.chunks;
    if (t.whole) return;
    const int r1 = tile * kRows + kRows - 1;
    const int m0 = tile * kRows / t.b.F, m1 = (r1 < t.rows ? r1 : t.rows - 1) / t.b.F;
    const long long span = p.L + (long long)t.b.g * (m1 - m0);
    if (span >= p.Cin) return;
    const int first = t.b.g * m0, end = first + (int)span;     // first < Cin
    q0 = first / 8;
    const int n = end <= p.Cin ? (end + 7) / 8 - q0 : t.chunks - q0 + (end - p.Cin + 7) / 8;
    count = n < t.chunks ? n : t.chunks;
}

inline Plan make_plan(const Problem& p, int es, bool grad)
{
    Plan t;
    t.b = make_band(p);
    const long long grid = padded_filters(p);      // P * F
    t.chunks = (p.Cin + 7) / 8;
    // K steps of either order; a tile of the window order spans L + g * (windows - 1) channels
    const long long span = p.L + (long long)t.b.g * ((kRows + t.b.F - 1) / t.b.F);
    const long long by_window = (grid + kRows - 1) / kRows * (span < p.Cin ? span : p.Cin);
    const long long own = grad ? grid : p.Cout;
    t.whole = (own + kRows - 1) / kRows * p.Cin < by_window;
    t.rows = (int)(t.whole ? own : grid);
    t.tiles = (t.rows + kRows - 1) / kRows;
    t.steps = 0;
    for (int i = 0; i < t.tiles; ++i) {
        int q0, count;
        walk_of(p, t, i, q0, count);
        const int s = (count + 1) / 2;
        t.steps = s > t.steps ? s : t.steps;
    }
    t.a_at = (uint32_t)((t.tiles * kRows * 4 + 255) / 256 * 256);
    t.bytes = t.a_at + (size_t)t.tiles * t.steps * 2 * (es == 2 ? 1 : 3) * 1024;
    return t;
}

// What a launch of the product does with a tile of columns.
struct Shape {
    int ct;             // columns are 32 * ct
    int v;              // pixels of a load; 1: single columns
    bool raw;           // binary32 stays whole in LDS and is cut when it is read
    int waves, lds;
    Deal deal;          // (column tile, share of the filter tiles)
};

// false: the layer's channels do not fit LDS
bool make_shape(const Problem& p, const Plan& t, int es, Shape* s);

// What comes before the product: the weights in operand layout, the table of the rows' filters and, for a gradient, what the
// layer of both projections' filters is given (scc_gated_prepare.hip).  A sample of few pixels is a row of channels: the gradient takes
// such layers, and those of few columns, as planes of one sample of all columns, zeros up to `width`.  One launch, from the type of the
// tensors to that of the kernels (binary32 for bfloat16 of few columns).
struct Planes {
    const void* from;       // null: not wanted
    void* to;
    int channels;
};
struct Prepare {
    const void* w;
    char* packed;           // null: no product follows
    void* wide;             // null, or both halves of the weights, each with rows of zeros up to `padded`
    int padded;
    Planes planes[2];       // x and dy
    long long width;
};
template <typename From, typename To>
hipError_t launch_prepare(const Prepare& a, const Problem& p, const Plan& t, hipStream_t st);

// And what comes after: dx from planes (null: it is there), dw from partial sums over slices of the batch, without the padding's rows.
struct Finish {
    Planes dx;
    long long width;
    SliceSum sum;
    void* dw;               // null: it is there
    int padded;
};
template <typename From, typename To, typename Grad>
hipError_t launch_finish(const Finish& a, const Problem& p, hipStream_t st);

// The gradient's first stage: for dy, the two projections are computed again and dh = (dy u act'(g), dy act(g)) is written as the output gradient of
// one layer of 2 * padded filters.
template <typename T>
hipError_t launch_product(const T* x, const char* packed, T* y, const Problem& p, const Plan& t, const Shape& s, int act, hipStream_t st);
template <typename T>
hipError_t launch_product_grad(const T* x, const char* packed, const T* dy, T* dh, int padded, const Problem& p, const Plan& t,
                               const Shape& s, int act, hipStream_t st);

// any shape (scc_gated_any.hip); dy null: y alone is written to out; the second half of w begins w_rows filters behind the first
template <typename T>
hipError_t launch_any(const T* x, const T* w, int w_rows, const T* dy, T* out, int padded, const Problem& p, int act, hipStream_t st);
// one column (scc_gated_any.hip)
bool one_preferred(const Problem& p);
template <typename T>
hipError_t launch_one(const T* x, const T* w, T* y, const Problem& p, int act, hipStream_t st);

// a batch of single tokens and the like (scc_gated_direct.hip)
bool direct_preferred(const Problem& p, int es, bool grad);
template <typename T>
hipError_t launch_direct(const T* x, const T* w, T* y, const Problem& p, int act, hipStream_t st);
// width: of dh's planes, 0 where it is N samples as y is
template <typename T, typename To>
hipError_t launch_direct_grad(const T* x, const T* w, const T* dy, To* dh, int padded, long long width, const Problem& p, int act, hipStream_t st);

// ---- device code that more than one kernel needs ----

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T> constexpr int pieces = sizeof(T) == 2 ? 1 : 3;

// 8 values as one operand piece (bfloat16) or three (binary32, cut)
template <typename T>
__device__ __forceinline__ void cut8(const T (&v)[8], u32x4 (&o)[pieces<T>])
{
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) o[0][e] = (uint32_t)v[2 * e] | (uint32_t)v[2 * e + 1] << 16;
    } else {
        uint32_t hi[4], mid[4], lo[4];
        split3<8>([&](int e) { return v[e]; }, hi, mid, lo);
        o[0] = u32x4{hi[0], hi[1], hi[2], hi[3]};
        o[1] = u32x4{mid[0], mid[1], mid[2], mid[3]};
        o[2] = u32x4{lo[0], lo[1], lo[2], lo[3]};
    }
}

// act(g) and act'(g), binary32; exp2 and the reciprocal are the hardware's (1 ulp).  GELU takes erfc from one exponential that its slope
// needs anyway: erfc(x) = exp(-x^2) q(t), t = 1 / (1 + 0.47 x), x >= 0, the form of Hastings' approximations, with a polynomial q of
// degree 7 fitted here (least absolute error of erfc: 1.2e-8; evaluated in binary32 g Phi(g) is off by 4e-7 at most, half an ulp
// of the larger values).  The library's erfcf is two branches of some 40 instructions, which a wavefront takes both: the dense
// layer of 16000 columns, bf16, 60 us of which 10 were that.
__device__ __forceinline__ void activate(int act, float g, float& a, float& slope)
{
    if (act == kSilu) {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269504f));
        a = g * s;
        slope = fmaf(a, 1.f - s, s);        // s (1 + g (1 - s))
    } else {
        const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(g), 0.47f * 0.70710678f, 1.f));
        const float e = __builtin_amdgcn_exp2f(g * g * -0.72134752f);      // exp(-g^2 / 2)
        float q = 0.5f * 0.08812381843455534f;
        q = fmaf(q, t, 0.5f * -0.4194991704701541f);
        q = fmaf(q, t, 0.5f * 0.6067626861569448f);
        q = fmaf(q, t, 0.5f * -0.1263565474407364f);
        q = fmaf(q, t, 0.5f * 0.337002785814188f);
        q = fmaf(q, t, 0.5f * 0.247573518153275f);
        q = fmaf(q, t, 0.5f * 0.26639289917563896f);
        const float tail = q * t * e;
        const float phi = g < 0.f ? tail : 1.f - tail;
        a = g * phi;
        slope = fmaf(g * 0.39894228f, e, phi);
    }
}

}  // namespace gated
}  // namespace scc
