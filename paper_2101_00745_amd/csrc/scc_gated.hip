// The gated layer on the matrix cores (see scc_gated.h): packed weights, a tile of columns on chip for all channels.
//
// A workgroup reads its 32*CT columns of x for ALL channels once, into LDS, in the layout of the
// other operand: chunks of 8 channels of a column, 16 bytes.  After one barrier its wavefronts go their own ways: each takes a tile of filters at a
// time, walks the tile's stretch of the channel circle with the weights coming from L2 straight into registers, and keeps g and u
// of the same filters and columns in the same lanes, so that the activation and the product are register arithmetic and only y is written.
// x crosses the memory bus once and neither projection ever does.
//
// What bounds it: the memory of a large map (f32 128 x 128 -> 512 on 32x32, cg 2: 160 us, where a copy of its 335 MB takes 68 and its
// products, six matrix instructions each, 79), the products of a dense layer (bf16 8 x 2000 tokens 512 -> 1024: 42 us after the weights, 33.5 GFLOP, 0.8 PFLOP/s of the
// 1.3 that a large library product reaches), and in between the filling of LDS, which nothing in the workgroup overlaps
// (f32 128 x 256 -> 256 on 16x16, cg 4: 25 us for 67 MB).  Operands straight from the tensors, with no LDS between, took 29 in place of 32 us there
// and 182 in place of 165 on 32x32, and were not kept.
#include "scc_gated.h"

namespace scc {
namespace gated {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 mfma(const u32x4& a, const u32x4& b, f32x16 c)
{
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// c += a * b: bf16 one product, binary32 six of the nine partial products of the cut factors (what is dropped is below 2^-21)
template <int NP>
__device__ __forceinline__ f32x16 product(const u32x4 (&a)[NP], const u32x4 (&b)[NP], f32x16 c)
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
struct Args {
    const T* x;
    const char* ws;
    const T* dy;    // gradient only
    T* out;         // y, or dh
    Problem p;
    Plan t;
    Groups q;       // groups of V pixels
    int padded;     // gradient only: filters of either half of dh
    Deal deal;      // (column tile, share of the filter tiles)
    int act;
};

// V: pixels of a plane that one load takes, 1: single columns.  LDS: [piece][chunk][column + 1 unused][8 bf16], or with RAW
// [chunk][half][column + 1][4 binary32]; column c of the tile lies at (c % CT) * 32 + c / CT, so that a lane's CT columns of a result are
// neighbours.  The unused column shifts the chunks against each other; lanes next to each other fill V/CT chunks, then the next group (of single
// columns 8 chunks, so that a row of tokens is read in whole cache lines), and so do not meet on the same banks.
template <typename T, int CT, int V, bool RAW, bool GRAD>
__global__ __launch_bounds__(512) void gated_product(Args<T> A)
{
    constexpr bool COLUMNS = V == 1;
    static_assert(!(COLUMNS && GRAD), "the gradient has its columns in planes");
    typedef T lvec __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    typedef T vec __attribute__((ext_vector_type(CT), aligned(sizeof(T))));
    constexpr int NP = pieces<T>;
    constexpr int kCols = 32 * CT, kPitch = (kCols + 1) * 16;
    constexpr int D = NP == 1 && !(GRAD && CT == 4) ? 4 : 2;       // K steps whose weights are in flight (four: 24 registers too many)
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const Problem& P = A.p;
    const Plan& t = A.t;
    int ct, share;
    if (!dealt(A.deal, (int)blockIdx.x, ct, share)) return;     // the whole workgroup leaves
    const int tid = threadIdx.x, threads = blockDim.x, waves = threads >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, f = lane & 31, h = lane >> 5;
    const int piece = t.chunks * kPitch;

    int q0, steps;
    const char* a_at;
    u32x4 a[D][2][NP];
    auto fetch = [&](int slot, int step) {
        const char* const from = a_at + (size_t)(step < steps ? step : steps - 1) * 2 * NP * 1024;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 0; k < NP; ++k) a[slot][i][k] = *(const u32x4*)(from + (i * NP + k) * 1024);
    };
    auto begin = [&](int tile) {            // a tile's walk, and its first weights on their way
        int count;
        walk_of(P, t, tile, q0, count);
        steps = (count + 1) / 2;
        a_at = A.ws + t.a_at + (size_t)tile * t.steps * 2 * NP * 1024 + lane * 16;
#pragma unroll
        for (int d = 0; d < D; ++d) fetch(d, d);
    };
    const int shares = A.deal.inner;
    int tile = share * waves + wave;
    if (tile < t.tiles) begin(tile);

    auto park = [&](int chunk, int column, const T (&v)[8]) {
        const int slot = column % CT * 32 + column / CT;
        if constexpr (RAW) {
            float* const to = (float*)(lds + (size_t)chunk * 2 * kPitch + slot * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                to[e] = v[e];
                to[kPitch / 4 + e] = v[4 + e];
            }
        } else {
            u32x4 o[NP];
            cut8(v, o);
#pragma unroll
            for (int i = 0; i < NP; ++i) *(u32x4*)(lds + i * piece + chunk * kPitch + slot * 16) = o[i];
        }
    };

    // where this lane's columns of a result are: CT pixels of a group, or CT single columns
    uint32_t n[COLUMNS ? CT : 1], px[COLUMNS ? CT : 1];
    bool live[COLUMNS ? CT : 1];
    if constexpr (COLUMNS) {
#pragma unroll
        for (int j = 0; j < CT; ++j) {
            const long long c = (long long)ct * kCols + CT * f + j;
            live[j] = c < P.NQ;
            const uint32_t u = (uint32_t)(live[j] ? c : P.NQ - 1);
            n[j] = u / (uint32_t)P.HW;
            px[j] = u - n[j] * (uint32_t)P.HW;
        }
        const int blocks = (t.chunks + 7) / 8;
        const bool whole = P.HW == 1 && P.Cin % 8 == 0 && ((uintptr_t)A.x & 15u) == 0;
        for (int unit = tid; unit < blocks * 8 * kCols; unit += threads) {
            const int chunk = unit / (8 * kCols) * 8 + (unit & 7), column = unit % (8 * kCols) >> 3;
            if (chunk >= t.chunks) continue;
            const long long c = (long long)ct * kCols + column;
            const uint32_t u = (uint32_t)(c < P.NQ ? c : P.NQ - 1);
            const uint32_t sample = u / (uint32_t)P.HW, pixel = u - sample * (uint32_t)P.HW;
            const T* const from = A.x + (size_t)sample * P.Cin * P.HW + pixel;
            T v[8];
            if (whole) {
#pragma unroll
                for (int i = 0; i < (int)sizeof(T) / 2; ++i)
                    *(u32x4*)((char*)v + 16 * i) = *(const u32x4*)((const char*)(from + 8 * chunk) + 16 * i);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int ch = 8 * chunk + e;
                    const T b = from[(size_t)(ch < P.Cin ? ch : P.Cin - 1) * P.HW];
                    v[e] = ch < P.Cin ? b : T(0);
                }
            }
            park(chunk, column, v);
        }
    } else {
        constexpr int kGroups = kCols / V, S = V / CT;
        const uint32_t base = (uint32_t)ct * kGroups, last = (uint32_t)(A.q.count - 1);
        {
            const uint32_t u = base + CT * f / V;
            live[0] = u <= last;
            column_of_group(live[0] ? u : last, A.q, n[0], px[0]);
            px[0] += CT * f % V;
        }
        const int g = tid / S % kGroups;        // the same in every round: a round's threads are a multiple of S * kGroups
        uint32_t sample, pixel;
        column_of_group(base + g < last ? base + g : last, A.q, sample, pixel);
        const T* const from = A.x + (size_t)sample * P.Cin * P.HW + pixel;
        const int per = threads / kGroups;      // chunks of a round
#pragma unroll 2
        for (int chunk = tid / (S * kGroups) * S + tid % S; chunk < t.chunks; chunk += per) {
            lvec r[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int ch = 8 * chunk + e;
                r[e] = *(const lvec*)(from + (size_t)(ch < P.Cin ? ch : P.Cin - 1) * P.HW);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                T v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 8 * chunk + e < P.Cin ? r[e][j] : T(0);
                park(chunk, g * V + j, v);
            }
        }
    }
    __syncthreads();

    // a filter's plane of these columns is k * HW on from here, which fits 32 bits
    T* out[COLUMNS ? CT : 1];
    const T* grad = nullptr;
#pragma unroll
    for (int j = 0; j < (COLUMNS ? CT : 1); ++j) out[j] = A.out + (size_t)n[j] * (GRAD ? 2 * (size_t)A.padded : (size_t)P.Cout) * P.HW + px[j];
    if constexpr (GRAD) grad = A.dy + (size_t)n[0] * P.Cout * P.HW + px[0];
    while (tile < t.tiles) {
        const int now = tile;
        f32x16 acc[2][CT];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < CT; ++j) acc[i][j] = f32x16{};
        const int* const table = (const int*)A.ws + now * kRows + 4 * h;
        i32x4 filters[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) filters[i] = *(const i32x4*)(table + 8 * i);
        // dy under way while the projections are computed: of rows without a filter, and of columns past the last, the first one's
        vec up[GRAD ? 16 : 1];
        if constexpr (GRAD) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int k = filters[r / 4][r % 4];
                const uint32_t plane = (uint32_t)k < (uint32_t)P.Cout ? (uint32_t)k * (uint32_t)P.HW : 0u;
                up[r] = *(const vec*)(grad + plane);
            }
        }
        for (int s0 = 0; s0 < steps; s0 += D) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                if (s0 + d < steps) {
                    int q = q0 + 2 * (s0 + d) + h;
                    q -= q >= t.chunks ? t.chunks : 0;
#pragma unroll
                    for (int j = 0; j < CT; ++j) {
                        u32x4 b[NP];
                        if constexpr (RAW) {
                            const float* const from = (const float*)(lds + (size_t)q * 2 * kPitch + (32 * j + f) * 16);
                            T v[8];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                v[e] = from[e];
                                v[4 + e] = from[kPitch / 4 + e];
                            }
                            cut8(v, b);
                        } else {
#pragma unroll
                            for (int i = 0; i < NP; ++i) b[i] = *(const u32x4*)(lds + i * piece + q * kPitch + (32 * j + f) * 16);
                        }
                        acc[0][j] = product<NP>(a[d][0], b, acc[0][j]);
                        acc[1][j] = product<NP>(a[d][1], b, acc[1][j]);
                    }
                    if (s0 + d + D < steps) fetch(d, s0 + d + D);
                }
            }
        }
        tile += shares * waves;
        if (tile < t.tiles) begin(tile);

        // acc[.][j][r]: row (r & 3) + 8 * (r >> 2) + 4 * h of the tile, column CT * f + j
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int k = filters[i][e], r = 4 * i + e;
                const bool there = (uint32_t)k < (uint32_t)P.Cout;      // else past the rows, or a hole, whose gradients are zeros
                const uint32_t plane = (uint32_t)k * (uint32_t)P.HW;
                if constexpr (!GRAD) {
                    float y[CT];
#pragma unroll
                    for (int j = 0; j < CT; ++j) {
                        float v, slope;
                        activate(A.act, acc[0][j][r], v, slope);
                        y[j] = v * acc[1][j][r];
                    }
                    if constexpr (COLUMNS) {
#pragma unroll
                        for (int j = 0; j < CT; ++j)
                            if (there & live[j]) out[j][plane] = from_f32<T>(y[j]);
                    } else {
                        vec o;
#pragma unroll
                        for (int j = 0; j < CT; ++j) o[j] = from_f32<T>(y[j]);
                        if (there & live[0]) *(vec*)(out[0] + plane) = o;
                    }
                } else {
                    vec dg, du;
#pragma unroll
                    for (int j = 0; j < CT; ++j) {
                        float v, slope;
                        activate(A.act, acc[0][j][r], v, slope);
                        const float d = to_f32((T)up[r][j]);
                        dg[j] = from_f32<T>(there ? d * acc[1][j][r] * slope : 0.f);
                        du[j] = from_f32<T>(there ? d * v : 0.f);
                    }
                    if ((k >= 0) & live[0]) {
                        *(vec*)(out[0] + plane) = dg;
                        *(vec*)(out[0] + (size_t)A.padded * P.HW + plane) = du;
                    }
                }
            }
        }
    }
}

template <typename T, int CT, int V, bool RAW, bool GRAD>
hipError_t start(const Args<T>& a, const Shape& s, hipStream_t st)
{
    auto* const kernel = gated_product<T, CT, V, RAW, GRAD>;
    static const hipError_t allowed = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (allowed != hipSuccess) return allowed;
    kernel<<<dim3(8u * (unsigned)a.deal.chunk), dim3(64 * s.waves), s.lds, st>>>(a);
    return hipGetLastError();
}

template <typename T, bool GRAD>
hipError_t start_as(const Args<T>& a, const Shape& s, hipStream_t st)
{
    if constexpr (!GRAD) {
        if (s.v == 1) {
            if (s.ct == 1) return s.raw ? start<T, 1, 1, sizeof(T) == 4, false>(a, s, st) : start<T, 1, 1, false, false>(a, s, st);
            if (s.ct == 2) return s.raw ? start<T, 2, 1, sizeof(T) == 4, false>(a, s, st) : start<T, 2, 1, false, false>(a, s, st);
            if constexpr (sizeof(T) == 2) return start<T, 4, 1, false, false>(a, s, st);
        }
    }
    if constexpr (sizeof(T) == 2) {
        switch (s.v * 8 + s.ct) {
            case 32 + 1: return start<T, 1, 4, false, GRAD>(a, s, st);
            case 32 + 2: return start<T, 2, 4, false, GRAD>(a, s, st);
            case 32 + 4: return start<T, 4, 4, false, GRAD>(a, s, st);
            case 64 + 1: return start<T, 1, 8, false, GRAD>(a, s, st);
            case 64 + 2: return start<T, 2, 8, false, GRAD>(a, s, st);
            case 64 + 4: return start<T, 4, 8, false, GRAD>(a, s, st);
            default: return hipErrorInvalidValue;
        }
    } else {
        switch (s.v * 8 + s.ct * 2 + (s.raw ? 1 : 0)) {
            case 32 + 2: return start<T, 1, 4, false, GRAD>(a, s, st);
            case 32 + 4: return start<T, 2, 4, false, GRAD>(a, s, st);
            case 32 + 3: return start<T, 1, 4, true, GRAD>(a, s, st);
            case 32 + 5: return start<T, 2, 4, true, GRAD>(a, s, st);
            default: return hipErrorInvalidValue;
        }
    }
}

int lds_of(const Plan& t, int es, int ct, bool raw) { return t.chunks * (32 * ct + 1) * 16 * (es == 2 ? 1 : raw ? 2 : 3); }

}  // namespace

// Columns of a tile: as many as LDS holds and as leave 192 of the CUs a workgroup, if the filters are shared out too.  us forward with 32, 64 and 128:
// f32 128 x 256 -> 256 on 16x16, cg 4 (512 tiles of 64) 35, 32, -; 128 x 128 -> 512 on 32x32, cg 2 200, 160, -; 16 x 256 -> 256 on 16x16, cg 2 (64 of 64,
// one share) 16.2, 19.2, -; bf16 8 x 2000 tokens 512 -> 1024 dense 63, 52, 45; 32 x 512 -> 512 on 14x14, cg 8 (49 tiles of 128, two shares) 15.0, 12.3,
// 14.7; 64 x 512 -> 1000 on 7x7, cg 2 20, 17, 21.
// Shares of the filters among workgroups with the same columns: about one workgroup a CU.  With 1, 2, 4, 8: f32 16x16 above (one) 32, 43, 77, 93; 7x7 (four) 93,
// 54, 36, 40; bf16 14x14 (two) 15.2, 12.4, 17.3, 21; 2000 tokens (two) 66, 46, 51, 61.
// Binary32 stays whole where its three pieces would take more than half of LDS, a workgroup a CU: cut and whole 16x16 31.3 and 32.1, 32x32 163 and
// 173; 7x7 (512 channels: 196 KB cut, so with 32 columns) 255 and 36.
bool make_shape(const Problem& p, const Plan& t, int es, Shape* s)
{
    s->v = p.HW < 4 ? 1 : es == 2 && p.HW % 8 == 0 ? 8 : 4;
    s->waves = 8;
    if (lds_of(t, es, 1, true) > kLds) return false;
    auto tiles = [&](int c) {
        const long long units = s->v == 1 ? p.NQ : column_groups(p, s->v).count;
        return (units + 32 * c / s->v - 1) / (32 * c / s->v);
    };
    const int most = (t.tiles + s->waves - 1) / s->waves;
    int ct = es == 2 ? 4 : 2;
    while (ct > 1 && (lds_of(t, es, ct, true) > kLds || tiles(ct) * most < 192)) ct /= 2;
    s->ct = ct;
    s->raw = es == 4 && lds_of(t, es, s->ct, false) > kLds / 2;
    s->lds = lds_of(t, es, s->ct, s->raw);
    const long long gx = tiles(s->ct);
    const long long gy = gx >= 192 ? 1 : (256 + gx / 2) / gx < most ? (256 + gx / 2) / gx : most;
    if (gx * gy > 1 << 22) return false;
    s->deal = make_deal(gx, (int)gy);
    return true;
}

template <typename T>
hipError_t launch_product(const T* x, const char* packed, T* y, const Problem& p, const Plan& t, const Shape& s, int act, hipStream_t st)
{
    const Groups q = s.v == 1 ? Groups{1, 0, 1, p.NQ} : column_groups(p, s.v);
    return start_as<T, false>(Args<T>{x, packed, nullptr, y, p, t, q, 0, s.deal, act}, s, st);
}

template <typename T>
hipError_t launch_product_grad(const T* x, const char* packed, const T* dy, T* dh, int padded, const Problem& p, const Plan& t,
                               const Shape& s, int act, hipStream_t st)
{
    const Groups q = s.v == 1 ? Groups{1, 0, 1, p.NQ} : column_groups(p, s.v);
    return start_as<T, true>(Args<T>{x, packed, dy, dh, p, t, q, padded, s.deal, act}, s, st);
}

#define INSTANCES(T)                                                                                                          \
    template hipError_t launch_product(const T*, const char*, T*, const Problem&, const Plan&, const Shape&, int, hipStream_t); \
    template hipError_t launch_product_grad(const T*, const char*, const T*, T*, int, const Problem&, const Plan&, const Shape&, \
                                            int, hipStream_t);
INSTANCES(float)
INSTANCES(bf16_t)

}  // namespace gated
}  // namespace scc
