// Root-mean-square norm over the channels with the residual's addition, its 8-bit output and its gradients.
//
// All of it is bound by memory: forward reads x and r and writes h and y, backward reads x, r, dy and dh and writes dx, each
// element once (128 x 512 x 32x32 fp32: 195 us forward, 5.5 TB/s, 246 backward, 4.4; 4096 x 512 tokens bf16, in the last-level cache: 4.5, and 6.3 with 5.5 for dw's sums).  So a
// token's channels stay in registers between the sum over them and their second use, as they were loaded (bf16 pairs are not widened
// before they are used).  Two layouts: tokens as rows (H*W = 1: the channels of a token are consecutive; a group of 16 to 1024 lanes per token)
// and tokens as columns (a workgroup has some consecutive columns and all their channels: lanes along the pixels, so that a channel's load
// is one piece of 64 or 128 bytes, wavefronts along the channels).  Vectors are 16 bytes; where their width does not divide a row the last one overlaps
// the one before it: both store the same bits, sums count the shared elements once.
#include "scc_norm.h"

namespace scc {
namespace norm {
namespace {

template <typename T, int V> struct VecOf { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };
template <typename T> struct VecOf<T, 1> { typedef T type; };

template <typename T, int V>
struct Vec {
    typename VecOf<T, V>::type v;
    __device__ __forceinline__ float get(int e) const
    {
        if constexpr (V == 1) return to_f32(v);
        else return to_f32((T)v[e]);
    }
    __device__ __forceinline__ void set(int e, float f)
    {
        if constexpr (V == 1) v = from_f32<T>(f);
        else v[e] = from_f32<T>(f);
    }
    __device__ __forceinline__ void load(const T* p) { v = *(const typename VecOf<T, V>::type*)p; }
    __device__ __forceinline__ void store(T* p) const { *(typename VecOf<T, V>::type*)p = v; }
    __device__ __forceinline__ void clear()
    {
        if constexpr (V == 1) v = 0;
        else
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = 0;
    }
};

// Keeps a vector as it was loaded: without it the compiler holds what it has widened for the sums until the second use, twice the registers
template <typename T, int V>
__device__ __forceinline__ void as_loaded(Vec<T, V>& v)
{
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    if constexpr (V * sizeof(T) == 16) {
        words t = __builtin_bit_cast(words, v.v);
        asm volatile("" : "+v"(t));
        v.v = __builtin_bit_cast(typename VecOf<T, V>::type, t);
    }
}

__device__ __forceinline__ float add(float a, float b) { return a + b; }

// Sum of a power of two of values as a tree: log N roundings behind one another instead of N
template <int N>
__device__ __forceinline__ float in_pairs(float (&v)[N])
{
#pragma unroll
    for (int n = N / 2; n > 0; n /= 2)
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] += v[i + n];
    return v[0];
}

// Squares of values beyond 2^60 leave binary32: sums that come out above this are taken again of scaled values.
constexpr float kLargeSum = 1e37f;
constexpr float kShrink = 8.077935669463161e-28f;    // 2^-90: the square of the largest value times 2^31 channels fits

__device__ __forceinline__ float inverse_rms(float sum, float shrink, const Shape& s)
{
    // shrink is 1, or kShrink with the sum of the shrunk squares
    return shrink / sqrtf(sum / (float)s.C + s.eps * shrink * shrink);
}

// The smallest power of two that brings `most` to 448, e4m3's largest value, or less; 1 for 0.  A NaN among y makes no difference here.
__device__ __forceinline__ float scale_of(float most)
{
    const uint32_t b = __float_as_uint(most);
    int k = (int)(b >> 23) - 127 - ((b & 0x7fffffu) <= 0x600000u ? 8 : 7);
    k = k < -120 ? -120 : k > 120 ? 120 : k;
    return most > 0.f ? __uint_as_float((uint32_t)(k + 127) << 23) : 1.f;
}

// e4m3 of v, to nearest even; what is not finite becomes NaN
__device__ __forceinline__ uint32_t e4m3(float v)
{
    const uint32_t q = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false) & 0xffu;
    return fabsf(v) <= 448.f ? q : 0x7fu;
}

template <int V>
__device__ __forceinline__ void store_bytes(uint8_t* to, const uint32_t (&q)[V])
{
    if constexpr (V == 1) {
        *to = (uint8_t)q[0];
    } else if constexpr (V == 2) {
        typedef uint16_t both __attribute__((aligned(1)));
        *(both*)to = (uint16_t)(q[0] | q[1] << 8);
    } else {
        typedef uint32_t words __attribute__((ext_vector_type(V / 4), aligned(1)));
        words o;
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const uint32_t packed = q[4 * i] | q[4 * i + 1] << 8 | q[4 * i + 2] << 16 | q[4 * i + 3] << 24;
            if constexpr (V == 4) { o = packed; } else { o[i] = packed; }
        }
        *(words*)to = o;
    }
}

// The forward pass has a workgroup for each of up to 2^31 tokens or tiles of columns, while a side of a grid has at most 2^32 lanes: two sides
constexpr int kGridSide = 1 << 20;
dim3 grid_of(long long blocks) { return blocks <= kGridSide ? dim3((uint32_t)blocks) : dim3(kGridSide, (uint32_t)((blocks + kGridSide - 1) / kGridSide)); }
__device__ __forceinline__ uint32_t block_of_grid() { return blockIdx.y * kGridSide + blockIdx.x; }

// ---- tokens as rows ----

template <int TPT, typename F>
__device__ __forceinline__ float over_group(float v, float* lds, F&& op)
{
#pragma unroll
    for (int m = 1; m < (TPT < 64 ? TPT : 64); m *= 2) v = op(v, __shfl_xor(v, m));
    if constexpr (TPT > 64) {
        constexpr int W = TPT / 64;
        __syncthreads();                        // the sums of the one before have been read
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        const int first = (threadIdx.x >> 6) / W * W;
        v = lds[first];
#pragma unroll
        for (int i = 1; i < W; ++i) v = op(v, lds[first + i]);
    }
    return v;
}

template <int TPT> constexpr int kRowThreads = TPT < 256 ? 256 : TPT;

// NV vectors of V channels per lane; NV = 0: any number, read again instead of kept
template <typename T, int V, int TPT, int NV, bool BYTES>
__global__ __launch_bounds__(kRowThreads<TPT>) void forward_rows(const T* __restrict__ x, const T* __restrict__ r, const T* __restrict__ w,
                                                                 T* __restrict__ h, void* __restrict__ y, float* __restrict__ scale,
                                                                 Shape s)
{
    __shared__ float lds[TPT > 64 ? kRowThreads<TPT> / 64 : 1];
    const int lane = threadIdx.x % TPT;
    const size_t token = (size_t)block_of_grid() * (kRowThreads<TPT> / TPT) + threadIdx.x / TPT;
    const bool there = token < (size_t)s.N;
    const size_t base = (there ? token : (size_t)s.N - 1) * s.C;
    const int count = NV ? NV : (s.C + V * TPT - 1) / (V * TPT);
    Vec<T, V> xs[NV ? NV : 1], rs[NV ? NV : 1], gs[NV ? NV : 1];
    auto place = [&](int j) { return (lane + j * TPT) * V; };
    auto start = [&](int at) { return at < s.C - V ? at : s.C - V; };
    // lanes behind the last channel read the last vector, none of which counts for them: no load waits for a branch
    auto fetch = [&](int j, int k) {
        const int from = start(place(j));
        xs[k].load(x + base + from);
        if (r) rs[k].load(r + base + from);
        else rs[k].clear();
        gs[k].load(w + from);
    };
    if constexpr (NV > 0)
#pragma unroll
        for (int j = 0; j < NV; ++j) fetch(j, j);
    float shrink = 1.f, sum;
    for (;;) {
        sum = 0.f;
#pragma unroll
        for (int j = 0; j < count; ++j) {
            const int k = NV ? j : 0;
            if constexpr (NV == 0) fetch(j, 0);
            const int at = place(j);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float v = (xs[k].get(e) + rs[k].get(e)) * shrink;
                if (start(at) + e >= at) sum = fmaf(v, v, sum);
            }
        }
        sum = over_group<TPT>(sum, lds, add);
        if (sum < kLargeSum || shrink != 1.f) break;
        shrink = kShrink;
    }
    const float rstd = inverse_rms(sum, shrink, s);
    auto value = [&](int k, int e) { return (xs[k].get(e) + rs[k].get(e)) * rstd * gs[k].get(e); };
    float unit = 1.f, inverse = 1.f;
    if constexpr (BYTES) {
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < count; ++j) {
            const int k = NV ? j : 0;
            if constexpr (NV == 0) fetch(j, 0);
#pragma unroll
            for (int e = 0; e < V; ++e) most = fmaxf(most, fabsf(value(k, e)));
        }
        unit = scale_of(over_group<TPT>(most, lds, fmaxf));
        inverse = 1.f / unit;
        if (there && lane == 0) scale[token] = unit;
    }
    if (!there) return;
#pragma unroll
    for (int j = 0; j < count; ++j) {
        const int k = NV ? j : 0, at = place(j);
        if constexpr (NV == 0) fetch(j, 0);
        if (at >= s.C) continue;
        const size_t to = base + start(at);
        Vec<T, V> o;
        if constexpr (BYTES) {
            uint32_t q[V];
#pragma unroll
            for (int e = 0; e < V; ++e) q[e] = e4m3(value(k, e) * inverse);
            store_bytes<V>((uint8_t*)y + to, q);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) o.set(e, value(k, e));
            o.store((T*)y + to);
        }
        if (h) {
#pragma unroll
            for (int e = 0; e < V; ++e) o.set(e, xs[k].get(e) + rs[k].get(e));
            o.store(h + to);
        }
    }
}

// A group of lanes takes every gridDim.x * groups'th token; one row of dw's sums for each workgroup.
template <typename T, int V, int TPT, int NV>
__global__ __launch_bounds__(kRowThreads<TPT>) void backward_rows(const T* __restrict__ x, const T* __restrict__ r, const T* __restrict__ w,
                                                                  const T* __restrict__ dy, const T* __restrict__ dh, T* __restrict__ dx, float* __restrict__ part,
                                                                  Shape s)
{
    constexpr int kGroups = kRowThreads<TPT> / TPT;
    __shared__ float lds[TPT > 64 ? kRowThreads<TPT> / 64 : 1];
    const int lane = threadIdx.x % TPT;
    const size_t groups = (size_t)gridDim.x * kGroups;
    auto place = [&](int j) { return (lane + j * TPT) * V; };
    auto start = [&](int at) { return at < s.C - V ? at : s.C - V; };
    float sums[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) sums[j][e] = 0.f;
    // every group of a workgroup makes as many rounds, the last perhaps on a token that is none
    for (size_t first = (size_t)blockIdx.x * kGroups; first < (size_t)s.N; first += groups) {
        const size_t token = first + threadIdx.x / TPT;
        const bool there = token < (size_t)s.N;
        const size_t base = (there ? token : (size_t)s.N - 1) * s.C;
        Vec<T, V> xs[NV], rs[NV], ds[NV], gs[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int from = start(place(j));
            xs[j].load(x + base + from);
            if (r) rs[j].load(r + base + from);
            else rs[j].clear();
            ds[j].load(dy + base + from);
            gs[j].load(w + from);
        }
        float shrink = 1.f, sum, dot;
        for (;;) {
            sum = dot = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int at = place(j);
                    const float v = start(at) + e >= at ? (xs[j].get(e) + rs[j].get(e)) * shrink : 0.f;
                    sum = fmaf(v, v, sum);
                    dot = fmaf(ds[j].get(e) * gs[j].get(e), v, dot);
                }
            sum = over_group<TPT>(sum, lds, add);
            dot = over_group<TPT>(dot, lds, add);
            if (sum < kLargeSum || shrink != 1.f) break;
            shrink = kShrink;
        }
        const float rstd = inverse_rms(sum, shrink, s);
        const float inner = dot * (rstd / shrink) / (float)s.C;      // mean_c(a h s)
        if (!there) continue;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            as_loaded(xs[j]);
            as_loaded(rs[j]);
            as_loaded(ds[j]);
            as_loaded(gs[j]);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int at = place(j);
            if (at >= s.C) continue;
            Vec<T, V> extra, o;
            extra.clear();
            if (dh) extra.load(dh + base + start(at));
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float hat = (xs[j].get(e) + rs[j].get(e)) * rstd, d = ds[j].get(e);
                o.set(e, fmaf(d * gs[j].get(e) - hat * inner, rstd, extra.get(e)));
                sums[j][e] = fmaf(d, hat, sums[j][e]);
            }
            o.store(dx + base + start(at));
        }
    }
    constexpr int kMost = V * TPT * NV;         // channels
    __shared__ float rows[kGroups > 1 ? kGroups * kMost : 1];
    float* const to = kGroups > 1 ? rows + threadIdx.x / TPT * kMost : part + (size_t)blockIdx.x * s.C;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int at = place(j);
            if (at < s.C && start(at) + e >= at) to[start(at) + e] = sums[j][e];
        }
    if constexpr (kGroups > 1) {
        __syncthreads();
        for (int c = threadIdx.x; c < s.C; c += kRowThreads<TPT>) {
            float v[kGroups];
#pragma unroll
            for (int i = 0; i < kGroups; ++i) v[i] = rows[i * kMost + c];
            part[(size_t)blockIdx.x * s.C + c] = in_pairs(v);
        }
    }
}

// ---- tokens as columns ----

// The i'th tile of workgroup `block` of `blocks`, a multiple of 8; -1: none.  Workgroups go to the XCDs in turn, and with `runs` each of these takes a run of
// tiles: where planes do not end at a line of the L2 neighbouring tiles share lines (8 x 512 x 2000 bf16: backward 24.2 -> 19.8 us; where they do, it is 261
// instead of 242 for 128 x 512 x 32x32 fp32).
__device__ __forceinline__ long long tile_of(uint32_t block, uint32_t blocks, uint32_t i, uint32_t tiles, bool runs)
{
    if (!runs) return block + (long long)i * blocks < tiles ? block + (long long)i * blocks : -1;
    const uint32_t each = (tiles + 7) / 8, in_run = (block >> 3) + i * (blocks >> 3), tile = (block & 7) * each + in_run;
    return in_run < each && tile < tiles ? (long long)tile : -1;
}

// LANES groups of V columns, THREADS / LANES channels at a time, NV times that in registers (0: any number, read again)
template <int V, int LANES, int THREADS, int SUMS>
struct Columns {
    static constexpr int kRows = THREADS / LANES, kWaves = THREADS / 64;
    float lds[SUMS][kWaves][LANES * V];

    // Sums (or what else op is) over all channels of each of the workgroup's columns, SUMS of them at a time; finish(column, totals) in one thread for each
    // column, which leaves what the others are to see in totals, and says whether the sums have to be taken again; then v is that of the thread's columns.
    // True if any column's have to.
    template <typename F, typename G>
    __device__ __forceinline__ bool reduce(float (&v)[SUMS][V], F&& op, G&& finish)
    {
#pragma unroll
        for (int i = 0; i < SUMS; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e)
#pragma unroll
                for (int m = LANES; m < 64; m *= 2) v[i][e] = op(v[i][e], __shfl_xor(v[i][e], m));
        __syncthreads();
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
        if (lane < LANES)
#pragma unroll
            for (int i = 0; i < SUMS; ++i)
#pragma unroll
                for (int e = 0; e < V; ++e) lds[i][wave][lane * V + e] = v[i][e];
        __syncthreads();
        bool again = false;
        if (threadIdx.x < LANES * V) {
            float total[SUMS];
#pragma unroll
            for (int i = 0; i < SUMS; ++i) {
                total[i] = lds[i][0][threadIdx.x];
#pragma unroll
                for (int j = 1; j < kWaves; ++j) total[i] = op(total[i], lds[i][j][threadIdx.x]);
            }
            again = finish((int)threadIdx.x, total);
#pragma unroll
            for (int i = 0; i < SUMS; ++i) lds[i][0][threadIdx.x] = total[i];
        }
        again = __syncthreads_or(again);
#pragma unroll
        for (int i = 0; i < SUMS; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) v[i][e] = lds[i][0][(threadIdx.x % LANES) * V + e];
        return again;
    }
};

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> where(bool there, Vec<T, V> v)
{
    Vec<T, V> none;
    none.clear();
    return there ? v : none;
}

template <typename T, int V, int LANES, int THREADS, int NV, bool BYTES>
__global__ __launch_bounds__(THREADS) void forward_columns(const T* __restrict__ x, const T* __restrict__ r, const T* __restrict__ w,
                                                           T* __restrict__ h, void* __restrict__ y, float* __restrict__ scale, Shape s,
                                                           Groups groups)
{
    typedef Columns<V, LANES, THREADS, 1> Cols;
    __shared__ Cols cols;
    const long long tile = tile_of(block_of_grid(), 8, 0, ((uint32_t)groups.count + LANES - 1) / LANES, true);
    if (tile < 0) return;
    const uint32_t group = (uint32_t)tile * LANES + threadIdx.x % LANES;
    const bool there = group < (uint32_t)groups.count;
    uint32_t n, p;
    column_of_group(there ? group : (uint32_t)groups.count - 1, groups, n, p);
    const size_t base = (size_t)n * s.C * s.HW + p;
    const int row = threadIdx.x / LANES;
    const int count = NV ? NV : (s.C + Cols::kRows - 1) / Cols::kRows;
    Vec<T, V> xs[NV ? NV : 1], rs[NV ? NV : 1];
    float gs[NV ? NV : 1];
    // rows behind the last channel read that one and count as zeros: no load waits for a branch
    auto fetch = [&](int j, int k) {
        const int c = row + j * Cols::kRows, from = c < s.C ? c : s.C - 1;
        xs[k].load(x + base + (size_t)from * s.HW);
        if (r) rs[k].load(r + base + (size_t)from * s.HW);
        else rs[k].clear();
        gs[k] = to_f32(w[from]);
    };
    if constexpr (NV > 0)
#pragma unroll
        for (int j = 0; j < NV; ++j) fetch(j, j);
    float rstd[1][V], shrink = 1.f, kept = 0.f;
    for (bool redo = false;;) {
#pragma unroll
        for (int e = 0; e < V; ++e) rstd[0][e] = 0.f;
#pragma unroll
        for (int j = 0; j < count; ++j) {
            const int k = NV ? j : 0;
            if constexpr (NV == 0) fetch(j, 0);
            const bool live = row + j * Cols::kRows < s.C;
            if (NV > 0) {
                xs[k] = where(live, xs[k]);
                rs[k] = where(live, rs[k]);
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float v = live ? (xs[k].get(e) + rs[k].get(e)) * shrink : 0.f;
                rstd[0][e] = fmaf(v, v, rstd[0][e]);
            }
        }
        const bool first = shrink == 1.f;
        const bool again = cols.reduce(rstd, add, [&](int, float (&total)[1]) {
            // a column whose sum left binary32 is taken again; what the others had stays
            const bool large = first && !(total[0] < kLargeSum);
            if (first || redo) kept = inverse_rms(total[0], shrink, s);
            redo = large;
            total[0] = kept;
            return large;
        });
        if (!again) break;
        shrink = kShrink;
    }
    if constexpr (NV > 0)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            as_loaded(xs[j]);
            as_loaded(rs[j]);
        }
    auto value = [&](int k, int e) { return (xs[k].get(e) + rs[k].get(e)) * rstd[0][e] * gs[k]; };
    float inverse[V];
    if constexpr (BYTES) {
        float most[1][V];
#pragma unroll
        for (int e = 0; e < V; ++e) most[0][e] = 0.f;
#pragma unroll
        for (int j = 0; j < count; ++j) {
            const int k = NV ? j : 0;
            if constexpr (NV == 0) fetch(j, 0);
#pragma unroll
            for (int e = 0; e < V; ++e) most[0][e] = fmaxf(most[0][e], fabsf(value(k, e)));
        }
        cols.reduce(most, fmaxf, [](int, float (&)[1]) { return false; });
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float unit = scale_of(most[0][e]);
            inverse[e] = 1.f / unit;
            if (there && row == 0) scale[(size_t)n * s.HW + p + e] = unit;
        }
    }
    if (!there) return;
#pragma unroll
    for (int j = 0; j < count; ++j) {
        const int k = NV ? j : 0, c = row + j * Cols::kRows;
        if constexpr (NV == 0) fetch(j, 0);
        if (c >= s.C) continue;
        const size_t to = base + (size_t)c * s.HW;
        Vec<T, V> o;
        if constexpr (BYTES) {
            uint32_t q[V];
#pragma unroll
            for (int e = 0; e < V; ++e) q[e] = e4m3(value(k, e) * inverse[e]);
            store_bytes<V>((uint8_t*)y + to, q);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) o.set(e, value(k, e));
            o.store((T*)y + to);
        }
        if (h) {
#pragma unroll
            for (int e = 0; e < V; ++e) o.set(e, xs[k].get(e) + rs[k].get(e));
            o.store(h + to);
        }
    }
}

// A workgroup takes every gridDim.x'th tile and keeps its sums of dw in registers; with NV = 0, where it may have any number of channels, in its row of
// the workspace, which only it writes.
template <typename T, int V, int LANES, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void backward_columns(const T* __restrict__ x, const T* __restrict__ r, const T* __restrict__ w,
                                                            const T* __restrict__ dy, const T* __restrict__ dh, T* __restrict__ dx,
                                                            float* __restrict__ part, Shape s,
                                                            Groups groups)
{
    typedef Columns<V, LANES, THREADS, 2> Cols;
    __shared__ Cols cols;
    const int row = threadIdx.x / LANES;
    const int count = NV ? NV : (s.C + Cols::kRows - 1) / Cols::kRows;
    const uint32_t tiles = ((uint32_t)groups.count + LANES - 1) / LANES;
    float sums[NV ? NV : 1];
#pragma unroll
    for (int j = 0; j < (NV ? NV : 1); ++j) sums[j] = 0.f;
    auto over_lanes = [&](float v) {
#pragma unroll
        for (int m = 1; m < LANES; m *= 2) v += __shfl_xor(v, m);
        return v;
    };
    const bool runs = (size_t)s.HW * sizeof(T) % 128 != 0;
    long long tile = tile_of(blockIdx.x, gridDim.x, 0, tiles, runs);
    if (NV == 0 && tile < 0)                    // a row of sums all the same
        for (int c = threadIdx.x; c < s.C; c += THREADS) part[(size_t)blockIdx.x * s.C + c] = 0.f;
    for (uint32_t i = 0; tile >= 0; tile = tile_of(blockIdx.x, gridDim.x, ++i, tiles, runs)) {
        const uint32_t group = (uint32_t)tile * LANES + threadIdx.x % LANES;
        const bool there = group < (uint32_t)groups.count;
        const uint32_t u = there ? group : (uint32_t)groups.count - 1;
        uint32_t n, p;
        column_of_group(u, groups, n, p);
        const uint32_t own = (u - n * (uint32_t)groups.per) * V - p;    // columns of this group that the one before it has
        const size_t base = (size_t)n * s.C * s.HW + p;
        Vec<T, V> xs[NV ? NV : 1], rs[NV ? NV : 1], ds[NV ? NV : 1];
        float gs[NV ? NV : 1];
        auto fetch = [&](int j, int k) {
            const int c = row + j * Cols::kRows, from = c < s.C ? c : s.C - 1;
            xs[k].load(x + base + (size_t)from * s.HW);
            if (r) rs[k].load(r + base + (size_t)from * s.HW);
            else rs[k].clear();
            ds[k].load(dy + base + (size_t)from * s.HW);
            gs[k] = to_f32(w[from]);
        };
        if constexpr (NV > 0)
#pragma unroll
            for (int j = 0; j < NV; ++j) fetch(j, j);
        float both[2][V], shrink = 1.f, kept[2] = {};         // sums of h^2 and of a h, then 1 / rms and mean_c(a h / rms)
        for (bool redo = false;;) {
#pragma unroll
            for (int e = 0; e < V; ++e) both[0][e] = both[1][e] = 0.f;
#pragma unroll
            for (int j = 0; j < count; ++j) {
                const int k = NV ? j : 0;
                if constexpr (NV == 0) fetch(j, 0);
                const bool live = row + j * Cols::kRows < s.C;
                if (NV > 0) {
                    xs[k] = where(live, xs[k]);
                    rs[k] = where(live, rs[k]);
                    ds[k] = where(live, ds[k]);
                }
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float v = live ? (xs[k].get(e) + rs[k].get(e)) * shrink : 0.f;
                    both[0][e] = fmaf(v, v, both[0][e]);
                    both[1][e] = fmaf(ds[k].get(e) * gs[k], v, both[1][e]);
                }
            }
            const bool first = shrink == 1.f;
            const bool again = cols.reduce(both, add, [&](int, float (&total)[2]) {
                const bool large = first && !(total[0] < kLargeSum);
                if (first || redo) {
                    kept[0] = inverse_rms(total[0], shrink, s);
                    kept[1] = total[1] * (kept[0] / shrink) / (float)s.C;
                }
                redo = large;
                total[0] = kept[0];
                total[1] = kept[1];
                return large;
            });
            if (!again) break;
            shrink = kShrink;
        }
        if constexpr (NV > 0)
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                as_loaded(xs[j]);
                as_loaded(rs[j]);
                as_loaded(ds[j]);
            }
#pragma unroll
        for (int j = 0; j < count; ++j) {
            const int k = NV ? j : 0, c = row + j * Cols::kRows;
            if constexpr (NV == 0) fetch(j, 0);
            float mine = 0.f;
            if (c < s.C && there) {
                const size_t at = base + (size_t)c * s.HW;
                Vec<T, V> extra, o;
                extra.clear();
                if (dh) extra.load(dh + at);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const float hat = (xs[k].get(e) + rs[k].get(e)) * both[0][e], d = ds[k].get(e);
                    o.set(e, fmaf(d * gs[k] - hat * both[1][e], both[0][e], extra.get(e)));
                    if ((uint32_t)e >= own) mine = fmaf(d, hat, mine);
                }
                o.store(dx + at);
            }
            if constexpr (NV > 0) {
                sums[j] += mine;
            } else {
                mine = over_lanes(mine);
                if (threadIdx.x % LANES == 0 && c < s.C) {
                    float* to = part + (size_t)blockIdx.x * s.C + c;
                    *to = i == 0 ? mine : *to + mine;
                }
            }
        }
    }
    if constexpr (NV > 0)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = row + j * Cols::kRows;
            const float v = over_lanes(sums[j]);
            if (threadIdx.x % LANES == 0 && c < s.C) part[(size_t)blockIdx.x * s.C + c] = v;
        }
}

// dw[c] = sum over rows of part[row][c], in a fixed order: 16 wavefronts take the rows in turn, 64 channels a workgroup
template <typename D>
__global__ __launch_bounds__(1024) void weight_sums(const float* __restrict__ part, D* __restrict__ dw, int rows, int C)
{
    __shared__ float lds[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    float sum = 0.f;
    if (c < C)
        for (int i = wave; i < rows; i += 8 * 16) {     // eight rows under way
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = part[(size_t)(i + j * 16 < rows ? i + j * 16 : rows - 1) * C + c];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = i + j * 16 < rows ? v[j] : 0.f;
            sum += in_pairs(v);
        }
    lds[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && c < C) {
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = lds[i][lane];
        dw[c] = from_f32<D>(in_pairs(v));
    }
}

// ---- which form a shape takes ----

// Vectors that a token's channels (or a plane's pixels) are read in: 16 bytes where there are as many.
template <typename T> constexpr int kWide = 16 / (int)sizeof(T);

constexpr int kKept = 4;            // most vectors of a lane that stay in registers

// f(V, TPT, NV) as constants for tokens as rows: as few lanes a token as keep its channels in one or two vectors of a lane, so that a wavefront or four sum without the
// others, and up to 1024 tokens, where a token's time counts, one vector of as many lanes as it takes.  bf16, forward / backward in us: 1024 channels, 64 tokens: 256 lanes
// 2.6 / 6.4, 64 lanes 2.9 / 6.1; 32768 tokens: 42 / 69 and 39 / 55.  4096 channels, one token: 1024 lanes 2.9 / 7.5, 256 lanes 3.0 / 8.0; 4096 tokens: 23 / 55 and 21 / 44.
template <typename T, typename F>
hipError_t with_rows(const Shape& s, F&& f)
{
    typedef std::integral_constant<int, 1> one;
    typedef std::integral_constant<int, 2> two;
    typedef std::integral_constant<int, kKept> kept;
    typedef std::integral_constant<int, 16> quarter;
    typedef std::integral_constant<int, 64> wave;
    typedef std::integral_constant<int, 256> four;
    typedef std::integral_constant<int, 1024> all;
    const int C = s.C;
    const bool few = s.N <= 1024;
    constexpr int V = kWide<T>;
    const std::integral_constant<int, V> v;
    if (C < V) return f(one(), quarter(), one());
    if (C <= V * 16) return f(v, quarter(), one());
    if (C <= V * 32 && !few) return f(v, quarter(), two());
    if (C <= V * 64) return f(v, wave(), one());
    if (C <= V * 128 && !few) return f(v, wave(), two());
    if (C <= V * 256) return f(v, four(), one());
    if (C <= V * 1024) return few ? f(v, all(), one()) : f(v, four(), kept());
    if (C <= V * 1024 * kKept) return f(v, all(), kept());
    return f(v, all(), std::integral_constant<int, 0>());
}

Groups groups_of(const Shape& s, int V)
{
    Problem p = {};
    p.N = s.N;
    p.HW = s.HW;
    return column_groups(p, V);
}

// f(V, LANES, THREADS, NV) as constants for tokens as columns.  V: 16 bytes of a plane, less where it has less.  A workgroup's piece of a plane is 128 bytes, of
// channels that do not fit into registers too, which are then read twice, the second time out of the last-level cache (64 x 1000 x 16x16 fp32: 4.4 TB/s
// forward, in pieces of 64 bytes that fit 4.2; 26 x 2016: 4.4, in pieces of 32 bytes 2.1); 64 or 32 bytes only where there were not 64 workgroups otherwise, 64 bytes read again
// only for 128 (8 x 2048 x 250 fp32, 126 of these: 37 us forward, 51 backward; 32 bytes that stay: 21 and 32).
template <typename T, typename F>
hipError_t with_columns(const Shape& s, F&& f)
{
    auto width = [&](auto v, auto whole) {
        constexpr int V = decltype(v)::value, L = decltype(whole)::value;
        typedef std::integral_constant<int, L / 2> half;
        typedef std::integral_constant<int, L / 4> quarter;
        typedef std::integral_constant<int, 256> few;
        typedef std::integral_constant<int, 1024> all;
        typedef std::integral_constant<int, kKept> kept;
        typedef std::integral_constant<int, 0> again;
        const long long groups = groups_of(s, V).count;
        auto enough = [&](int lanes, int blocks = 64) { return (groups + lanes - 1) / lanes >= blocks; };
        auto fits = [&](int lanes) { return s.C <= 1024 / lanes * kKept; };
        if (s.C <= 256 / L * kKept) return f(v, whole, few(), kept());
        if constexpr (V > 1) {
            if (fits(L) && (enough(L) || s.C < 2048 / L)) return f(v, whole, all(), kept());
            if (enough(L)) return f(v, whole, all(), again());
            if (fits(L / 2) && (enough(L / 2) || s.C < 4096 / L)) return f(v, half(), all(), kept());
            if (enough(L / 2, 128)) return f(v, half(), all(), again());
            if (fits(L / 4)) return f(v, quarter(), all(), kept());
            return f(v, quarter(), all(), again());
        } else {
            return f(v, whole, all(), again());     // single pixels come here with few channels or with more than as rows fit, both backward
        }
    };
    if (s.HW >= kWide<T>) return width(std::integral_constant<int, kWide<T>>(), std::integral_constant<int, 8>());
    if (kWide<T> > 4 && s.HW >= 4) return width(std::integral_constant<int, 4>(), std::integral_constant<int, 16>());
    if (s.HW >= 2) return width(std::integral_constant<int, 2>(), std::integral_constant<int, sizeof(T) == 4 ? 16 : 32>());
    return width(std::integral_constant<int, 1>(), std::integral_constant<int, 32>());
}

constexpr int kSumRows = 1024;      // most rows of dw's sums, one for each workgroup

// Workgroups of the backward pass and the rows of sums that they leave
struct Grid {
    int blocks, rows;
};

template <typename T>
Grid backward_grid(const Shape& s)
{
    Grid g = {1, 1};
    // tokens as rows, of too many channels for registers: as planes of one pixel
    const bool rows = s.HW == 1 && s.C <= kWide<T> * 1024 * kKept && s.C >= kWide<T>;
    if (rows) {
        (void)with_rows<T>(s, [&](auto, auto tpt, auto) {
            constexpr int TPT = decltype(tpt)::value, G = kRowThreads<TPT> / TPT;
            const int most = (int)(((long long)s.N + G - 1) / G);
            g.blocks = g.rows = most < kSumRows ? most : kSumRows;
            return hipSuccess;
        });
    } else {
        (void)with_columns<T>(s, [&](auto v, auto lanes, auto threads, auto) {
            const long long tiles = (groups_of(s, decltype(v)::value).count + decltype(lanes)::value - 1) / decltype(lanes)::value;
            const int wanted = decltype(threads)::value == 256 ? kSumRows : 512;
            g.blocks = g.rows = (int)(tiles < wanted ? (tiles + 7) / 8 * 8 : wanted);
            return hipSuccess;
        });
    }
    return g;
}

}  // namespace

template <typename T>
hipError_t launch_forward(const T* x, const T* r, const T* w, T* h, void* y, float* scale, const Shape& s, hipStream_t st)
{
    if (s.HW == 1)
        return with_rows<T>(s, [&](auto v, auto tpt, auto nv) {
            constexpr int V = decltype(v)::value, TPT = decltype(tpt)::value, NV = decltype(nv)::value, G = kRowThreads<TPT> / TPT;
            const dim3 blocks = grid_of(((long long)s.N + G - 1) / G);
            if (scale) forward_rows<T, V, TPT, NV, true><<<blocks, kRowThreads<TPT>, 0, st>>>(x, r, w, h, y, scale, s);
            else forward_rows<T, V, TPT, NV, false><<<blocks, kRowThreads<TPT>, 0, st>>>(x, r, w, h, y, scale, s);
            return hipGetLastError();
        });
    return with_columns<T>(s, [&](auto v, auto lanes, auto threads, auto nv) {
        constexpr int V = decltype(v)::value, L = decltype(lanes)::value, TH = decltype(threads)::value, NV = decltype(nv)::value;
        if constexpr (V > 1) {
            const Groups g = groups_of(s, V);
            const dim3 blocks = grid_of((((long long)g.count + L - 1) / L + 7) / 8 * 8);
            if (scale) forward_columns<T, V, L, TH, NV, true><<<blocks, TH, 0, st>>>(x, r, w, h, y, scale, s, g);
            else forward_columns<T, V, L, TH, NV, false><<<blocks, TH, 0, st>>>(x, r, w, h, y, scale, s, g);
        }
        return hipGetLastError();           // single pixels are rows
    });
}

size_t backward_workspace(const Shape& s, int es)
{
    const Grid g = es == 4 ? backward_grid<float>(s) : backward_grid<bf16_t>(s);
    return (size_t)g.rows * s.C * sizeof(float);
}

template <typename T, typename D>
hipError_t launch_backward(const T* x, const T* r, const T* w, const T* dy, const T* dh, T* dx, D* dw, float* part, const Shape& s, hipStream_t st)
{
    const Grid g = backward_grid<T>(s);
    hipError_t e;
    if (s.HW == 1 && s.C <= kWide<T> * 1024 * kKept && s.C >= kWide<T>)
        e = with_rows<T>(s, [&](auto v, auto tpt, auto nv) {
            constexpr int V = decltype(v)::value, TPT = decltype(tpt)::value, NV = decltype(nv)::value;
            if constexpr (NV > 0 && V > 1)
                backward_rows<T, V, TPT, NV><<<g.blocks, kRowThreads<TPT>, 0, st>>>(x, r, w, dy, dh, dx, part, s);
            return hipGetLastError();
        });
    else
        e = with_columns<T>(s, [&](auto v, auto lanes, auto threads, auto nv) {
            constexpr int V = decltype(v)::value, L = decltype(lanes)::value, TH = decltype(threads)::value, NV = decltype(nv)::value;
            backward_columns<T, V, L, TH, NV><<<g.blocks, TH, 0, st>>>(x, r, w, dy, dh, dx, part, s, groups_of(s, V));
            return hipGetLastError();
        });
    if (e != hipSuccess) return e;
    weight_sums<D><<<(s.C + 63) / 64, 1024, 0, st>>>(part, dw, g.rows, s.C);
    return hipGetLastError();
}

#define INSTANCE(T)                                                                                                                        \
    template hipError_t launch_forward<T>(const T*, const T*, const T*, T*, void*, float*, const Shape&, hipStream_t);                     \
    template hipError_t launch_backward<T, float>(const T*, const T*, const T*, const T*, const T*, T*, float*, float*, const Shape&, hipStream_t);
INSTANCE(float)
INSTANCE(bf16_t)
template hipError_t launch_backward<bf16_t, bf16_t>(const bf16_t*, const bf16_t*, const bf16_t*, const bf16_t*, const bf16_t*, bf16_t*, bf16_t*, float*, const Shape&, hipStream_t);

}  // namespace norm
}  // namespace scc
