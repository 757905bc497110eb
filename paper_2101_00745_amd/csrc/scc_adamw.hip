// AdamW on lists of weights.  Bound by memory: every element of w, g, m and v is read once and of w, m and v written once, in one
// launch for 60 weights (states in 8 bits: 65.5 million fp32 elements, 1.05 GB, 190 us, 5.5 TB/s; 19.5 million bf16 ones, 195 MB, 43 us, 4.5 TB/s, where the rounding's vector
// instructions take nearly as long).  A workgroup has 2048 consecutive elements of one weight, a lane 4 or 8 consecutive ones.
//
// States in 8 bits.  A block of 256 elements shares a power of two that brings its largest |m| (largest root of v) into [128, 256), so that from step to
// step the representable values of a block stay where they are while its scale moves.  e4m3 has values 1/16 apart or closer, and v
// moves by a thousandth of itself a step: rounded to nearest it would never move.  So both states go up or down at random with the
// probability that makes their expectation exact; for v, whose root is stored, between the squares of the two neighbouring roots.  A
// positive v does not become 0, which would leave a momentum over a denominator of eps alone.
#include "scc_adamw.h"

namespace scc {
namespace adamw {
namespace {

template <typename T, int E> struct Lanes { typedef T type __attribute__((ext_vector_type(E))); };

template <typename T, int E>
__device__ __forceinline__ void read(const T* p, float (&v)[E], bool whole, long long left)
{
    if (whole) {
        const typename Lanes<T, E>::type t = *(const typename Lanes<T, E>::type*)p;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = to_f32((T)t[e]);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = e < left ? to_f32(p[e]) : 0.f;
    }
}

template <typename T, int E>
__device__ __forceinline__ void write(T* p, const float (&v)[E], bool whole, long long left)
{
    if (whole) {
        typename Lanes<T, E>::type t;
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = from_f32<T>(v[e]);
        *(typename Lanes<T, E>::type*)p = t;
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < left) p[e] = from_f32<T>(v[e]);
    }
}

// 8 values of e4m3 from two words
__device__ __forceinline__ void widen(const uint32_t (&q)[2], float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], true);
        v[4 * i] = a[0];
        v[4 * i + 1] = a[1];
        v[4 * i + 2] = b[0];
        v[4 * i + 3] = b[1];
    }
}

__device__ __forceinline__ void read_bytes(const uint8_t* p, float (&v)[8], bool whole, long long left)
{
    typedef uint32_t two __attribute__((ext_vector_type(2)));
    uint32_t q[2] = {0, 0};
    if (whole) {
        const two t = *(const two*)p;
        q[0] = t[0];
        q[1] = t[1];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) q[e / 4] |= (uint32_t)p[e] << 8 * (e % 4);
    }
    widen(q, v);
}

__device__ __forceinline__ void write_bytes(uint8_t* p, const uint32_t (&code)[8], bool whole, long long left)
{
    typedef uint32_t two __attribute__((ext_vector_type(2)));
    if (whole) {
        two t;
#pragma unroll
        for (int i = 0; i < 2; ++i) t[i] = code[4 * i] | code[4 * i + 1] << 8 | code[4 * i + 2] << 16 | code[4 * i + 3] << 24;
        *(two*)p = t;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < left) p[e] = (uint8_t)code[e];
    }
}

__device__ __forceinline__ bool finite(float v) { return fabsf(v) <= 3.4028235e38f; }

// Magnitudes are compared as the bits of their binary32 values: in that order, and what is not finite last.
constexpr uint32_t kInfinity = 0x7f800000u;
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

// largest of 32 lanes' values: the lanes of a block
__device__ __forceinline__ uint32_t over_block(uint32_t v)
{
#pragma unroll
    for (int m = 1; m < 32; m *= 2) v = larger(v, (uint32_t)__shfl_xor((int)v, m));
    return v;
}

// k of a block's scale 2^k from its largest value, `halves`: of v, whose root is stored
__device__ __forceinline__ int exponent_of(uint32_t bits, bool halves)
{
    const float most = __uint_as_float(bits);
    int e = __builtin_amdgcn_frexp_expf(most) - 1;
    e = (halves ? e >> 1 : e) - 7;
    return most > 0.f ? (e < -100 ? -100 : e > 120 ? 120 : e) : -100;
}

__device__ __forceinline__ float power(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// |m| / scale < 256 as e4m3, up with the probability that the bits behind the third say.  Below 2^-6, where steps are of 2^-9, those bits are brought to
// the same place.  No branches, here and below: lanes differ in which side they take.
__device__ __forceinline__ uint32_t round_first(float m, float inverse, uint32_t random)
{
    const float a = fabsf(m) * inverse;
    const uint32_t below = (uint32_t)(a * 536870912.f), above = __float_as_uint(a) - (960u << 20);
    const uint32_t code = ((a < 0.015625f ? below : above) + ((random & 0xffffu) << 4 | 8u)) >> 20;
    return code | (__float_as_uint(m) >> 24 & 0x80u);
}

// The root of v / scale^2 as e4m3: v lies between the squares of the neighbours low and high, and goes up with the probability that makes its expectation v.
// Squares and differences are exact, and so is the comparison; the root itself may be rounded onto a neighbour, which moves that border by 2^-23 of it.
// Below 2^-6 a bias of 2^-6 gives all steps the same size.
__device__ __forceinline__ uint32_t round_second(float v, float root, float inverse, uint32_t random)
{
    const float q = (v * inverse) * inverse, at = root * inverse;
    const bool below = at < 0.015625f;
    const float bias = below ? 0.015625f : 0.f;
    const uint32_t bits = __float_as_uint(at + bias) & 0xfff00000u;
    const float low = __uint_as_float(bits) - bias, high = __uint_as_float(bits + 0x100000u) - bias;
    const float square = low * low, u = (float)(random >> 8) * 5.9604644775390625e-8f;
    const float over = fmaf(-u, fmaf(high, high, -square), q - square);
    const uint32_t code = (bits >> 20) - (below ? 968u : 960u);
    return code + ((over > 0.f) | ((code == 0u) & (v > 0.f)) ? 1u : 0u);
}

template <typename T, bool BYTES>
__global__ __launch_bounds__(256) void step_kernel(Batch b, Step s)
{
#pragma clang fp contract(off)
    constexpr int E = BYTES || sizeof(T) == 2 ? 8 : 4;
    int i = 0;
    for (int step = 32; step; step >>= 1)
        if (i + step < b.count && b.first[i + step] <= blockIdx.x) i += step;
    const Weight t = b.weight[i];
    uint32_t key = s.key;
    float c1 = s.c1, c2 = s.c2;
    if (s.at) {
        __shared__ float corrections[2];
        const long long at = *s.at;
        if (threadIdx.x == 0) {
            corrections[0] = (float)(1.0 / -expm1((double)at * s.log_b1));
            corrections[1] = (float)sqrt(1.0 / -expm1((double)at * s.log_b2));
        }
        __syncthreads();
        c1 = corrections[0];
        c2 = corrections[1];
        key = step_key(s.seed, at);
    }
    const float rate = s.lr * c1;
    key = mix(key + (b.index + (uint32_t)i) * 0x9E3779B1u);
    const uintptr_t places = (uintptr_t)t.w | (uintptr_t)t.g | (BYTES ? ((uintptr_t)t.m | (uintptr_t)t.v) << 1 : (uintptr_t)t.m | (uintptr_t)t.v);
    const bool aligned = (places & 15u) == 0;
    const long long begin = (long long)(blockIdx.x - b.first[i]) * kChunk;
#pragma unroll
    for (int round = 0; round < kChunk / (256 * E); ++round) {
        const long long at = begin + (round * 256 + (int)threadIdx.x) * E, left = t.n - at;
        const bool whole = aligned && left >= E;
        float w[E], g[E], m[E], v[E], root[E];
        float ms = 0.f, vs = 0.f;
        // lanes behind the end read nothing; they take part in their block's largest value as zeros
        const long long from = left > 0 ? at : 0;
        read<T, E>((const T*)t.w + from, w, whole, left);
        read<T, E>((const T*)t.g + from, g, whole, left);
        if constexpr (BYTES) {
            read_bytes((const uint8_t*)t.m + from, m, whole, left);
            read_bytes((const uint8_t*)t.v + from, v, whole, left);
            if (left > 0) {
                ms = t.ms[at / kBlock];
                vs = t.vs[at / kBlock];
            }
        } else {
            read<float, E>((const float*)t.m + from, m, whole, left);
            read<float, E>((const float*)t.v + from, v, whole, left);
        }
        // of a state in 8 bits the scale, a power of two, goes into the factor that follows: the same bits
        const float from_m = BYTES ? ms * s.b1 : s.b1;
        bool small = false;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (BYTES) {
                v[e] *= vs;
                v[e] *= v[e];
            }
            m[e] = m[e] * from_m + g[e] * s.d1;
            v[e] = v[e] * s.b2 + (g[e] * g[e]) * s.d2;
            root[e] = __builtin_amdgcn_sqrtf(v[e]);
            small |= __float_as_uint(v[e]) - 1u < 0x7fffffu;
        }
        if (__any(small)) {
            asm volatile("");                   // a branch: rare
            // the instruction takes what is below 2^-126 for 0; the root of it is no less than 2^-75
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (__float_as_uint(v[e]) - 1u < 0x7fffffu) root[e] = __builtin_amdgcn_sqrtf(v[e] * 18446744073709551616.f) * 2.3283064365386963e-10f;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = fmaf(w[e], s.keep, -(m[e] * rate) * __builtin_amdgcn_rcpf(fmaf(root[e], c2, s.eps)));
        write<T, E>((T*)t.w + from, w, whole, left);
        if constexpr (BYTES) {
            uint32_t most_m = 0, most_v = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                most_m = larger(most_m, __float_as_uint(m[e]) & 0x7fffffffu);
                most_v = larger(most_v, __float_as_uint(v[e]));
            }
            const bool strange = __any(larger(most_m, most_v) >= kInfinity);
            if (strange) {
                asm volatile("");                   // a branch: rare
                most_m = most_v = 0;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    most_m = larger(most_m, finite(m[e]) ? __float_as_uint(m[e]) & 0x7fffffffu : 0u);
                    most_v = larger(most_v, finite(v[e]) ? __float_as_uint(v[e]) : 0u);
                }
            }
            const int km = exponent_of(over_block(most_m), false), kv = exponent_of(over_block(most_v), true);
            uint32_t qm[E], qv[E];
            const float im = power(-km), iv = power(-kv);
            const uint32_t place = (uint32_t)at + (uint32_t)((uint64_t)at >> 32) * 0x85157AF5u + key;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const uint32_t random = mix(place + (uint32_t)e);
                qm[e] = round_first(m[e], im, random);
                qv[e] = round_second(v[e], root[e], iv, random);
            }
            if (strange) {
                asm volatile("");
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    qm[e] = finite(m[e]) ? qm[e] : 0x7fu;
                    qv[e] = finite(v[e]) ? qv[e] : 0x7fu;
                }
            }
            write_bytes((uint8_t*)t.m + from, qm, whole, left);
            write_bytes((uint8_t*)t.v + from, qv, whole, left);
            if (left > 0 && threadIdx.x % 32 == 0) {
                t.ms[at / kBlock] = power(km);
                t.vs[at / kBlock] = power(kv);
            }
        } else {
            write<float, E>((float*)t.m + from, m, whole, left);
            write<float, E>((float*)t.v + from, v, whole, left);
        }
    }
}

}  // namespace

template <typename T>
hipError_t launch_step(const Batch& batch, const Step& step, uint32_t chunks, bool bytes, hipStream_t st)
{
    if (bytes) step_kernel<T, true><<<chunks, 256, 0, st>>>(batch, step);
    else step_kernel<T, false><<<chunks, 256, 0, st>>>(batch, step);
    return hipGetLastError();
}

template hipError_t launch_step<float>(const Batch&, const Step&, uint32_t, bool, hipStream_t);
template hipError_t launch_step<bf16_t>(const Batch&, const Step&, uint32_t, bool, hipStream_t);

}  // namespace adamw
}  // namespace scc
