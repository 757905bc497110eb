// AdamW on lists of weights, states in 32 bits or in 8: declarations shared by its kernel and entry point.
//
//   m <- b1 m + (1 - b1) g;   v <- b2 v + (1 - b2) g^2;   w <- (1 - lr wd) w - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// States in 8 bits: blocks of 256 elements with a power of two each, m = e4m3 * 2^k, v = (e4m3 * 2^k)^2.
#pragma once
#include "scc_common.h"

namespace scc {
namespace adamw {

constexpr int kBatch = 60;          // weights of one launch: their descriptions are kernel arguments (4 KB at most)
constexpr int kBlock = 256;         // elements of a scale
constexpr int kChunk = 2048;        // elements of a workgroup
constexpr long long kMostChunks = 1 << 23;      // of a launch, whose lanes are counted in 32 bits

struct Weight {
    void* w;
    const void* g;
    void *m, *v;
    float *ms, *vs;
    long long n;
};

struct Batch {
    Weight weight[kBatch];
    uint32_t first[kBatch];         // chunk with which each begins
    int count;
    uint32_t index;                 // of the first weight in the caller's list
};

struct Step {
    const long long* at;            // the step's number in device memory; null: c1, c2 and key are of the step
    double log_b1, log_b2;
    uint64_t seed;
    float b1, b2, d1, d2;           // d = 1 - b
    float keep, lr, eps;            // keep = 1 - lr wd
    float c1, c2;                   // 1 / (1 - b1^t), the root of 1 / (1 - b2^t)
    uint32_t key;                   // of the step's random numbers
};

// A permutation of the 32-bit numbers in which every bit of the result depends on all of x (two rounds of multiplying and folding the upper half onto
// the lower one; the multipliers are the leading bits of the roots of 2 and 3).
inline __host__ __device__ uint32_t mix(uint32_t x)
{
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}

inline __host__ __device__ uint32_t step_key(uint64_t seed, long long step)
{
    return mix((uint32_t)seed + (uint32_t)(seed >> 32) * 0x85157AF5u + (uint32_t)step * 0x9E3779B1u);
}

template <typename T>
hipError_t launch_step(const Batch& batch, const Step& step, uint32_t chunks, bool bytes, hipStream_t st);

}  // namespace adamw
}  // namespace scc
