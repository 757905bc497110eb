// Cross entropy over a vocabulary: declarations shared by its kernels and entry points.
//
//   l_tv = sum_c x_tc w_vc,   lse_t = log sum_v exp(l_tv),   loss_t = lse_t - l_{t,y_t}
//   dx_tc = d_t sum_v p_tv w_vc,   dw_vc = sum_t d_t p_tv x_tc,   p_tv = exp(l_tv - lse_t) - [v = y_t],   d_t the gradient of loss_t
// Tokens whose target is the ignored one have loss 0 and no part in anything else: the others are packed, one after the other.
#pragma once
#include "scc_common.h"

namespace scc {
namespace vocabulary {

struct Shape {
    int N, C, HW, V;
    long long T() const { return (long long)N * HW; }
};

constexpr int kPad = 256;           // packed tokens end at a multiple of this
inline __host__ __device__ long long padded(long long v) { return (v + kPad - 1) / kPad * kPad; }

// A workspace that is handed out piece by piece; with a null base it only counts.
struct Room {
    char* base;
    size_t used = 0;
    template <typename P> P* take(size_t count)
    {
        const size_t at = used;
        used += (count * sizeof(P) + 255) / 256 * 256;
        return (P*)(base + at);
    }
};

// Which tokens count, and what is kept of them in both passes (arrays of the packed tokens, padded)
struct Tokens {
    int *order, *place;             // of a packed token in x; of a token of x among the packed ones, -1: ignored
    int* count;                     // one value
    long long* target;
    float *known, *lse;             // the target's logit (of the loss); log-sum-exp
};

template <typename T>
hipError_t launch_loss(const T* x, const T* w, const long long* target, long long ignored, int reduction, float* loss, float* lse, const Shape& s,
                       char* workspace, hipStream_t st);
size_t loss_workspace(const Shape& s, int es, bool aligned, int reduction);

template <typename T>
hipError_t launch_gradients(const T* x, const T* w, const long long* target, long long ignored, int reduction, const float* lse, const float* dloss,
                            T* dx, void* dw, bool wide, const Shape& s, char* workspace, hipStream_t st);
size_t gradients_workspace(const Shape& s, int es);

}  // namespace vocabulary
}  // namespace scc
