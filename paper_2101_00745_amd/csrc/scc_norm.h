// Root-mean-square norm over the channels with the residual's addition in front: declarations shared by its kernels and entry points.
//
//   h = x + r,   s = (mean_c h^2 + eps)^(-1/2),   y = h s w
// and, from dy and dh, with a = dy w:   dx = dr = dh + s (a - h s mean_c(a h s)),   dw = sum over tokens of dy h s
#pragma once
#include "scc_common.h"

namespace scc {
namespace norm {

struct Shape {
    int N, C, HW;
    float eps;
};

// y in the type of x, or (q, scale) in 8 bits: q then has y's place and scale is not null.  r and h: both null or both not, or h null where the
// sum is not wanted.
template <typename T>
hipError_t launch_forward(const T* x, const T* r, const T* w, T* h, void* y, float* scale, const Shape& s, hipStream_t st);

// Sums of dw over the tokens of a workgroup, one row of C for each, in the workspace.
size_t backward_workspace(const Shape& s, int es);

// h = x + r; r and dh may be null; dw: of the type D (float or T).
template <typename T, typename D>
hipError_t launch_backward(const T* x, const T* r, const T* w, const T* dy, const T* dh, T* dx, D* dw, float* part, const Shape& s, hipStream_t st);

}  // namespace norm
}  // namespace scc
