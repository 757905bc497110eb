// C ABI of the residual norm: argument checks.
#include "scc_entry.h"
#include "scc_norm.h"

#include <cmath>

using namespace scc;

namespace {

int check(const void* x, const void* w, int N, int C, int H, int W, float eps, scc_dtype dtype, norm::Shape* s)
{
    if (!x || !w) return SCC_ERR_NULL;
    if (N < 1 || C < 1 || C > 1 << 26 || H < 1 || W < 1 || (long long)H * W > 0x7fffffff || (long long)N * H * W > 0x7fffffff) return SCC_ERR_SHAPE;
    if (!dtype_ok(dtype)) return SCC_ERR_DTYPE;
    if (!(eps > 0.f) || !std::isfinite(eps)) return SCC_ERR_OPTION;
    *s = {N, C, H * W, eps};
    return SCC_OK;
}

int forward(const void* x, const void* residual, const void* w, void* h, void* y, float* scale, int N, int C, int H, int W, float eps,
            scc_dtype dtype, void* stream)
{
    norm::Shape s;
    const int rc = check(x, w, N, C, H, W, eps, dtype, &s);
    if (rc != SCC_OK) return rc;
    if (!y || (h && !residual)) return SCC_ERR_NULL;
    drop_stale_error();
    return with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return launch_status(norm::launch_forward<T>((const T*)x, (const T*)residual, (const T*)w, (T*)h, y, scale, s, (hipStream_t)stream));
    });
}

}  // namespace

extern "C" {

int scc_norm_forward(const void* x, const void* residual, const void* w, void* h, void* y, int N, int C, int H, int W, float eps,
                     scc_dtype dtype, void* stream)
{
    return forward(x, residual, w, h, y, nullptr, N, C, H, W, eps, dtype, stream);
}

int scc_norm_quantised(const void* x, const void* residual, const void* w, void* h, uint8_t* q, float* scale, int N, int C, int H, int W,
                       float eps, scc_dtype dtype, void* stream)
{
    if (!scale) return SCC_ERR_NULL;
    return forward(x, residual, w, h, q, scale, N, C, H, W, eps, dtype, stream);
}

size_t scc_norm_backward_workspace_bytes(int N, int C, int H, int W, scc_dtype dtype)
{
    norm::Shape s;
    static const int something = 0;
    return check(&something, &something, N, C, H, W, 1.f, dtype, &s) == SCC_OK ? align256(norm::backward_workspace(s, size_of(dtype))) : 0;
}

int scc_norm_backward(const void* x, const void* residual, const void* w, const void* dy, const void* dh, void* dx, void* dw, int N, int C, int H, int W,
                      float eps, scc_dtype dtype, scc_dtype grad, void* workspace, size_t workspace_bytes, void* stream)
{
    norm::Shape s;
    const int rc = check(x, w, N, C, H, W, eps, dtype, &s);
    if (rc != SCC_OK) return rc;
    if (!dy || !dx || !dw) return SCC_ERR_NULL;
    if (!dtype_ok(grad) || (dtype == SCC_F32 && grad != SCC_F32)) return SCC_ERR_DTYPE;
    if (!holds(align256(norm::backward_workspace(s, size_of(dtype))), workspace, workspace_bytes)) return SCC_ERR_WORKSPACE;
    drop_stale_error();
    const hipStream_t st = (hipStream_t)stream;
    float* part = (float*)workspace;
    if (dtype == SCC_F32)
        return launch_status(norm::launch_backward<float, float>((const float*)x, (const float*)residual, (const float*)w, (const float*)dy, (const float*)dh,
                                                                 (float*)dx, (float*)dw, part, s, st));
    if (grad == SCC_F32)
        return launch_status(norm::launch_backward<bf16_t, float>((const bf16_t*)x, (const bf16_t*)residual, (const bf16_t*)w, (const bf16_t*)dy, (const bf16_t*)dh,
                                                                  (bf16_t*)dx, (float*)dw, part, s, st));
    return launch_status(norm::launch_backward<bf16_t, bf16_t>((const bf16_t*)x, (const bf16_t*)residual, (const bf16_t*)w, (const bf16_t*)dy, (const bf16_t*)dh,
                                                               (bf16_t*)dx, (bf16_t*)dw, part, s, st));
}

}  // extern "C"
