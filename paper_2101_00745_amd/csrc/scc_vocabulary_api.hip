// C ABI of the vocabulary loss: argument checks.
#include "scc_entry.h"
#include "scc_vocabulary.h"

using namespace scc;

namespace {

int check(int N, int C, int H, int W, int V, scc_dtype dtype, scc_reduction reduction, vocabulary::Shape* s)
{
    if (N < 1 || C < 1 || H < 1 || W < 1 || V < 1) return SCC_ERR_SHAPE;
    const long long HW = (long long)H * W, T = HW * N;
    // tokens are counted in 32 bits, also padded, and so are the tiles of a product, of 2^15 logits or more where there are so many
    if (HW > 0x7fffffff || T > 1 << 26 || C > 1 << 20 || V > 1 << 26 || T * V > 1ll << 45) return SCC_ERR_SHAPE;
    if (!dtype_ok(dtype)) return SCC_ERR_DTYPE;
    if (reduction != SCC_NONE && reduction != SCC_SUM && reduction != SCC_MEAN) return SCC_ERR_OPTION;
    *s = {N, C, (int)HW, V};
    return SCC_OK;
}

}  // namespace

extern "C" {

size_t scc_vocabulary_loss_workspace_bytes(int N, int C, int H, int W, int V, scc_reduction reduction, scc_dtype dtype)
{
    vocabulary::Shape s;
    return check(N, C, H, W, V, dtype, reduction, &s) == SCC_OK ? vocabulary::loss_workspace(s, size_of(dtype), false, reduction) : 0;
}

int scc_vocabulary_loss(const void* x, const void* w, const long long* target, float* loss, float* lse, int N, int C, int H, int W, int V,
                        long long ignored, scc_reduction reduction, scc_dtype dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!x || !w || !target || !loss || !lse) return SCC_ERR_NULL;
    vocabulary::Shape s;
    const int rc = check(N, C, H, W, V, dtype, reduction, &s);
    if (rc != SCC_OK) return rc;
    if (!holds(vocabulary::loss_workspace(s, size_of(dtype), ((uintptr_t)w & 15u) == 0, reduction), workspace, workspace_bytes))
        return SCC_ERR_WORKSPACE;
    drop_stale_error();
    return with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return launch_status(vocabulary::launch_loss<T>((const T*)x, (const T*)w, target, ignored, reduction, loss, lse, s, (char*)workspace,
                                                        (hipStream_t)stream));
    });
}

size_t scc_vocabulary_gradients_workspace_bytes(int N, int C, int H, int W, int V, scc_dtype dtype)
{
    vocabulary::Shape s;
    return check(N, C, H, W, V, dtype, SCC_NONE, &s) == SCC_OK ? vocabulary::gradients_workspace(s, size_of(dtype)) : 0;
}

int scc_vocabulary_gradients(const void* x, const void* w, const long long* target, const float* lse, const float* dloss, void* dx, void* dw,
                             int N, int C, int H, int W, int V, long long ignored, scc_reduction reduction, scc_dtype dtype, scc_dtype grad,
                             void* workspace, size_t workspace_bytes, void* stream)
{
    if (!x || !w || !target || !lse || !dloss || !dx || !dw) return SCC_ERR_NULL;
    vocabulary::Shape s;
    const int rc = check(N, C, H, W, V, dtype, reduction, &s);
    if (rc != SCC_OK) return rc;
    if (!dtype_ok(grad) || (dtype == SCC_F32 && grad != SCC_F32)) return SCC_ERR_DTYPE;
    if (!holds(vocabulary::gradients_workspace(s, size_of(dtype)), workspace, workspace_bytes)) return SCC_ERR_WORKSPACE;
    drop_stale_error();
    return with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return launch_status(vocabulary::launch_gradients<T>((const T*)x, (const T*)w, target, ignored, reduction, lse, dloss, (T*)dx, dw,
                                                             grad == SCC_F32, s, (char*)workspace, (hipStream_t)stream));
    });
}

}  // extern "C"
