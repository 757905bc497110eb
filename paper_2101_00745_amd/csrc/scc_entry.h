// What the entry points of the C ABI share: argument checks, the storage types, the status of a launch.
#pragma once
#include "scc.h"
#include "scc_common.h"

namespace scc {

// Algorithm 1 in closed form (scc_api.hip).  Returns SCC_OK or the status that rejects the arguments.
int make_problem(int N, int Cin, int Cout, int H, int W, int cg, double co, Problem* out);

// scc_backward (scc_api.hip); with `later`, a sum over slices of the batch is left to the caller: *later says of what, dw itself where there is one.
int backward(const void* x, const void* dy, const void* w, void* dx, void* dw, int N, int Cin, int Cout, int H, int W, int cg, double co,
             scc_dtype dtype, void* workspace, size_t workspace_bytes, void* stream, SliceSum* later);

inline bool dtype_ok(scc_dtype d) { return d == SCC_F32 || d == SCC_BF16; }

inline int launch_status(hipError_t e) { return e == hipSuccess ? SCC_OK : SCC_ERR_LAUNCH; }

// The launchers report hipGetLastError(), which also returns (and clears) an error an EARLIER, unrelated call of
// the process left behind.  Every entry point that launches drops such a leftover first, so that SCC_ERR_LAUNCH
// always speaks of this call's own kernels.
inline void drop_stale_error() { (void)hipGetLastError(); }

// f(T()) with T the storage type of `dtype`
template <typename F>
int with_type(scc_dtype dtype, F&& f)
{
    return dtype == SCC_F32 ? f(float()) : f(bf16_t());
}

inline int size_of(scc_dtype dtype) { return dtype == SCC_F32 ? 4 : 2; }

// Whether a call may use `need` bytes of its workspace.
inline bool holds(size_t need, const void* workspace, size_t workspace_bytes)
{
    return need == 0 || (workspace && workspace_bytes >= need && ((uintptr_t)workspace & 255u) == 0);
}

inline size_t align256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace scc
