// C ABI of the gated layer: argument checks, kernel selection, the workspace's parts.
#include "scc_entry.h"
#include "scc_gated.h"

#include <limits>

using namespace scc;
using namespace scc::gated;

namespace {

bool act_ok(scc_activation act) { return act == SCC_SILU || act == SCC_GELU; }

int act_of(scc_activation act) { return act == SCC_SILU ? kSilu : kGelu; }

// SCC_GATED_*, and for the product what its launch does
int forward_path(const Problem& p, int es, Plan* plan, Shape* shape)
{
    if (few_preferred(p)) return SCC_GATED_FEW;
    *plan = make_plan(p, es, false);
    return make_shape(p, *plan, es, p.NQ, shape) ? SCC_GATED_PRODUCT : SCC_GATED_ANY;
}

// The parts of the gradient's workspace.  dh, the gradient of both projections, is the output gradient of one sliding-channel layer
// of 2 * padded filters (the second half starts on the first window again), whose gradients scc_backward takes.  Rows of single
// tokens (HW == 1) are turned into planes of one sample for it, its kernels' layout, and dx turned back.
struct Parts {
    Plan plan;
    Shape shape;
    bool product;       // the two projections run on the matrix cores
    int padded;
    bool tokens, spread, gathered;
    int N, HW;          // of the wide layer
    size_t packed, dh, wide_w, wide_dw, planes, dplanes, rest, rest_bytes, bytes;
};

int make_parts(const Problem& p, int cg, double co, scc_dtype dtype, scc_dtype grad, Parts* out)
{
    Parts t;
    const size_t es = size_of(dtype);
    const long long padded = padded_filters(p), most = std::numeric_limits<int>::max();
    t.tokens = p.HW == 1;
    const long long HW = t.tokens ? (p.NQ + 7) / 8 * 8 : p.HW;
    if (2 * padded * HW > most || 2 * padded * p.L > most || HW * p.Cin > most) return SCC_ERR_SHAPE;
    t.padded = (int)padded;
    t.N = t.tokens ? 1 : p.N;
    t.HW = (int)HW;
    t.plan = make_plan(p, (int)es, true);
    t.product = make_shape(p, t.plan, (int)es, t.tokens ? HW : p.NQ, &t.shape);
    t.spread = padded != p.Cout;
    t.gathered = t.spread || grad == SCC_BF16;
    size_t at = 0;
    auto part = [&](bool used, size_t bytes) {
        const size_t here = at;
        at += used ? align256(bytes) : 0;
        return here;
    };
    const size_t columns = (size_t)t.N * t.HW;
    t.packed = part(t.product, t.plan.bytes);
    t.dh = part(true, columns * 2 * padded * es);
    t.wide_w = part(t.spread, (size_t)2 * padded * p.L * es);
    t.wide_dw = part(t.gathered, (size_t)2 * padded * p.L * 4);
    t.planes = part(t.tokens, columns * p.Cin * es);
    t.dplanes = part(t.tokens, columns * p.Cin * es);
    t.rest_bytes = scc_backward_workspace_bytes(t.N, p.Cin, 2 * t.padded, t.HW, 1, cg, co, dtype);
    t.rest = part(true, t.rest_bytes);
    t.bytes = at;
    *out = t;
    return SCC_OK;
}

// bfloat16 layers of fewer columns are widened, and their gradients are those of binary32: dg and du are then not rounded between the
// stages.  Rounded, they leave 2^-9 of every product in dw, and with few columns that shows where products cancel.  Such a
// call's time is its launches' (two more), not its bytes'.
constexpr int kWidened = 64;

bool widened(const Problem& p, scc_dtype dtype) { return dtype == SCC_BF16 && p.NQ < kWidened; }

// The widened call's workspace: x, w, dy and dx in binary32, then what the binary32 call takes.
struct Wide {
    size_t w, dy, dx, rest, rest_bytes, bytes;
};

Wide wide_of(const Problem& p, size_t rest_bytes)
{
    Wide t;
    t.w = align256((size_t)p.NQ * p.Cin * 4);
    t.dy = t.w + align256((size_t)2 * p.Cout * p.L * 4);
    t.dx = t.dy + align256((size_t)p.NQ * p.Cout * 4);
    t.rest = t.dx + t.w;
    t.rest_bytes = rest_bytes;
    t.bytes = t.rest + rest_bytes;
    return t;
}

}  // namespace

extern "C" {

size_t scc_gated_forward_workspace_bytes(int N, int Cin, int Cout, int H, int W, int cg, double co, scc_dtype dtype)
{
    Problem p;
    if (make_problem(N, Cin, Cout, H, W, cg, co, &p) != SCC_OK || !dtype_ok(dtype)) return 0;
    Plan plan;
    Shape shape;
    return forward_path(p, size_of(dtype), &plan, &shape) == SCC_GATED_PRODUCT ? plan.bytes : 0;
}

int scc_gated_forward_path(int N, int Cin, int Cout, int H, int W, int cg, double co, scc_dtype dtype)
{
    Problem p;
    const int rc = make_problem(N, Cin, Cout, H, W, cg, co, &p);
    if (rc != SCC_OK) return rc;
    if (!dtype_ok(dtype)) return SCC_ERR_DTYPE;
    Plan plan;
    Shape shape;
    return forward_path(p, size_of(dtype), &plan, &shape);
}

int scc_gated_forward(const void* x, const void* w, void* y, int N, int Cin, int Cout, int H, int W, int cg, double co,
                      scc_activation act, scc_dtype dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!x || !w || !y) return SCC_ERR_NULL;
    Problem p;
    const int rc = make_problem(N, Cin, Cout, H, W, cg, co, &p);
    if (rc != SCC_OK) return rc;
    if (!dtype_ok(dtype)) return SCC_ERR_DTYPE;
    if (!act_ok(act)) return SCC_ERR_OPTION;
    if (2ll * p.Cout * p.L > std::numeric_limits<int>::max()) return SCC_ERR_SHAPE;
    Plan plan;
    Shape shape;
    const int path = forward_path(p, size_of(dtype), &plan, &shape);
    if (path == SCC_GATED_PRODUCT && !holds(plan.bytes, workspace, workspace_bytes)) return SCC_ERR_WORKSPACE;
    drop_stale_error();
    const hipStream_t st = (hipStream_t)stream;
    return with_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        const T *tx = (const T*)x, *tw = (const T*)w;
        if (path == SCC_GATED_FEW) return launch_status(launch_few(tx, tw, (T*)y, p, act_of(act), st));
        if (path == SCC_GATED_ANY) return launch_status(launch_any(tx, tw, (const T*)nullptr, (T*)y, GradOut{0, 0, 0, 0}, p, act_of(act), st));
        const int e = launch_status(launch_pack(tw, (char*)workspace, p, plan, st));
        return e != SCC_OK ? e : launch_status(launch_product(tx, (const char*)workspace, (T*)y, p, plan, shape, act_of(act), st));
    });
}

size_t scc_gated_backward_workspace_bytes(int N, int Cin, int Cout, int H, int W, int cg, double co, scc_dtype dtype, scc_dtype grad)
{
    Problem p;
    Parts t;
    if (make_problem(N, Cin, Cout, H, W, cg, co, &p) != SCC_OK || !dtype_ok(dtype) || !dtype_ok(grad)) return 0;
    if (make_parts(p, cg, co, widened(p, dtype) ? SCC_F32 : dtype, grad, &t) != SCC_OK) return 0;
    return widened(p, dtype) ? wide_of(p, t.bytes).bytes : t.bytes;
}

int scc_gated_backward(const void* x, const void* w, const void* dy, void* dx, void* dw, int N, int Cin, int Cout, int H, int W, int cg,
                       double co, scc_activation act, scc_dtype dtype, scc_dtype grad, void* workspace, size_t workspace_bytes,
                       void* stream)
{
    if (!x || !w || !dy || !dx || !dw) return SCC_ERR_NULL;
    Problem p;
    int rc = make_problem(N, Cin, Cout, H, W, cg, co, &p);
    if (rc != SCC_OK) return rc;
    if (!dtype_ok(dtype) || !dtype_ok(grad)) return SCC_ERR_DTYPE;
    if (!act_ok(act)) return SCC_ERR_OPTION;
    Parts t;
    rc = make_parts(p, cg, co, widened(p, dtype) ? SCC_F32 : dtype, grad, &t);
    if (rc != SCC_OK) return rc;
    const hipStream_t st = (hipStream_t)stream;
    char* const ws = (char*)workspace;
    if (widened(p, dtype)) {
        const Wide v = wide_of(p, t.bytes);
        if (!holds(v.bytes, workspace, workspace_bytes)) return SCC_ERR_WORKSPACE;
        drop_stale_error();
        const bf16_t* const from[3] = {(const bf16_t*)x, (const bf16_t*)w, (const bf16_t*)dy};
        float* const to[3] = {(float*)ws, (float*)(ws + v.w), (float*)(ws + v.dy)};
        const int counts[3] = {(int)p.NQ * p.Cin, 2 * p.Cout * p.L, (int)p.NQ * p.Cout};
        const int r = launch_status(launch_widen(from, to, counts, st));
        if (r != SCC_OK) return r;
        rc = scc_gated_backward(to[0], to[1], to[2], ws + v.dx, dw, N, Cin, Cout, H, W, cg, co, act, SCC_F32, grad, ws + v.rest,
                                v.rest_bytes, stream);
        return rc != SCC_OK ? rc : launch_status(launch_narrow((const float*)(ws + v.dx), (bf16_t*)dx, counts[0], st));
    }
    if (!holds(t.bytes, workspace, workspace_bytes)) return SCC_ERR_WORKSPACE;
    drop_stale_error();
    return with_type(dtype, [&](auto v) {
        typedef decltype(v) T;
        const T *tx = (const T*)x, *tw = (const T*)w, *ty = (const T*)dy;
        const long long plane = t.HW;
        const GradOut o = {t.tokens ? 1 : 2ll * t.padded * plane, plane, t.padded, t.tokens ? plane : p.NQ};
        hipError_t e = hipSuccess;
        if (t.product) {
            e = launch_pack(tw, ws + t.packed, p, t.plan, st);
            if (e == hipSuccess)
                e = launch_product_grad(tx, ws + t.packed, ty, (T*)(ws + t.dh), o, p, t.plan, t.shape, act_of(act), st);
        } else {
            e = launch_any(tx, tw, ty, (T*)(ws + t.dh), o, p, act_of(act), st);
        }
        const void *wide_w = w, *wide_x = x;
        if (e == hipSuccess && t.spread) {
            wide_w = ws + t.wide_w;
            e = launch_spread(tw, (T*)(ws + t.wide_w), p, t.padded, st);
        }
        if (e == hipSuccess && t.tokens) {
            wide_x = ws + t.planes;
            e = launch_transpose(tx, (T*)(ws + t.planes), p.NQ, p.Cin, p.Cin, plane, plane, st);
        }
        if (e != hipSuccess) return (int)SCC_ERR_LAUNCH;
        void* const wide_dx = t.tokens ? (void*)(ws + t.dplanes) : dx;
        void* const wide_dw = t.gathered ? (void*)(ws + t.wide_dw) : dw;
        const int r = scc_backward(wide_x, ws + t.dh, wide_w, wide_dx, wide_dw, t.N, Cin, 2 * t.padded, t.HW, 1, cg, co, dtype,
                                   ws + t.rest, t.rest_bytes, stream);
        if (r != SCC_OK) return r;
        if (t.tokens) e = launch_transpose((const T*)(ws + t.dplanes), (T*)dx, p.Cin, (int)p.NQ, plane, p.Cin, p.Cin, st);
        if (e == hipSuccess && t.gathered)
            e = grad == SCC_F32 ? launch_gather((const float*)(ws + t.wide_dw), (float*)dw, p, t.padded, st)
                                : launch_gather((const float*)(ws + t.wide_dw), (bf16_t*)dw, p, t.padded, st);
        return launch_status(e);
    });
}

}  // extern "C"
