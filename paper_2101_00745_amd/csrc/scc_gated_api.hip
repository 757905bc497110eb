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
    if (one_preferred(p)) return SCC_GATED_ONE;
    if (direct_preferred(p, es, false)) return SCC_GATED_DIRECT;
    *plan = make_plan(p, es, false);
    return make_shape(p, *plan, es, shape) ? SCC_GATED_PRODUCT : SCC_GATED_ANY;
}

// A gradient as it is computed.  dh, the gradient of both projections, is the output gradient of one sliding-channel layer of 2 * padded filters (the
// second half starts on the first window again), whose gradients the framework's other kernels take.  They want planes of some
// pixels and 64 columns at least: layers of less are turned into planes of one sample, filled up with zeros, and dx turned back.
// bfloat16 layers of fewer columns than that, or of few weights, are widened to binary32 on the way.  dg and du are then not rounded between the
// stages: rounded, they leave 2^-9 of every product in dw, which shows where products cancel, with few columns or where no weight of few has a
// sum much larger than its terms'.  Of 2255 random layers of 64 columns or more the rounding left dw of the 122 with fewer than 16 weights up to 18 times as far
// off as one rounding at the end (0.010 of its norm; inputs were found with 0.1 of the largest value), of the 412 up to 128 weights 4.7 times, of the 1721 with more
// 2.6 times (0.004 of the norm), half of all 1.4 times.  Widened, those of up to 128 weights take 1.1 times as long, 7 us more, in the middle; 3.7 times at most, with
// a hundred thousand columns.
// The others hand dg and du on in bfloat16, as the gradient that one layer hands the next.  A second bfloat16 part of both would make them exact for
// twice the filters in the products behind:
// us of these, without and with it, 64 x 512 -> 512 on 14x14, cg 8 25 and 36 (of a step's 66), 4096 tokens 256 -> 512, cg 2 14 and 27 (68), 65536 of them
// 66 and 122, 64 x 512 -> 1024 on 7x7, cg 2 44 and 109, 8 x 2000 tokens 512 -> 1024 dense 109 and 574.
constexpr int kFewColumns = 64, kFewWeights = 128;

struct Parts {
    Problem p;          // the layer in planes
    scc_dtype type;     // of the kernels
    bool planes, widened, direct, product, spread, gathered;
    Plan plan;
    Shape shape;
    int padded;
    size_t packed, dh, wide_w, wide_dw, x, dy, dx, rest, rest_bytes, bytes;
};

int make_parts(const Problem& p, int cg, double co, scc_dtype dtype, scc_dtype grad, Parts* out)
{
    Parts t;
    const long long padded = padded_filters(p), most = std::numeric_limits<int>::max();
    // one sample of all columns has to fit an index, which the layer's own samples may where it does not
    const bool few = 2ll * p.Cout * p.L <= kFewWeights && 2 * padded * (p.NQ + 7) <= most && p.Cin * (p.NQ + 7) <= most;
    t.widened = dtype == SCC_BF16 && (p.NQ < kFewColumns || few);
    t.planes = p.HW < 4 || p.NQ < kFewColumns || t.widened;
    t.type = t.widened ? SCC_F32 : dtype;
    t.p = p;
    if (t.planes) {
        const long long width = p.NQ < kFewColumns ? kFewColumns : (p.NQ + 7) / 8 * 8;
        if (width > most) return SCC_ERR_SHAPE;
        t.p.N = 1;
        t.p.HW = (int)width;
        t.p.NQ = width;
    }
    if (2 * padded * t.p.HW > most || 2 * padded * p.L > most || (long long)t.p.HW * p.Cin > most) return SCC_ERR_SHAPE;
    t.padded = (int)padded;
    const size_t es = size_of(t.type), columns = (size_t)t.p.NQ;
    t.plan = make_plan(t.p, (int)es, true);
    t.direct = direct_preferred(p, (int)size_of(dtype), true);
    t.product = !t.direct && make_shape(t.p, t.plan, (int)es, &t.shape);
    t.spread = padded != p.Cout || t.widened;
    t.gathered = padded != p.Cout || grad == SCC_BF16;
    size_t at = 0;
    auto part = [&](bool used, size_t bytes) {
        const size_t here = at;
        at += used ? align256(bytes) : 0;
        return here;
    };
    t.packed = part(t.product, t.plan.bytes);
    t.dh = part(true, columns * 2 * padded * es);
    t.wide_w = part(t.spread, (size_t)2 * padded * p.L * es);
    t.wide_dw = part(t.gathered, (size_t)2 * padded * p.L * 4);
    t.x = part(t.planes, columns * p.Cin * es);
    t.dy = part(t.planes && !t.direct, columns * p.Cout * es);
    t.dx = part(t.planes, columns * p.Cin * es);
    t.rest_bytes = scc_backward_workspace_bytes(t.p.N, p.Cin, 2 * t.padded, t.p.HW, 1, cg, co, t.type);
    t.rest = part(true, t.rest_bytes);
    t.bytes = at;
    *out = t;
    return SCC_OK;
}

// From: the tensors' type; T: the kernels'
template <typename From, typename T>
int run_backward(const From* x, const From* w, const From* dy, From* dx, void* dw, const Problem& p, const Parts& t, int cg, double co,
                 int act, scc_dtype grad, char* ws, hipStream_t st)
{
    Prepare before = {};
    before.w = w;
    before.packed = t.product ? ws + t.packed : nullptr;
    before.wide = t.spread ? ws + t.wide_w : nullptr;
    before.padded = t.padded;
    before.width = t.p.HW;
    if (t.planes) before.planes[0] = {x, ws + t.x, p.Cin};
    if (t.planes && !t.direct) before.planes[1] = {dy, ws + t.dy, p.Cout};
    hipError_t e = launch_prepare<From, T>(before, p, t.plan, st);
    if (e != hipSuccess) return SCC_ERR_LAUNCH;
    const T* const px = t.planes ? (const T*)(ws + t.x) : (const T*)x;
    const T* const py = t.planes ? (const T*)(ws + t.dy) : (const T*)dy;
    const T* const pw = t.spread ? (const T*)(ws + t.wide_w) : (const T*)w;
    T* const pdx = t.planes ? (T*)(ws + t.dx) : (T*)dx;
    T* const dh = (T*)(ws + t.dh);
    if (t.direct) {
        e = launch_direct_grad(x, w, dy, dh, t.padded, t.planes ? (long long)t.p.HW : 0ll, p, act, st);
    } else if (t.product) {
        e = launch_product_grad(px, ws + t.packed, py, dh, t.padded, t.p, t.plan, t.shape, act, st);
    } else {
        e = launch_any(px, pw, t.spread ? t.padded : p.Cout, py, dh, t.padded, t.p, act, st);
    }
    if (e != hipSuccess) return SCC_ERR_LAUNCH;
    SliceSum sum;
    float* const wide_dw = t.gathered ? (float*)(ws + t.wide_dw) : (float*)dw;
    const int r = scc::backward(px, dh, pw, pdx, wide_dw, t.p.N, p.Cin, 2 * t.padded, t.p.HW, 1, cg, co, t.type, ws + t.rest, t.rest_bytes,
                                st, &sum);
    if (r != SCC_OK) return r;
    Finish after = {};
    after.width = t.p.HW;
    if (t.planes) after.dx = {pdx, dx, p.Cin};
    after.sum = sum;
    after.dw = t.gathered || sum.slices > 1 ? dw : nullptr;
    after.padded = t.padded;
    return launch_status(grad == SCC_F32 ? launch_finish<T, From, float>(after, p, st) : launch_finish<T, From, bf16_t>(after, p, st));
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
        if (path == SCC_GATED_ONE) return launch_status(launch_one(tx, tw, (T*)y, p, act_of(act), st));
        if (path == SCC_GATED_DIRECT) return launch_status(launch_direct(tx, tw, (T*)y, p, act_of(act), st));
        if (path == SCC_GATED_ANY) return launch_status(launch_any(tx, tw, p.Cout, (const T*)nullptr, (T*)y, 0, p, act_of(act), st));
        Prepare before = {};
        before.w = w;
        before.packed = (char*)workspace;
        const int e = launch_status(launch_prepare<T, T>(before, p, plan, st));
        return e != SCC_OK ? e : launch_status(launch_product(tx, (const char*)workspace, (T*)y, p, plan, shape, act_of(act), st));
    });
}

size_t scc_gated_backward_workspace_bytes(int N, int Cin, int Cout, int H, int W, int cg, double co, scc_dtype dtype, scc_dtype grad)
{
    Problem p;
    Parts t;
    if (make_problem(N, Cin, Cout, H, W, cg, co, &p) != SCC_OK || !dtype_ok(dtype) || !dtype_ok(grad)) return 0;
    return make_parts(p, cg, co, dtype, grad, &t) == SCC_OK ? t.bytes : 0;
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
    rc = make_parts(p, cg, co, dtype, grad, &t);
    if (rc != SCC_OK) return rc;
    if (!holds(t.bytes, workspace, workspace_bytes)) return SCC_ERR_WORKSPACE;
    drop_stale_error();
    const hipStream_t st = (hipStream_t)stream;
    char* const ws = (char*)workspace;
    auto run = [&](auto from, auto to) {
        typedef decltype(from) From;
        return run_backward<From, decltype(to)>((const From*)x, (const From*)w, (const From*)dy, (From*)dx, dw, p, t, cg, co, act_of(act), grad,
                                                ws, st);
    };
    if (t.widened) return run(bf16_t(), float());
    return dtype == SCC_F32 ? run(float(), float()) : run(bf16_t(), bf16_t());
}

}  // extern "C"
