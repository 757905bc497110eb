// C ABI of the orthogonalised update: argument checks, and the list in batches whose descriptions fit a launch's arguments.
#include "scc_entry.h"
#include "scc_orthogonal.h"

#include <cmath>
#include <limits>

using namespace scc;
using namespace scc::orthogonal;

namespace {

// SCC_OK, or why the list cannot be run
int check_shapes(int count, const int* rows, const int* cols)
{
    if (!rows || !cols) return SCC_ERR_NULL;
    if (count < 1) return SCC_ERR_SHAPE;
    for (int i = 0; i < count; ++i) {
        if (rows[i] < 1 || cols[i] < 1) return SCC_ERR_SHAPE;
        // a batch's workgroups are counted in 32 bits
        if ((long long)rows[i] * cols[i] > std::numeric_limits<int>::max() / kBatch) return SCC_ERR_SHAPE;
    }
    return SCC_OK;
}

void tiles_of(int rows, int cols, int* s, int* l)
{
    const int a = (rows + kTile - 1) / kTile, b = (cols + kTile - 1) / kTile;
    *s = a < b ? a : b;
    *l = a < b ? b : a;
}

Layout list_layout(int count, const int* rows, const int* cols)
{
    size_t half = 0, tiles = 0;
    for (int i = 0; i < count; ++i) {
        int s, l;
        tiles_of(rows[i], cols[i], &s, &l);
        half += (size_t)s * (s + 1) / 2;
        tiles += (size_t)s * l;
    }
    return layout_of(half, tiles);
}

size_t workspace_of(int count, const int* rows, const int* cols)
{
    size_t most = 0;
    for (int at = 0; at < count; at += kBatch) {        // batches run one after the other in the same workspace
        const int n = count - at < kBatch ? count - at : kBatch;
        size_t now = list_layout(n, rows + at, cols + at).matrices;
        for (int i = at; i < at + n; ++i) {
            int s, l;
            tiles_of(rows[i], cols[i], &s, &l);
            now += parts_of(s, l).bytes;
        }
        most = now > most ? now : most;
    }
    return most;
}

int check_options(const scc_orthogonal_options* o)
{
    if (!o) return SCC_ERR_NULL;
    if (o->steps < 1 || o->steps > 100) return SCC_ERR_OPTION;
    const float all[] = {o->lr, o->momentum, o->weight_decay, o->a, o->b, o->c, o->eps};
    for (const float v : all)
        if (!std::isfinite(v)) return SCC_ERR_OPTION;
    return o->eps < 0.f ? SCC_ERR_OPTION : SCC_OK;
}

int run(int count, void* const* w, const void* const* g, float* const* m, const int* rows, const int* cols,
        const scc_orthogonal_options* options, scc_dtype dtype, bool update, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!w || !g || (update && !m)) return SCC_ERR_NULL;
    int rc = check_shapes(count, rows, cols);
    if (rc != SCC_OK) return rc;
    for (int i = 0; i < count; ++i)
        if (!w[i] || !g[i] || (update && !m[i])) return SCC_ERR_NULL;
    if (!dtype_ok(dtype)) return SCC_ERR_DTYPE;
    rc = check_options(options);
    if (rc != SCC_OK) return rc;
    if (!holds(workspace_of(count, rows, cols), workspace, workspace_bytes)) return SCC_ERR_WORKSPACE;
    const Options o = {options->lr, options->momentum, options->weight_decay, options->a, options->b, options->c, options->eps,
                       options->nesterov, options->steps};
    drop_stale_error();
    for (int at = 0; at < count; at += kBatch) {
        Batch b;
        b.count = count - at < kBatch ? count - at : kBatch;
        size_t bytes = list_layout(b.count, rows + at, cols + at).matrices;
        for (int i = 0; i < b.count; ++i) {
            Matrix& t = b.mat[i];
            t = {g[at + i], update ? m[at + i] : nullptr, w[at + i], rows[at + i], cols[at + i], 0, 0, bytes};
            tiles_of(t.rows, t.cols, &t.s, &t.l);
            bytes += parts_of(t.s, t.l).bytes;
        }
        rc = with_type(dtype, [&](auto t) {
            return launch_status(launch_orthogonal<decltype(t)>(b, o, update, (char*)workspace, (hipStream_t)stream));
        });
        if (rc != SCC_OK) return rc;
    }
    return SCC_OK;
}

}  // namespace

extern "C" {

size_t scc_orthogonal_workspace_bytes(int count, const int* rows, const int* cols)
{
    return check_shapes(count, rows, cols) == SCC_OK ? workspace_of(count, rows, cols) : 0;
}

int scc_orthogonalise(int count, const void* const* g, void* const* o, const int* rows, const int* cols,
                      const scc_orthogonal_options* options, scc_dtype dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    return run(count, o, g, nullptr, rows, cols, options, dtype, false, workspace, workspace_bytes, stream);
}

int scc_orthogonal_step(int count, void* const* w, const void* const* g, float* const* m, const int* rows, const int* cols,
                        const scc_orthogonal_options* options, scc_dtype dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    return run(count, w, g, m, rows, cols, options, dtype, true, workspace, workspace_bytes, stream);
}

}  // extern "C"
