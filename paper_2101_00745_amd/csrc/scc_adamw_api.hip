// C ABI of AdamW over lists: argument checks, and the list in batches whose descriptions fit a launch's arguments.
#include "scc_adamw.h"
#include "scc_entry.h"

#include <cmath>

using namespace scc;
using namespace scc::adamw;

extern "C" int scc_adamw_step(int count, void* const* w, const void* const* g, void* const* first, void* const* second,
                              float* const* first_scales, float* const* second_scales, const long long* sizes,
                              const scc_adamw_options* o, long long step, const long long* device_step, scc_dtype dtype, void* stream)
{
    const bool bytes = first_scales != nullptr;
    if (!w || !g || !first || !second || !sizes || !o || bytes != (second_scales != nullptr)) return SCC_ERR_NULL;
    if (count < 1) return SCC_ERR_SHAPE;
    for (int i = 0; i < count; ++i) {
        if (!w[i] || !g[i] || !first[i] || !second[i] || (bytes && (!first_scales[i] || !second_scales[i]))) return SCC_ERR_NULL;
        if (sizes[i] < 1 || sizes[i] > kMostChunks * kChunk) return SCC_ERR_SHAPE;
    }
    if (!dtype_ok(dtype)) return SCC_ERR_DTYPE;
    for (const double v : {o->lr, o->eps, o->weight_decay})
        if (!std::isfinite(v)) return SCC_ERR_OPTION;
    for (const double b : {o->beta1, o->beta2})
        if (!(b >= 0.0 && b < 1.0)) return SCC_ERR_OPTION;
    if (o->eps < 0.0 || (!device_step && step < 1)) return SCC_ERR_OPTION;
    Step s = {};
    s.at = device_step;
    s.log_b1 = std::log(o->beta1);              // -inf for 0: the correction is 1
    s.log_b2 = std::log(o->beta2);
    s.seed = o->seed;
    s.b1 = (float)o->beta1;
    s.b2 = (float)o->beta2;
    s.d1 = (float)(1.0 - o->beta1);
    s.d2 = (float)(1.0 - o->beta2);
    s.keep = (float)(1.0 - o->lr * o->weight_decay);
    s.lr = (float)o->lr;
    s.eps = (float)o->eps;
    if (!device_step) {
        s.c1 = (float)(1.0 / -std::expm1((double)step * s.log_b1));
        s.c2 = (float)std::sqrt(1.0 / -std::expm1((double)step * s.log_b2));
        s.key = step_key(s.seed, step);
    }
    drop_stale_error();
    Batch b;
    b.count = 0;
    b.index = 0;
    long long chunks = 0;
    auto launch = [&]() {
        const int rc = with_type(dtype, [&](auto t) {
            return launch_status(launch_step<decltype(t)>(b, s, (uint32_t)chunks, bytes, (hipStream_t)stream));
        });
        b.index += (uint32_t)b.count;
        b.count = 0;
        chunks = 0;
        return rc;
    };
    for (int i = 0; i < count; ++i) {
        const long long own = (sizes[i] + kChunk - 1) / kChunk;
        if (b.count == kBatch || (b.count && chunks + own > kMostChunks)) {
            const int rc = launch();
            if (rc != SCC_OK) return rc;
        }
        b.first[b.count] = (uint32_t)chunks;
        b.weight[b.count++] = {w[i], g[i], first[i], second[i], bytes ? first_scales[i] : nullptr, bytes ? second_scales[i] : nullptr, sizes[i]};
        chunks += own;
    }
    return launch();
}
