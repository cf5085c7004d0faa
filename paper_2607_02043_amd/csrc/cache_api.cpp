// C ABI of the compact latent cache: argument checks and launches.  The entry
// points and their contracts are declared in include/mla_cache.h.
#include "mla_cache.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <exception>

#include "api_util.h"
#include "mla_kernels.h"

namespace {

using mla::set_error;

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

int check_base(float base, bool zero_ok) {
    if (zero_ok && base == 0.f) return MLA_OK;
    if (!std::isfinite(base) || base <= 1.f)
        return set_error(MLA_ERR_INVALID_ARG, "rope_base = %g is not a finite number above 1", (double)base);
    return MLA_OK;
}

// The last base's table is kept per thread (32 powers of 2, a microsecond).
const mla::RopeTable &rope_table(float base) {
    thread_local mla::RopeTable t;
    thread_local float of = 0.f;
    if (of != base) {
        const double log2_base = std::log2((double)base);
        for (int i = 0; i < 32; ++i) t.turns[i] = std::exp2(-(double)i / 32.0 * log2_base) * 0.15915494309189533577;
        of = base;
    }
    return t;
}

int check_window(const mla_window *w, bool null_ok) {
    if (!w) return null_ok ? MLA_OK : set_error(MLA_ERR_INVALID_ARG, "window is NULL");
    if (w->window < 1) return set_error(MLA_ERR_INVALID_ARG, "window of %d keys < 1", w->window);
    if (w->sinks < 0) return set_error(MLA_ERR_INVALID_ARG, "%d sinks < 0", w->sinks);
    return MLA_OK;
}

int check_cache8(const mla_cache8 *c) {
    if (!c || !c->data || !c->scales) return set_error(MLA_ERR_INVALID_ARG, "the cache, its data or its scales are NULL");
    if (misaligned(c->data) || misaligned(c->scales))
        return set_error(MLA_ERR_INVALID_ARG, "cache data / scales must be 16-byte aligned");
    return MLA_OK;
}

int check_new(const uint16_t *new_latents) {
    if (!new_latents) return set_error(MLA_ERR_INVALID_ARG, "new_latents is NULL");
    if (misaligned(new_latents)) return set_error(MLA_ERR_INVALID_ARG, "new_latents must be 16-byte aligned");
    return MLA_OK;
}

// The window as the planner and the kernels take it: beyond 2^30 keys, more than a
// request may have, nothing changes any more.
mla::Band band_of(const mla_window *w) {
    mla::Band b{};
    if (!w) return b;
    const long long most = 1LL << 30;
    b.window = (int32_t)std::min<long long>(w->window, most);
    b.sinks = (int32_t)std::min<long long>(w->sinks, most);
    const long long sink_keys = ((long long)b.sinks + mla::kKeysPerTile - 1) / mla::kKeysPerTile * mla::kKeysPerTile;
    b.sink_keys = (int32_t)sink_keys;
    b.span = (int32_t)std::min(most, sink_keys + b.window + mla::kChunkBlockTokens + mla::kKeysPerTile - 2);
    return b;
}

// Checks what the form adds to a batch's own arguments, and makes the form, without the 8-bit cache's pointers.
int make_form(const mla_batch *batch, bool eight, const mla_window *window, mla::Form *form) {
    if (eight && batch->page_size < MLA_CACHE8_BLOCK)
        return set_error(MLA_ERR_UNSUPPORTED, "page_size = %d: the 8-bit cache needs pages of at least %d tokens", batch->page_size,
                         MLA_CACHE8_BLOCK);
    const int st = check_window(window, eight);
    if (st != MLA_OK) return st;
    form->eight = eight;
    form->band = band_of(window);
    return MLA_OK;
}

// Runs an entry point's body: an exception (the planner and check mode take host memory) becomes its error.
template <class Body>
int guarded(const Body &body) {
    try {
        return body();
    } catch (const std::exception &e) {
        return set_error(MLA_ERR_HIP, "host side: %s", e.what());
    }
}

size_t workspace(const mla_batch *batch, const mla_window *window, bool eight) {
    size_t bytes = 0;
    const int st = guarded([&]() -> int {
        int T = 0;
        mla::Form form;
        int st = mla::batch_rows(batch, &T);
        if (st != MLA_OK || batch->num_reqs == 0) return st;
        if ((st = make_form(batch, eight, window, &form)) != MLA_OK) return st;
        return mla::attn_workspace(batch, &bytes, mla::kAbsorbAll, form);
    });
    return st == MLA_OK ? bytes : 0;
}

}  // namespace

extern "C" {

size_t mla_cache8_scale_bytes(int32_t num_pages, int32_t page_size) {
    if (num_pages < 1 || page_size < MLA_CACHE8_BLOCK || page_size > 1024 || (page_size & (page_size - 1)) != 0) return 0;
    const size_t n = (size_t)num_pages * (size_t)(page_size / MLA_CACHE8_BLOCK) * 4;
    return (n + 15) & ~size_t(15);
}

int append_latent_kv_rope(const mla_batch *batch, const uint16_t *new_latents, float rope_base, uint16_t *kv_cache, void *stream) {
    return guarded([&]() -> int {
        int T = 0, log2_page = 0;
        int st = mla::batch_shape(batch, &T, &log2_page);
        if (st != MLA_OK || batch->num_reqs == 0) return st;
        if ((st = check_new(new_latents)) != MLA_OK || (st = check_base(rope_base, false)) != MLA_OK) return st;
        if (!kv_cache || misaligned(kv_cache)) return set_error(MLA_ERR_INVALID_ARG, "kv_cache is NULL or not 16-byte aligned");
        mla::AppendArgs a;
        a.src = new_latents;
        a.kv = kv_cache;
        a.cu_q = batch->cu_q_dev;
        a.prefix = batch->prefix_lens_dev;
        a.bt = batch->block_table_dev;
        a.num_reqs = batch->num_reqs;
        a.num_rows = T;
        a.page_size = batch->page_size;
        a.log2_page = log2_page;
        a.max_pages = batch->max_pages_per_req;
        a.num_pages = batch->num_pages;
        if ((st = mla::check_before(batch, mla::append_use(1), stream)) != MLA_OK) return st;
        const hipError_t e = mla::launch_append_rope(a, rope_table(rope_base), static_cast<hipStream_t>(stream));
        if (e != hipSuccess) return mla::hip_error(e, "append kernel launch");
        return mla::check_after("append_latent_kv_rope", stream);
    });
}

int append_latent_kv8(const mla_batch *batch, const uint16_t *new_latents, float rope_base, const mla_cache8 *cache, void *stream) {
    return guarded([&]() -> int {
        int T = 0, log2_page = 0;
        int st = mla::batch_shape(batch, &T, &log2_page);
        if (st != MLA_OK || batch->num_reqs == 0) return st;
        mla::Form form;
        if ((st = make_form(batch, true, nullptr, &form)) != MLA_OK || (st = check_cache8(cache)) != MLA_OK ||
            (st = check_new(new_latents)) != MLA_OK || (st = check_base(rope_base, true)) != MLA_OK)
            return st;
        long long blocks = 0;
        for (int r = 0; r < batch->num_reqs; ++r) {
            const long long p = batch->prefix_lens[r], last = p + batch->q_lens[r] - 1;
            blocks += last / MLA_CACHE8_BLOCK - p / MLA_CACHE8_BLOCK + 1;
        }
        mla::Append8Args a;
        a.src = new_latents;
        a.data = cache->data;
        a.scales = cache->scales;
        a.cu_q = batch->cu_q_dev;
        a.prefix = batch->prefix_lens_dev;
        a.bt = batch->block_table_dev;
        a.rotate = rope_base != 0.f;
        a.num_reqs = batch->num_reqs;
        a.num_rows = T;
        a.num_blocks = (int)blocks;  // at most one per row
        a.log2_page = log2_page;
        a.page_size = batch->page_size;
        a.max_pages = batch->max_pages_per_req;
        a.num_pages = batch->num_pages;
        if ((st = mla::check_before(batch, mla::append_use(MLA_CACHE8_BLOCK), stream)) != MLA_OK) return st;
        const hipError_t e = mla::launch_append8(a, rope_table(rope_base), static_cast<hipStream_t>(stream));
        if (e != hipSuccess) return mla::hip_error(e, "8-bit append kernel launch");
        return mla::check_after("append_latent_kv8", stream);
    });
}

size_t mixed_step_attn8_workspace_bytes(const mla_batch *batch, const mla_window *window) { return workspace(batch, window, true); }

size_t mixed_step_attn_window_workspace_bytes(const mla_batch *batch, const mla_window *window) {
    return workspace(batch, window, false);
}

int mixed_step_attn8(const mla_batch *batch, const uint16_t *q, const mla_cache8 *cache, const mla_window *window,
                     float softmax_scale, void *out, int32_t out_dtype, float *lse, void *workspace, size_t workspace_bytes,
                     void *stream) {
    return guarded([&]() -> int {
        int T = 0;
        mla::Form form;
        int st = mla::batch_rows(batch, &T);
        if (st != MLA_OK || batch->num_reqs == 0) return st;
        if ((st = make_form(batch, true, window, &form)) != MLA_OK || (st = check_cache8(cache)) != MLA_OK) return st;
        form.kv8 = cache->data;
        form.kv8_scales = cache->scales;
        return mla::attend_form(batch, q, nullptr, form, softmax_scale, out, out_dtype, lse, workspace, workspace_bytes, stream,
                                "mixed_step_attn8");
    });
}

int mixed_step_attn_window(const mla_batch *batch, const uint16_t *q, const uint16_t *kv_cache, const mla_window *window,
                           float softmax_scale, void *out, int32_t out_dtype, float *lse, void *workspace, size_t workspace_bytes,
                           void *stream) {
    return guarded([&]() -> int {
        int T = 0;
        mla::Form form;
        int st = mla::batch_rows(batch, &T);
        if (st != MLA_OK || batch->num_reqs == 0) return st;
        if ((st = make_form(batch, false, window, &form)) != MLA_OK) return st;
        return mla::attend_form(batch, q, kv_cache, form, softmax_scale, out, out_dtype, lse, workspace, workspace_bytes, stream,
                                "mixed_step_attn_window");
    });
}

}  // extern "C"
