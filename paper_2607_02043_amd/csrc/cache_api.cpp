// C ABI of the compact latent cache: argument checks and launches.  The entry
// points and their contracts are declared in include/mla_cache.h.
#include "mla_cache.h"

#include <hip/hip_runtime.h>

#include <cmath>

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

int check_window(const mla_window *w, bool null_ok) {
    if (!w) return null_ok ? MLA_OK : set_error(MLA_ERR_INVALID_ARG, "window is NULL");
    if (w->window < 1) return set_error(MLA_ERR_INVALID_ARG, "window of %d keys < 1", w->window);
    if (w->sinks < 0) return set_error(MLA_ERR_INVALID_ARG, "%d sinks < 0", w->sinks);
    return MLA_OK;
}

int check_cache8(const mla_batch *b, const mla_cache8 *c) {
    if (b->page_size < MLA_CACHE8_BLOCK)
        return set_error(MLA_ERR_UNSUPPORTED, "page_size = %d: the 8-bit cache needs pages of at least %d tokens", b->page_size,
                         MLA_CACHE8_BLOCK);
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

// Attention of both forms: exactly one of kv and cache is set.
int attend(const mla_batch *b, const uint16_t *q, const uint16_t *kv, const mla_cache8 *cache, const mla_window *win, float scale,
           void *out, int32_t out_dtype, float *lse, void *stream, const char *what) {
    int T = 0, log2_page = 0;
    int st = mla::batch_shape(b, &T, &log2_page);
    if (st != MLA_OK || b->num_reqs == 0) return st;
    if (!q || !out) return set_error(MLA_ERR_INVALID_ARG, "q / out is NULL");
    if (misaligned(q) || misaligned(out)) return set_error(MLA_ERR_INVALID_ARG, "q / out must be 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(lse) & 3) return set_error(MLA_ERR_INVALID_ARG, "lse must be 4-byte aligned");
    if (out_dtype != MLA_OUT_F32 && out_dtype != MLA_OUT_BF16)
        return set_error(MLA_ERR_INVALID_ARG, "out_dtype = %d is neither MLA_OUT_F32 nor MLA_OUT_BF16", out_dtype);
    if (!std::isfinite(scale) || scale <= 0.f) return set_error(MLA_ERR_INVALID_ARG, "softmax_scale must be finite and > 0");
    mla::AttnArgs a{};
    a.q = q;
    a.kv = kv;
    a.kv8 = cache ? cache->data : nullptr;
    a.kv8_scales = cache ? cache->scales : nullptr;
    a.window = win ? win->window : 0;
    a.sinks = win ? win->sinks : 0;
    a.cu_q = b->cu_q_dev;
    a.prefix = b->prefix_lens_dev;
    a.bt = b->block_table_dev;
    a.out = out;
    a.lse = lse;
    a.num_reqs = b->num_reqs;
    a.num_rows = T;
    a.page_size = b->page_size;
    a.log2_page = log2_page;
    a.max_pages = b->max_pages_per_req;
    a.num_pages = b->num_pages;
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.out_bf16 = out_dtype == MLA_OUT_BF16 ? 1 : 0;
    const mla::CheckUse use{cache ? MLA_CACHE8_BLOCK : 1, a.window, a.sinks};
    if ((st = mla::check_before(b, use, stream)) != MLA_OK) return st;
    const hipError_t e = mla::launch_rows(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return mla::hip_error(e, "attention kernel launch");
    return mla::check_after(what, stream);
}

size_t workspace(const mla_batch *b, const mla_window *win, bool eight) {
    int T = 0, log2_page = 0;
    if (mla::batch_shape(b, &T, &log2_page) != MLA_OK || b->num_reqs == 0) return 0;
    if (check_window(win, eight) != MLA_OK) return 0;
    if (eight && b->page_size < MLA_CACHE8_BLOCK) {
        set_error(MLA_ERR_UNSUPPORTED, "page_size = %d: the 8-bit cache needs pages of at least %d tokens", b->page_size, MLA_CACHE8_BLOCK);
        return 0;
    }
    return 0;
}

}  // namespace

extern "C" {

size_t mla_cache8_scale_bytes(int32_t num_pages, int32_t page_size) {
    if (num_pages < 1 || page_size < MLA_CACHE8_BLOCK || page_size > 1024 || (page_size & (page_size - 1)) != 0) return 0;
    const size_t n = (size_t)num_pages * (size_t)(page_size / MLA_CACHE8_BLOCK) * 4;
    return (n + 15) & ~size_t(15);
}

int append_latent_kv_rope(const mla_batch *batch, const uint16_t *new_latents, float rope_base, uint16_t *kv_cache, void *stream) {
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
    if ((st = mla::check_before(batch, {}, stream)) != MLA_OK) return st;
    const hipError_t e = mla::launch_append_rope(a, std::log2((double)rope_base), static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return mla::hip_error(e, "append kernel launch");
    return mla::check_after("append_latent_kv_rope", stream);
}

int append_latent_kv8(const mla_batch *batch, const uint16_t *new_latents, float rope_base, const mla_cache8 *cache, void *stream) {
    int T = 0, log2_page = 0;
    int st = mla::batch_shape(batch, &T, &log2_page);
    if (st != MLA_OK || batch->num_reqs == 0) return st;
    if ((st = check_cache8(batch, cache)) != MLA_OK || (st = check_new(new_latents)) != MLA_OK ||
        (st = check_base(rope_base, true)) != MLA_OK)
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
    a.log2_base = rope_base == 0.f ? 0.0 : std::log2((double)rope_base);
    a.num_reqs = batch->num_reqs;
    a.num_rows = T;
    a.num_blocks = (int)blocks;  // at most one per row
    a.log2_page = log2_page;
    a.page_size = batch->page_size;
    a.max_pages = batch->max_pages_per_req;
    a.num_pages = batch->num_pages;
    const mla::CheckUse use{MLA_CACHE8_BLOCK, 0, 0};
    if ((st = mla::check_before(batch, use, stream)) != MLA_OK) return st;
    const hipError_t e = mla::launch_append8(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return mla::hip_error(e, "8-bit append kernel launch");
    return mla::check_after("append_latent_kv8", stream);
}

size_t mixed_step_attn8_workspace_bytes(const mla_batch *batch, const mla_window *window) { return workspace(batch, window, true); }

size_t mixed_step_attn_window_workspace_bytes(const mla_batch *batch, const mla_window *window) {
    return workspace(batch, window, false);
}

int mixed_step_attn8(const mla_batch *batch, const uint16_t *q, const mla_cache8 *cache, const mla_window *window,
                     float softmax_scale, void *out, int32_t out_dtype, float *lse, void *workspace, size_t workspace_bytes,
                     void *stream) {
    int T = 0, log2_page = 0;
    int st = mla::batch_shape(batch, &T, &log2_page);
    if (st != MLA_OK || batch->num_reqs == 0) return st;
    if ((st = check_cache8(batch, cache)) != MLA_OK || (st = check_window(window, true)) != MLA_OK) return st;
    return attend(batch, q, nullptr, cache, window, softmax_scale, out, out_dtype, lse, stream, "mixed_step_attn8");
}

int mixed_step_attn_window(const mla_batch *batch, const uint16_t *q, const uint16_t *kv_cache, const mla_window *window,
                           float softmax_scale, void *out, int32_t out_dtype, float *lse, void *workspace, size_t workspace_bytes,
                           void *stream) {
    int T = 0, log2_page = 0;
    int st = mla::batch_shape(batch, &T, &log2_page);
    if (st != MLA_OK || batch->num_reqs == 0) return st;
    if (!kv_cache || misaligned(kv_cache)) return set_error(MLA_ERR_INVALID_ARG, "kv_cache is NULL or not 16-byte aligned");
    if ((st = check_window(window, false)) != MLA_OK) return st;
    return attend(batch, q, kv_cache, nullptr, window, softmax_scale, out, out_dtype, lse, stream, "mixed_step_attn_window");
}

}  // extern "C"
