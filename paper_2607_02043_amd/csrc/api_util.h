// Error reporting and batch checks shared by the entry points of libmlastep.
#pragma once
#include "mla_step.h"

#include <hip/hip_runtime.h>
#include "chunk_route.h"
#include "mla_kernels.h"

namespace mla {

// What a call uses of the cache, for check mode: writes in blocks of `block`
// tokens, and, with a window (0: none), no key in [sinks, p - window].  An append
// reads no key before the first block that it writes into, as with a window of 1.
struct CheckUse {
    long long block = 1, window = 0, sinks = 0;
};
inline CheckUse append_use(long long block) { return CheckUse{block, 1, 0}; }

// Status and message of a failed HIP call.
int hip_error(hipError_t e, const char *what);

// Host checks of a batch, its rows and log2 of its page size (set only if there are requests).
int batch_shape(const mla_batch *batch, int *num_rows, int *log2_page);

// Check mode's tests before and after a launch; MLA_OK at once when it is off.
int check_before(const mla_batch *batch, const CheckUse &use, void *stream);
int check_after(const char *what, void *stream);


// Sets the thread's mla_last_error message (printf format) and returns code.
int set_error(int code, const char *fmt, ...);

// Host checks of a batch (those of every entry point); *num_rows = T on success.
// Clears the thread's error message first.
int batch_rows(const mla_batch *batch, int *num_rows);

// Workspace bytes of the attention launch for this batch (mixed_step_workspace_bytes
// with the status of the checks and the planning), leaving out the chunk
// requests that `route` sends to the multi-head path.
int attn_workspace(const mla_batch *batch, size_t *bytes, ChunkRoute route = kAbsorbAll, const Form &form = {});

// mixed_step_attn in a form of mla_cache.h, whose own arguments are checked already.
int attend_form(const mla_batch *batch, const uint16_t *q, const uint16_t *kv_cache, const Form &form, float softmax_scale,
                void *out, int32_t out_dtype, float *lse, void *workspace, size_t workspace_bytes, void *stream, const char *what);

// mixed_step (no lse) over every row except those of the chunk requests that
// `route` sends to the multi-head path, which are left untouched: neither
// attended nor appended.  new_latents NULL: no append (mixed_step_attn).
int attend_rows(const mla_batch *batch, const uint16_t *q, const uint16_t *new_latents, uint16_t *kv_cache,
                float softmax_scale, void *out, int32_t out_dtype, void *workspace, size_t workspace_bytes, void *stream,
                ChunkRoute route);

}  // namespace mla
