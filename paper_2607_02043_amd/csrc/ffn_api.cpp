// C ABI of the feed-forward half of a layer: argument checks, workspace layout and
// launches.  The entry points and their contracts are declared in include/mla_ffn.h.
#include "mla_ffn.h"

#include <hip/hip_runtime.h>

#include "api_util.h"
#include "ffn_kernels.h"

namespace {

using mla::set_error;

constexpr int kMaxSize = 1 << 24;

size_t a256(size_t v) { return (v + 255) & ~size_t(255); }
bool bad_ptr(const void *p) { return !p || (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
bool bad_size(int32_t v, int32_t step) { return v < 1 || v > kMaxSize || v % step != 0; }

int check_size(const char *name, int32_t v, int32_t step) {
    if (v < 1) return set_error(MLA_ERR_INVALID_ARG, "%s = %d < 1", name, v);
    if (v % step != 0 || v > kMaxSize)
        return set_error(MLA_ERR_UNSUPPORTED, "%s = %d is not a multiple of %d up to %d", name, v, step, kMaxSize);
    return MLA_OK;
}

int check_rows(int32_t T, const void *x, const void *out, int32_t out_dtype) {
    if (out_dtype != MLA_OUT_F32 && out_dtype != MLA_OUT_BF16)
        return set_error(MLA_ERR_INVALID_ARG, "out_dtype = %d is neither MLA_OUT_F32 nor MLA_OUT_BF16", out_dtype);
    if (bad_ptr(x) || bad_ptr(out)) return set_error(MLA_ERR_INVALID_ARG, "x / out must be non-NULL and 16-byte aligned");
    return MLA_OK;
}

int check_bf16(const char *name, const uint16_t *w) {
    return bad_ptr(w) ? set_error(MLA_ERR_INVALID_ARG, "%s must be non-NULL and 16-byte aligned", name) : MLA_OK;
}
int check_mx4(const char *name, const mla_mx4 *w) {
    if (!w || bad_ptr(w->codes) || bad_ptr(w->scales))
        return set_error(MLA_ERR_INVALID_ARG, "codes and scales of %s must be non-NULL and 16-byte aligned", name);
    return MLA_OK;
}

int check_workspace(const void *ws, size_t have, size_t need, int32_t T) {
    if (bad_ptr(ws) || have < need)
        return set_error(MLA_ERR_WORKSPACE, "workspace of %zu bytes at %p; %d rows need %zu", have, ws, T, need);
    return MLA_OK;
}

// Planes of h: one bf16 where the output is rounded to bf16 anyway, three (24 bits) in front of fp32.
int planes_of(int32_t out_dtype) { return out_dtype == MLA_OUT_F32 ? 3 : 1; }

// Workspace: the counters, then h (room for three planes).
size_t h_at() { return MLA_FFN_COUNTER_BYTES; }
size_t ffn_bytes(int32_t T, int32_t inner) { return h_at() + a256((size_t)T * (size_t)inner * 3 * 2); }
size_t linear_bytes() { return MLA_FFN_COUNTER_BYTES; }

int cu_count() {
    int ncu = 256, dev = 0, v = 0;
    if (hipGetDevice(&dev) == hipSuccess &&
        hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && v > 0)
        ncu = v;
    return ncu;
}

ffn::Shape pick_shape(const ffn::GemmArgs &g, ffn::Epilogue epi) {
    static const ffn::Shape shapes[] = {{256, 256}, {128, 128}, {64, 128}, {32, 128}};
    const long long need = cu_count() * 85LL / 100;
    ffn::Shape t{};
    for (const ffn::Shape &c : shapes) {
        t = c;
        const int cols = epi == ffn::kGate ? c.bn / 2 : c.bn;
        if ((long long)((g.M + c.bm - 1) / c.bm) * ((g.N + cols - 1) / cols) >= need) break;
    }
    return t;
}

int launch(const ffn::GemmArgs &g, bool four, ffn::Epilogue epi, hipStream_t s, const char *what) {
    const hipError_t e = ffn::launch_gemm(g, four, epi, pick_shape(g, epi), s);
    return e == hipSuccess ? MLA_OK : mla::hip_error(e, what);
}

int ffn_run(int32_t T, const uint16_t *x, const ffn::Weights (&w)[3], bool four, int32_t H, int32_t I, void *out, int32_t out_dtype,
            void *workspace, size_t workspace_bytes, hipStream_t s) {
    int st = check_workspace(workspace, workspace_bytes, ffn_bytes(T, I), T);
    if (st != MLA_OK) return st;
    char *const ws = static_cast<char *>(workspace);
    ffn::GemmArgs g{};
    g.a = x;
    g.a_planes = 1;
    g.b = w[0];
    g.up = w[1];
    g.M = T;
    g.N = I;
    g.K = H;
    g.out = ws + h_at();
    g.h_planes = planes_of(out_dtype);
    if ((st = launch(g, four, ffn::kGate, s, "gate and up projection")) != MLA_OK) return st;
    ffn::GemmArgs d{};
    d.a = reinterpret_cast<const uint16_t *>(ws + h_at());
    d.a_planes = g.h_planes;
    d.b = w[2];
    d.M = T;
    d.N = H;
    d.K = I;
    d.out = out;
    return launch(d, four, out_dtype == MLA_OUT_F32 ? ffn::kStoreF32 : ffn::kStoreBf16, s, "down projection");
}

}  // namespace

extern "C" {

size_t mla_linear4_workspace_bytes(int32_t num_rows, int32_t in_features, int32_t out_features) {
    if (num_rows <= 0 || bad_size(in_features, MLA_MX4_GROUP) || bad_size(out_features, 8)) return 0;
    return linear_bytes();
}

int mla_linear4(int32_t num_rows, const uint16_t *x, const mla_mx4 *w, int32_t in_features, int32_t out_features, void *out,
                int32_t out_dtype, void *workspace, size_t workspace_bytes, void *stream) {
    set_error(MLA_OK, "");
    if (num_rows < 0) return set_error(MLA_ERR_INVALID_ARG, "num_rows = %d < 0", num_rows);
    int st = check_size("in_features", in_features, MLA_MX4_GROUP);
    if (st != MLA_OK || (st = check_size("out_features", out_features, 8)) != MLA_OK) return st;
    if (num_rows == 0) return MLA_OK;
    if ((st = check_rows(num_rows, x, out, out_dtype)) != MLA_OK || (st = check_mx4("w", w)) != MLA_OK ||
        (st = check_workspace(workspace, workspace_bytes, linear_bytes(), num_rows)) != MLA_OK)
        return st;
    ffn::GemmArgs g{};
    g.a = x;
    g.a_planes = 1;
    g.b = ffn::Weights{nullptr, w->codes, w->scales};
    g.M = num_rows;
    g.N = out_features;
    g.K = in_features;
    g.out = out;
    return launch(g, true, out_dtype == MLA_OUT_F32 ? ffn::kStoreF32 : ffn::kStoreBf16, static_cast<hipStream_t>(stream),
                  "product with 4-bit weights");
}

size_t mla_gated_ffn_workspace_bytes(int32_t num_rows, int32_t hidden, int32_t inner) {
    if (num_rows <= 0 || bad_size(hidden, 8) || bad_size(inner, 8)) return 0;
    return ffn_bytes(num_rows, inner);
}

int mla_gated_ffn(int32_t num_rows, const uint16_t *x, const mla_ffn_weights *w, void *out, int32_t out_dtype, void *workspace,
                  size_t workspace_bytes, void *stream) {
    set_error(MLA_OK, "");
    if (num_rows < 0) return set_error(MLA_ERR_INVALID_ARG, "num_rows = %d < 0", num_rows);
    if (!w) return set_error(MLA_ERR_INVALID_ARG, "weights is NULL");
    int st = check_size("hidden", w->hidden, 8);
    if (st != MLA_OK || (st = check_size("inner", w->inner, 8)) != MLA_OK) return st;
    if (num_rows == 0) return MLA_OK;
    if ((st = check_rows(num_rows, x, out, out_dtype)) != MLA_OK || (st = check_bf16("w_gate", w->w_gate)) != MLA_OK ||
        (st = check_bf16("w_up", w->w_up)) != MLA_OK || (st = check_bf16("w_down", w->w_down)) != MLA_OK)
        return st;
    const ffn::Weights ws[3] = {{w->w_gate, nullptr, nullptr}, {w->w_up, nullptr, nullptr}, {w->w_down, nullptr, nullptr}};
    return ffn_run(num_rows, x, ws, false, w->hidden, w->inner, out, out_dtype, workspace, workspace_bytes,
                   static_cast<hipStream_t>(stream));
}

int mla_gated_ffn4(int32_t num_rows, const uint16_t *x, const mla_ffn4_weights *w, void *out, int32_t out_dtype, void *workspace,
                   size_t workspace_bytes, void *stream) {
    set_error(MLA_OK, "");
    if (num_rows < 0) return set_error(MLA_ERR_INVALID_ARG, "num_rows = %d < 0", num_rows);
    if (!w) return set_error(MLA_ERR_INVALID_ARG, "weights is NULL");
    int st = check_size("hidden", w->hidden, MLA_MX4_GROUP);
    if (st != MLA_OK || (st = check_size("inner", w->inner, MLA_MX4_GROUP)) != MLA_OK) return st;
    if (num_rows == 0) return MLA_OK;
    if ((st = check_rows(num_rows, x, out, out_dtype)) != MLA_OK || (st = check_mx4("w_gate", &w->w_gate)) != MLA_OK ||
        (st = check_mx4("w_up", &w->w_up)) != MLA_OK || (st = check_mx4("w_down", &w->w_down)) != MLA_OK)
        return st;
    const ffn::Weights ws[3] = {{nullptr, w->w_gate.codes, w->w_gate.scales},
                                {nullptr, w->w_up.codes, w->w_up.scales},
                                {nullptr, w->w_down.codes, w->w_down.scales}};
    return ffn_run(num_rows, x, ws, true, w->hidden, w->inner, out, out_dtype, workspace, workspace_bytes,
                   static_cast<hipStream_t>(stream));
}

}  // extern "C"
