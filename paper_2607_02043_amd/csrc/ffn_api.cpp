// C ABI of the feed-forward half of a layer: argument checks, workspace layout and
// launches.  The entry points and their contracts are declared in include/mla_ffn.h.
#include "mla_ffn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "api_util.h"
#include "ffn_kernels.h"

namespace {

using mla::set_error;

constexpr int kMaxSize = 1 << 24;
constexpr int kMaxRows = 1 << 28;

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
    if (T > kMaxRows) return set_error(MLA_ERR_UNSUPPORTED, "num_rows = %d > %d", T, kMaxRows);
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

// Workspace: the counters, room for the parts of split sums (as much as any launch takes: the choice for fewer rows may
// split where that for more does not), then h (room for three planes, as the output's type is not known here).
size_t h_at() { return MLA_FFN_COUNTER_BYTES + ffn::kPartBytes; }
size_t ffn_bytes(int32_t T, int32_t inner) { return h_at() + a256((size_t)T * (size_t)inner * 3 * 2); }
size_t linear_bytes() { return MLA_FFN_COUNTER_BYTES + ffn::kPartBytes; }
static_assert(MLA_FFN_COUNTER_BYTES == ffn::kMaxSplitTiles * 4, "a counter for each tile of a split launch");
void use_workspace(ffn::GemmArgs *g, char *ws) {
    g->counters = reinterpret_cast<uint32_t *>(ws);
    g->parts = reinterpret_cast<float *>(ws + MLA_FFN_COUNTER_BYTES);
}

int cu_count() {
    int ncu = 256, dev = 0, v = 0;
    if (hipGetDevice(&dev) == hipSuccess &&
        hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && v > 0)
        ncu = v;
    return ncu;
}

// What a launch takes, in us, fitted to sweeps of the kernels and numbers of parts on an MI355X with weights from memory.
// A workgroup walks its stages of 64 k (1 / groups of them) at `stage` us each; where a CU gets up to `resident` workgroups,
// a stage takes `share` us for each of them, and rounds of them follow each other.  All but `groups` are numbers of the fit:
// `resident` is not what registers and LDS let a CU hold (one to three workgroups, fewer than `resident` for the few-row
// kernels, kTile32 and kMid16 to kMid48).  Parts are stored at 2.5 TB/s by all, and read by the workgroup that joins a
// tile's at 60 GB/s.  Of 143 products of 1 to 2200 rows the choice takes 1.7 % longer than the best in the mean, 18 more
// than 6 % and seven more than 12 %, all seven with 4-bit weights (64 rows of 2048 columns, K = 5504 in three planes:
// 20.6 against 16.4 us).
struct Cost {
    float fixed, stage, share;
    int resident, groups;
};
constexpr Cost kCostBf16[ffn::kVariants] = {
    {3.f, 1.4f, 1.7f, 4, 8}, {2.3f, 1.f, .94f, 3, 8},
    {3.5f, .5f, .5f, 2, 1}, {4.5f, .48f, .4f, 2, 1}, {4.5f, .65f, .65f, 1, 1},
    {}, {}, {}, {}, {}, {}, {}, {},
    {5.f, 1.f, 1.f, 1, 1}, {7.f, 1.32f, 1.32f, 1, 1},
};
constexpr Cost kCost4[ffn::kVariants] = {
    {3.f, .77f, 1.f, 4, 8}, {2.3f, .68f, .72f, 4, 8},
    {}, {}, {},
    {3.f, .7f, .6f, 4, 4}, {3.f, .9f, .85f, 4, 4}, {3.f, 1.15f, 1.2f, 2, 4}, {3.f, 1.25f, 1.3f, 1, 4},
    {3.f, .7f, .57f, 2, 1}, {3.f, .9f, .6f, 2, 1}, {3.f, .6f, .3f, 2, 1},
    {3.f, .85f, .9f, 1, 2},
    {5.f, 1.04f, 1.04f, 1, 1}, {8.f, 1.45f, 1.45f, 1, 1},
};

// The kernels that take three planes of x together.
constexpr Cost kCostBf16x3[] = {{3.f, 2.f, 2.f, 1, 8}, {2.3f, 1.75f, 1.75f, 1, 8}, {5.f, .86f, .53f, 2, 1}, {5.f, .8f, .8f, 1, 1}, {6.f, 1.4f, 1.4f, 1, 1}};
constexpr Cost kCost4x3[] = {{3.f, 1.5f, 1.5f, 1, 8}, {2.3f, 1.3f, 1.3f, 1, 8}, {}, {}, {}};

float cost_of(const ffn::GemmArgs &g, bool four, ffn::Epilogue epi, const ffn::Shape &t, int ncu) {
    const bool together = g.a_planes == 3 && ffn::planes_together(t.variant);
    const Cost &c = together ? (four ? kCost4x3 : kCostBf16x3)[t.variant] : (four ? kCost4 : kCostBf16)[t.variant];
    const ffn::VariantSize &v = ffn::kSizes[t.variant];
    const ffn::Tiles n = ffn::tiles_of(g, epi, t.variant);
    const double tiles = (double)(n.m * n.n);
    const double chain = std::ceil(std::ceil(g.K / 64.0) * (together ? 1 : g.a_planes) / t.splits / c.groups), load = tiles * t.splits / ncu;
    const double part = 4.0 * v.bm * v.bn, joined = t.splits > 1 ? 2.0 + t.splits * part / 6e4 + tiles * t.splits * part / 2.5e6 : 0.0;
    // workgroups a CU has at once, and how many times (past one and a half rounds they no longer end together)
    const double once = std::min<double>(c.resident, std::ceil(load)), rounds = load > 1.5 * c.resident && c.resident > 1 ? load / c.resident : std::ceil(load / once);
    // (the few-row kernel reads each row of x for itself: a single one costs it less)
    const double rows = t.variant > ffn::kRows16Narrow ? 1.0 : four ? .55 + .45 * std::min(g.M, 16) / 16 : .7 + .3 * std::min(g.M, 16) / 16;
    const double walk = rounds * (c.fixed + chain * rows * (once > 1 ? std::max<double>(c.stage, once * c.share) : c.stage)) + joined;
    // what the weights take to arrive: 5 TB/s in bf16, in 4 bits 3.4 where wave groups share K and 2.7 where they do not
    const double bytes = (epi == ffn::kGate ? 2.0 : 1.0) * g.N * (double)g.K * (four ? .53 : 2.0);
    return (float)std::max(walk, bytes / (!four ? 5e6 : c.groups >= 4 ? 3.4e6 : 2.7e6) + c.fixed);
}

struct Plan {
    ffn::Shape shape{};
    float us = 0;
    int rest = 0;  // rows at the end that a launch of their own takes
    ffn::Shape rest_shape{};
};

// The cheapest kernel and number of parts for these rows.
Plan best_whole(const ffn::GemmArgs &g, bool four, ffn::Epilogue epi, int ncu) {
    Plan best;
    best.us = INFINITY;
    for (int v = 0; v < ffn::kVariants; ++v) {
        ffn::Shape t{static_cast<ffn::Variant>(v), 1};
        if (!ffn::fits(g, four, epi, t)) continue;
        const ffn::Tiles n = ffn::tiles_of(g, epi, t.variant);
        for (; t.splits <= 32; ++t.splits) {
            if (t.splits > 1 && (n.m * n.n * t.splits > 2LL * ncu || !ffn::fits(g, four, epi, t))) break;
            const float us = cost_of(g, four, epi, t, ncu);
            if (us < best.us) best = {t, us};
        }
    }
    return best;
}

// One launch for all rows, or one for a multiple of 128 or 256 and one for the rows behind it, which would
// cost the first a round of workgroups (4160 rows x 2048 of K = 10944: 219 us, as 4096 and 64 rows 156 + 20).
// A thread keeps those of the last kKeptPlans sizes that it planned: a step calls with the same ones for every layer.
// (On the host planning a launch takes 1 to 4 us, finding it 0.03: products of 1 to 4160 rows, 8 sizes in turn.)
constexpr int kKeptPlans = 16;
Plan plan_of(const ffn::GemmArgs &g, bool four, ffn::Epilogue epi) {
    struct Entry {
        int dev = -1, M = 0, N = 0, K = 0, kind = 0;
        Plan plan;
    };
    thread_local Entry kept[kKeptPlans];
    thread_local int oldest = 0;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) dev = 0;
    const int kind = (four ? 1 : 0) + 2 * epi + 8 * g.a_planes;
    for (const Entry &e : kept)
        if (e.dev == dev && e.M == g.M && e.N == g.N && e.K == g.K && e.kind == kind) return e.plan;
    const int ncu = cu_count();
    Plan best = best_whole(g, four, epi, ncu);
    for (int step : {128, 256}) {
        ffn::GemmArgs part = g;
        const int rest = g.M % step;
        if (rest == 0 || g.M < 2 * step) continue;
        part.M = g.M - rest;
        Plan p = best_whole(part, four, epi, ncu);
        part.M = rest;
        const Plan behind = best_whole(part, four, epi, ncu);
        p.us = 1.05f * (p.us + behind.us);  // not for a few per cent
        p.rest = rest;
        p.rest_shape = behind.shape;
        if (p.us < best.us) best = p;
    }
    kept[oldest] = {dev, g.M, g.N, g.K, kind, best};
    oldest = (oldest + 1) % kKeptPlans;
    return best;
}

int launch(ffn::GemmArgs g, bool four, ffn::Epilogue epi, hipStream_t s, const char *what) {
    const Plan plan = plan_of(g, four, epi);
    if (plan.shape.splits < 1) return set_error(MLA_ERR_UNSUPPORTED, "%s: %d x %d outputs are more tiles than a launch takes", what, g.M, g.N);
    const int rows = g.M;
    g.M = rows - plan.rest;
    hipError_t e = ffn::launch_gemm(g, four, epi, plan.shape, s);
    if (e == hipSuccess && plan.rest > 0) {
        const size_t width = epi == ffn::kStoreF32 ? 4 : 2;
        g.a += (size_t)g.M * g.K;
        g.out = static_cast<char *>(g.out) + (size_t)g.M * g.N * width;
        g.M = plan.rest;
        e = ffn::launch_gemm(g, four, epi, plan.rest_shape, s);
    }
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
    g.M = g.plane_rows = T;
    g.N = I;
    g.K = H;
    g.out = ws + h_at();
    g.h_planes = planes_of(out_dtype);
    use_workspace(&g, ws);
    if ((st = launch(g, four, ffn::kGate, s, "gate and up projection")) != MLA_OK) return st;
    ffn::GemmArgs d{};
    d.a = reinterpret_cast<const uint16_t *>(ws + h_at());
    d.a_planes = g.h_planes;
    d.b = w[2];
    d.M = d.plane_rows = T;
    d.N = H;
    d.K = I;
    d.out = out;
    use_workspace(&d, ws);
    return launch(d, four, out_dtype == MLA_OUT_F32 ? ffn::kStoreF32 : ffn::kStoreBf16, s, "down projection");
}

}  // namespace

extern "C" {

size_t mla_linear4_workspace_bytes(int32_t num_rows, int32_t in_features, int32_t out_features) {
    if (num_rows <= 0 || num_rows > kMaxRows || bad_size(in_features, MLA_MX4_GROUP) || bad_size(out_features, 8)) return 0;
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
    g.M = g.plane_rows = num_rows;
    g.N = out_features;
    g.K = in_features;
    g.out = out;
    use_workspace(&g, static_cast<char *>(workspace));
    return launch(g, true, out_dtype == MLA_OUT_F32 ? ffn::kStoreF32 : ffn::kStoreBf16, static_cast<hipStream_t>(stream),
                  "product with 4-bit weights");
}

size_t mla_gated_ffn_workspace_bytes(int32_t num_rows, int32_t hidden, int32_t inner) {
    if (num_rows <= 0 || num_rows > kMaxRows || bad_size(hidden, 8) || bad_size(inner, 8)) return 0;
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
