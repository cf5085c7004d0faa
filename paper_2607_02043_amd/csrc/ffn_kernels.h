// Launch-side description of the feed-forward kernels of libmlastep (host <-> device).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ffn {

constexpr int kBK = 64;       // reduction depth of a tile's stage
constexpr int kMxGroup = 32;  // 4-bit weights that share a scale

// One weight matrix [N][K]: bf16 values, or 4-bit codes with their scales.
struct Weights {
    const uint16_t *w = nullptr;       // bf16 [N][K]
    const uint8_t *codes = nullptr;    // [N][K / 2]
    const uint8_t *scales = nullptr;   // [N][K / 32]
};

enum Epilogue : int {
    kStoreBf16 = 0,  // out bf16
    kStoreF32 = 1,   // out fp32
    kGate = 2,       // h = silu(g) u, as `planes` bf16 planes whose sum it is
};

// out[m][n] = sum_k a[m][k] b[n][k], a the sum of `a_planes` bf16 planes; with
// kGate also the products with `up`, and n counts columns of h.
struct GemmArgs {
    const uint16_t *a;        // bf16 [a_planes][plane_rows][K], rows 0 .. M - 1 of each plane
    int a_planes;
    Weights b, up;
    int M, N, K;
    int plane_rows;           // rows of a plane, of a and of h
    void *out;                // [M][N], kGate: bf16 [h_planes][plane_rows][N], rows 0 .. M - 1
    int h_planes;
    int splits;               // parts that K is cut into (set by launch_gemm)
    float *parts;             // and their workspace
    uint32_t *counters;
};

// The kernels: bm rows x bn weight rows a workgroup (kGate: bn / 2 columns of h).
enum Variant : int {
    kRows16, kRows16Narrow,                       // few rows, either kind of weights
    kTile32, kTile64, kTile128,                   // bf16 weights
    kMid16, kMid32, kMid48, kMid64,               // 4-bit weights, four wave groups on K
    kMid32Wide, kMid64Wide, kMid64Cols, kMid64Long,  // 4-bit weights, one or two
    kBig128, kBig256,                             // many rows, either kind
    kVariants
};
struct VariantSize {
    int bm, bn;
    bool bf16, four;
};
constexpr VariantSize kSizes[kVariants] = {
    {16, 32, true, true}, {16, 16, true, true},
    {32, 128, true, false}, {64, 128, true, false}, {128, 128, true, false},
    {16, 64, false, true}, {32, 64, false, true}, {48, 64, false, true}, {64, 64, false, true},
    {32, 256, false, true}, {64, 256, false, true}, {64, 128, false, true}, {64, 128, false, true},
    {128, 256, true, true}, {256, 256, true, true},
};
constexpr int kUnitStages = 4;  // stages of 64 k that a part of K has at least in the kernels for many rows

// A launch: K cut into `splits` parts, which meet in `parts` (tiles x splits x bm x bn fp32, at most kPartBytes); the
// workgroup that ends last joins them.  `counters` holds a zero for each of at most kMaxSplitTiles tiles.
struct Shape {
    Variant variant;
    int splits;
};
constexpr int kMaxSplitTiles = 1024;
constexpr size_t kPartBytes = size_t(64) << 20;

struct Tiles {
    long long m, n;
};
inline Tiles tiles_of(const GemmArgs &g, Epilogue epi, Variant v) {
    const int cols = epi == kGate ? kSizes[v].bn / 2 : kSizes[v].bn;
    return {((long long)g.M + kSizes[v].bm - 1) / kSizes[v].bm, ((long long)g.N + cols - 1) / cols};
}
// Whether a kernel takes the planes of x together, each weight read once; else one after the other, as a longer K.
inline bool planes_together(Variant v) { return v <= kTile128; }
// Whether the launch is one that the kernels take.
constexpr long long kMaxTiles = (1 << 23) - 1;  // (of up to 512 threads: a grid has fewer than 2^32)
inline bool fits(const GemmArgs &g, bool four_bit, Epilogue epi, const Shape &t) {
    if (t.variant < 0 || t.variant >= kVariants || !(four_bit ? kSizes[t.variant].four : kSizes[t.variant].bf16)) return false;
    if (g.M < 1 || g.N < 8 || g.N % 8 != 0 || g.K < 1 || g.K % (four_bit ? kMxGroup : 8) != 0 || t.splits < 1) return false;
    // three planes in front of fp32, with bf16 weights always
    if (g.a_planes != 1 && (g.a_planes != 3 || epi != kStoreF32)) return false;
    if (!four_bit && epi == kStoreF32 && g.a_planes != 3) return false;
    const Tiles n = tiles_of(g, epi, t.variant);
    if (n.m * n.n > kMaxTiles || (t.variant <= kRows16Narrow && n.m > 0xffff)) return false;
    const int stages = (g.K + kBK - 1) / kBK;
    const bool big = t.variant == kBig128 || t.variant == kBig256;
    if (big && stages < 2) return false;
    if (t.splits == 1) return true;
    // no part is empty: those for few rows deal out slices of two stages to eight waves, those for many count in units of
    // stages, the others in stages or in slices of up to four
    const int once = t.variant <= kRows16Narrow ? ((stages + 1) / 2 + 7) / 8 : big ? (stages < kUnitStages ? 1 : stages / kUnitStages) : (stages + 3) / 4;
    const long long pieces = (long long)once * (planes_together(t.variant) ? 1 : g.a_planes);
    return n.m * n.n <= kMaxSplitTiles && t.splits <= pieces &&
           (size_t)(n.m * n.n) * t.splits * kSizes[t.variant].bm * kSizes[t.variant].bn * 4 <= kPartBytes;
}
hipError_t launch_gemm(GemmArgs g, bool four_bit, Epilogue epi, const Shape &t, hipStream_t s);

}  // namespace ffn
