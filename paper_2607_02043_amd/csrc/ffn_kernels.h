// Launch-side description of the feed-forward kernels of libmlastep (host <-> device).
#pragma once
#include <hip/hip_runtime.h>
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
    kRows16,                                      // few rows, either kind of weights
    kTile32, kTile64, kTile128,                   // bf16 weights
    kMid16, kMid32, kMid48, kMid64,               // 4-bit weights, four wave groups on K
    kMid32Wide, kMid64Wide, kMid64Cols, kMid64Pair, kMid64Long,  // 4-bit weights, one or two
    kBig128, kBig256,                             // many rows, either kind
    kVariants
};
struct VariantSize {
    int bm, bn;
    bool bf16, four;
};
constexpr VariantSize kSizes[kVariants] = {
    {16, 32, true, true},
    {32, 128, true, false}, {64, 128, true, false}, {128, 128, true, false},
    {16, 64, false, true}, {32, 64, false, true}, {48, 64, false, true}, {64, 64, false, true},
    {32, 256, false, true}, {64, 256, false, true}, {64, 128, false, true}, {64, 128, false, true}, {64, 128, false, true},
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

// Whether the launch is one that the kernels take.
bool fits(const GemmArgs &g, bool four_bit, Epilogue epi, const Shape &t);
hipError_t launch_gemm(GemmArgs g, bool four_bit, Epilogue epi, const Shape &t, hipStream_t s);

}  // namespace ffn
