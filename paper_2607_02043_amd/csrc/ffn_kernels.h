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
    const uint16_t *a;        // bf16 [a_planes][M][K]
    int a_planes;
    Weights b, up;
    int M, N, K;
    void *out;                // [M][N], kGate: bf16 [h_planes][M][N]
    int h_planes;
};

// Tile of one launch: bm rows x bn weight rows (kGate: bn / 2 columns of h).
// Instantiated: (32, 128), (64, 128), (128, 128) on four waves, (256, 256) on eight.
struct Shape {
    int bm, bn;
};

hipError_t launch_gemm(const GemmArgs &g, bool four_bit, Epilogue epi, const Shape &t, hipStream_t s);

}  // namespace ffn
