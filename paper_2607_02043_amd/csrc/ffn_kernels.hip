// Feed-forward kernels for gfx950: products of bf16 rows with bf16 or 4-bit
// weights, and the gated first half of the block.  Host-side contracts are in
// include/mla_ffn.h.
//
// Every product is out = A . B^T with both operands K-contiguous, on bf16 MFMA
// 16x16x32 with fp32 sums, taken as B . A^T so that a lane holds neighbouring
// columns of one row.  4-bit weights become bf16 on the way (exactly, scale
// included, two an instruction), so both formats share the products.
#include "ffn_kernels.h"

namespace ffn {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ uint32_t bf16_of(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ float bf16_value(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ __forceinline__ uint32_t pack2(float lo, float hi) { return bf16_of(lo) | (bf16_of(hi) << 16); }

// A scale byte b as the number 2^(b - 127): its bits as an fp32 exponent (0 and 255,
// which are no fp32 powers of two, the conversion takes as 2^-127 and NaN).
__device__ __forceinline__ float mx_scale(uint32_t b) { return __uint_as_float(b << 23); }
// Eight codes (even ones in the low halves) times their scale, as bf16.
__device__ __forceinline__ u32x4 mx_values(uint32_t codes, float scale) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

// h = silu(g) u.  exp(-g) overflows to infinity where silu(g) is below the smallest
// fp32: the quotient is then 0, as it should.
__device__ __forceinline__ float gated(float g, float u) { return g / (1.f + expf(-g)) * u; }

// v as the sum of bf16 values, most significant first: the next plane takes what the
// last one left.  A value whose first rounding is not finite has zeros behind it.
__device__ __forceinline__ uint32_t next_plane(float &v) {
    const uint32_t b = bf16_of(v);
    const float r = v - bf16_value(b);
    v = fabsf(r) < INFINITY ? r : 0.f;
    return b;
}

// One 16-byte global -> LDS load per lane: lane i writes LDS bytes [lds + 16 i, lds + 16 i + 16); `lds` must be
// wave-uniform.  Completion is tracked by hand with vmcnt (the compiler does not see these loads).
__device__ __forceinline__ void dma16(const void *gsrc, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "{m0}"(lds), "v"(gsrc) : "memory");
}

template <int N>
__device__ __forceinline__ void wait_vm() {
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// Wait until at most r * NPW of this wave's loads are in flight (r <= R).
template <int NPW, int R>
__device__ __forceinline__ void wait_stages(int r) {
    if constexpr (R == 0) {
        wait_vm<0>();
    } else {
        if (r >= R) wait_vm<R * NPW>();
        else wait_stages<NPW, R - 1>(r);
    }
}

__device__ const u32x4 kZeros = {0u, 0u, 0u, 0u};  // what a chunk behind the last k holds

// 16-byte slot of (row, k-chunk) in one LDS stage of 64 k.  The XOR spreads the 16
// rows of an operand read, and 16 consecutive lanes of a store pass, over the banks.
// B rows are read in another order: lane l of a pair of 16-column blocks takes
// column 8 (l / 4) + 4 b + l % 4 of block b, so that the products of both blocks
// give a lane 8 consecutive columns of one row.
__device__ __forceinline__ int swz_a(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int swz_b(int row) { return ((row >> 1) & 1) | (((row >> 3) & 3) << 1); }
__device__ __forceinline__ int pair_column(int lane, int nb) { return 32 * (nb >> 1) + 8 * ((lane & 15) >> 2) + 4 * (nb & 1) + (lane & 3); }

// Tile of workgroup blockIdx.x: groups of kGroup row tiles, row tile fastest, and each
// XCD (workgroups are dealt to the 8 XCDs in turn) a contiguous run of that order.
constexpr int kGroup = 8;
__device__ __forceinline__ void tile_of(int mtiles, int ntiles, int *mt, int *nt) {
    const int tiles = mtiles * ntiles, per = tiles >> 3;
    int t = blockIdx.x;
    if (t < per * 8) t = (t & 7) * per + (t >> 3);
    const int g = t / (kGroup * ntiles), first = g * kGroup, gm = min(kGroup, mtiles - first), r = t - g * kGroup * ntiles;
    *mt = first + r % gm;
    *nt = r / gm;
}

// Eight consecutive columns of a row.
template <int EPI>
__device__ __forceinline__ void store_eight(const GemmArgs &g, f32x4 x, f32x4 y, int row, int n) {
    const size_t at = (size_t)row * g.N + n;
    if constexpr (EPI == kStoreF32) {
        f32x4 *dst = reinterpret_cast<f32x4 *>(static_cast<float *>(g.out) + at);
        dst[0] = x;
        dst[1] = y;
    } else {
        *reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(g.out) + at) =
            u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(y[0], y[1]), pack2(y[2], y[3])};
    }
}
__device__ __forceinline__ void store_h(const GemmArgs &g, f32x4 g0, f32x4 g1, f32x4 u0, f32x4 u1, int row, int n) {
    float h[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[i] = gated(g0[i], u0[i]);
        h[4 + i] = gated(g1[i], u1[i]);
    }
    uint16_t *dst = static_cast<uint16_t *>(g.out) + (size_t)row * g.N + n;
    for (int p = 0; p < g.h_planes; ++p, dst += (size_t)g.M * g.N) {
        u32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t lo = next_plane(h[2 * k]), hi = next_plane(h[2 * k + 1]);
            v[k] = lo | (hi << 16);
        }
        *reinterpret_cast<u32x4 *>(dst) = v;
    }
}

// BM x BN tile on WR x WC waves, K in stages of 64 through a ring of D LDS stages
// that direct global -> LDS loads fill ahead.  4-bit weights pass through registers,
// a stage ahead.  With kGate the BN weight rows are, for each column of waves, 32
// rows of the gate and the same 32 of the up projection, so that a lane ends up with
// both products of its columns.
template <int BM, int BN, int D, int WR, int WC, bool FOUR, int EPI>
__global__ __launch_bounds__(64 * WR * WC) void tile_kernel(const GemmArgs g) {
    constexpr int NT = 64 * WR * WC, NW = WR * WC;
    constexpr int STAGE = (BM + BN) * 8;                       // 16-byte slots per stage
    constexpr int LOADED = FOUR ? BM * 8 : STAGE;              // those that direct loads fill
    constexpr int NPW = LOADED / 64 / NW;                      // loads per wave per stage
    constexpr int WM = BM / WR, MB = WM / 16, WN = BN / WC, NB = WN / 16;
    static_assert(LOADED % NT == 0 && WN == 64 && MB >= 1 && NB == 4, "shape");
    static_assert(!FOUR || BN * 2 == NT, "one group of codes a thread and stage");
    __shared__ __attribute__((aligned(1024))) u32x4 ring[D * STAGE];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    constexpr int COLS = EPI == kGate ? BN / 2 : BN;           // output columns of a tile
    int mt, nt;
    tile_of((g.M + BM - 1) / BM, (g.N + COLS - 1) / COLS, &mt, &nt);
    const int m0 = mt * BM, n0 = nt * COLS;
    const int nk = (g.K + kBK - 1) / kBK, stages = nk * g.a_planes;

    // weight row of the tile's B row rb: (second matrix?, row); rows past the end repeat the last, never stored
    const auto weight_row = [&](int rb, bool *second) {
        *second = EPI == kGate && (rb & 32) != 0;
        return min(n0 + (EPI == kGate ? (rb >> 6) * 32 + (rb & 31) : rb), g.N - 1);
    };
    const uint16_t *src[NPW];
#pragma unroll
    for (int i = 0; i < NPW; ++i) {
        const int s = (wave * NPW + i) * 64 + lane, row = s >> 3;
        if (row < BM) {
            src[i] = g.a + (size_t)min(m0 + row, g.M - 1) * g.K + ((s & 7) ^ swz_a(row)) * 8;
        } else {
            bool second;
            const size_t n = weight_row(row - BM, &second);
            src[i] = (second ? g.up.w : g.b.w) + n * g.K + ((s & 7) ^ swz_b(row)) * 8;
        }
    }
    const uint32_t ring_lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ring));
    const size_t plane = (size_t)g.M * g.K;
    const auto issue = [&](int st) {
        const int p = st / nk, k0 = (st - p * nk) * kBK;
        const uint32_t dst = ring_lds + (uint32_t)((st % D) * STAGE * 16 + wave * NPW * 1024);
        const bool tail = k0 + kBK > g.K;
#pragma unroll
        for (int i = 0; i < NPW; ++i) {
            const int s = (wave * NPW + i) * 64 + lane, row = s >> 3;
            const void *from = src[i] + k0 + (row < BM ? p * plane : 0);
            if (tail && k0 + ((s & 7) ^ (row < BM ? swz_a(row) : swz_b(row))) * 8 >= g.K) from = &kZeros;
            dma16(from, __builtin_amdgcn_readfirstlane(dst + i * 1024));
        }
    };
    // 4-bit weights: thread t holds group t % 2 of B row t / 2
    const uint8_t *codes = nullptr, *scales = nullptr;
    if constexpr (FOUR) {
        bool second;
        const size_t n = weight_row(tid >> 1, &second);
        codes = (second ? g.up.codes : g.b.codes) + n * (g.K / 2) + (tid & 1) * 16;
        scales = (second ? g.up.scales : g.b.scales) + n * (g.K / kMxGroup) + (tid & 1);
    }
    u32x4 held = {0u, 0u, 0u, 0u};
    uint32_t held_scale = 0u;
    const auto load_codes = [&](int st) {
        const int k0 = st % nk * kBK;
        const bool in = k0 + (tid & 1) * kMxGroup < g.K;
        held = in ? *reinterpret_cast<const u32x4 *>(codes + k0 / 2) : u32x4{0u, 0u, 0u, 0u};
        held_scale = in ? scales[k0 / kMxGroup] : 0u;
    };
    const auto put_codes = [&](int st) {
        u32x4 *const to = ring + (st % D) * STAGE;
        const int row = BM + (tid >> 1);
        const float s = mx_scale(held_scale);
#pragma unroll
        for (int c = 0; c < 4; ++c) to[row * 8 + (((tid & 1) * 4 + c) ^ swz_b(row))] = mx_values(held[c], s);
    };

    f32x4 acc[MB][NB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int wr = (wave / WC) * WM, wc = BM + (wave % WC) * WN;

    if constexpr (FOUR) {
        load_codes(0);
        put_codes(0);
    }
#pragma unroll
    for (int st = 0; st < D - 1; ++st)
        if (st < stages) issue(st);
    for (int kt = 0; kt < stages; ++kt) {
        if (kt + D - 1 < stages) issue(kt + D - 1);
        // stage kt has landed once no more than the stages issued after it are in flight
        wait_stages<NPW, D - 1>(min(D - 1, stages - 1 - kt));
        __syncthreads();
        if (FOUR && kt + 1 < stages) load_codes(kt + 1);
        const u32x4 *cur = ring + (kt % D) * STAGE;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int kc = s * 4 + (lane >> 4);
            u32x4 fa[MB], fb[NB];
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                const int row = wr + mb * 16 + (lane & 15);
                fa[mb] = cur[row * 8 + (kc ^ swz_a(row))];
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int row = wc + pair_column(lane, nb);
                fb[nb] = cur[row * 8 + (kc ^ swz_b(row))];
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = mfma(fb[nb], fa[mb], acc[mb][nb]);
        }
        if (FOUR && kt + 1 < stages) put_codes(kt + 1);
        __syncthreads();  // the slot of stage kt is refilled by the next iteration's loads
    }

    // acc[mb][2 p + b][i] = C[16 mb + lane % 16][32 p + 8 (lane / 16) + 4 b + i]
    const int cw = n0 + (wave % WC) * (EPI == kGate ? 32 : 64) + 8 * (lane >> 4);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int row = m0 + wr + mb * 16 + (lane & 15);
        if (row >= g.M) continue;
        if constexpr (EPI == kGate) {
            if (cw < g.N) store_h(g, acc[mb][0], acc[mb][1], acc[mb][2], acc[mb][3], row, cw);
        } else {
#pragma unroll
            for (int p = 0; p < NB / 2; ++p)
                if (cw + 32 * p < g.N) store_eight<EPI>(g, acc[mb][2 * p], acc[mb][2 * p + 1], row, cw + 32 * p);
        }
    }
}

template <int BM, int BN, int D, int WR, int WC, bool FOUR>
hipError_t launch_tiles(const GemmArgs &g, Epilogue epi, hipStream_t s) {
    const int cols = epi == kGate ? BN / 2 : BN;
    const long long tiles = (long long)((g.M + BM - 1) / BM) * ((g.N + cols - 1) / cols);
    if (tiles > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)tiles);
    constexpr int NT = 64 * WR * WC;
    if (epi == kStoreBf16) tile_kernel<BM, BN, D, WR, WC, FOUR, kStoreBf16><<<grid, NT, 0, s>>>(g);
    else if (epi == kStoreF32) tile_kernel<BM, BN, D, WR, WC, FOUR, kStoreF32><<<grid, NT, 0, s>>>(g);
    else tile_kernel<BM, BN, D, WR, WC, FOUR, kGate><<<grid, NT, 0, s>>>(g);
    return hipGetLastError();
}

template <bool FOUR>
hipError_t launch_shape(const GemmArgs &g, Epilogue epi, const Shape &t, hipStream_t s) {
    if (t.bm == 256 && t.bn == 256) return launch_tiles<256, 256, 2, 2, 4, FOUR>(g, epi, s);
    if (t.bm == 128 && t.bn == 128) return launch_tiles<128, 128, 2, 2, 2, FOUR>(g, epi, s);
    if (t.bm == 64 && t.bn == 128) return launch_tiles<64, 128, 3, 2, 2, FOUR>(g, epi, s);
    if (t.bm == 32 && t.bn == 128) return launch_tiles<32, 128, 4, 2, 2, FOUR>(g, epi, s);
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_gemm(const GemmArgs &g, bool four_bit, Epilogue epi, const Shape &t, hipStream_t s) {
    if (g.M <= 0) return hipSuccess;
    if (g.N <= 0 || g.N % 8 != 0 || g.K <= 0 || g.K % (four_bit ? kMxGroup : 8) != 0 || g.a_planes < 1) return hipErrorInvalidValue;
    return four_bit ? launch_shape<true>(g, epi, t, s) : launch_shape<false>(g, epi, t, s);
}

}  // namespace ffn
