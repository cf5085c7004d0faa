// Feed-forward kernels for gfx950: products of bf16 rows with bf16 or 4-bit
// weights, and the gated first half of the block.  Host-side contracts are in
// include/mla_ffn.h.
//
// Every product is out = A . B^T with both operands K-contiguous, on bf16 MFMA
// 16x16x32 with fp32 sums, taken as B . A^T so that a lane holds neighbouring
// columns of one row.  4-bit weights become bf16 on the way (exactly, scale
// included, two an instruction), so both formats share the products.
#include "ffn_kernels.h"

#include <type_traits>

namespace ffn {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));

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

// h = silu(g) u = g u / (1 + exp(-g)), silu off by less than 2^-21 of itself where exp(-g) is a number, down to g = -88.72:
// exp(-g) as 2^(-g log2 e) with the product's own rounding put back, then the hardware's reciprocal (1 ulp).  That gives
// no subnormal numbers, so it takes a quarter of the sum, which stays below 2^126, and a quarter of g (whose last bits count
// below 2^-124 alone, 2^-149 of the result).  Further down exp(-g) is infinite and silu, less than 2^-121, is -0; from 200 on
// silu is g.  (The library's expf and division: a sixth of a 256 x 256 tile's time, 9 of 57 us.)
__device__ __forceinline__ float gated(float g, float u) {
    constexpr float kLog2e = 1.44269502f, kLog2eRest = 1.92596303e-8f, kLn2 = 0.693147182f;
    const float c = __builtin_amdgcn_fmed3f(g, -200.f, 200.f), t = c * kLog2e;
    const float rest = __builtin_fmaf(c, kLog2e, -t) + c * kLog2eRest;
    const float e = __builtin_amdgcn_exp2f(-t);
    return .25f * g * __builtin_amdgcn_rcpf(.25f + e * (.25f - rest * (.25f * kLn2))) * u;
}

// h as the sum of three bf16 values of one sign, most significant first: h itself from 2^-110 on, below that the nearest
// multiple of kLeast = 2^-133, the least bf16.  None is zero unless h is, so that an infinite weight, or an infinite h, makes
// a sum infinite as it should and not inf - inf or 0 inf.  So the first two leave `room` for each one behind them: h's last
// bit, at least kLeast.  Then the first leaves at most 2^16 + 1 of h's last bits and the second at most 2^8, which the third
// holds; every partial sum is a multiple of that bit, and exact in fp32.  A nonzero h counts as 3 kLeast at least.
// (Planes filled up with kLeast, which the others did not make room for, put h off by up to 2 kLeast: 1.6 % at 2^-126.)
constexpr float kLeast = 0x1p-133f;
__device__ __forceinline__ float least_plane(float h) { return h != 0.f ? kLeast : 0.f; }
__device__ __forceinline__ float plane_room(float h, float least) { return fmaxf(__uint_as_float(__float_as_uint(h) & 0x7f800000u) * 0x1p-23f, least); }
// One of the first two of v = |h| or what the one before left, and v what it leaves.  (Of an infinite v the largest number,
// and v stays as it is; so does a NaN.)
__device__ __forceinline__ uint32_t next_plane(float &v, float room, float least) {
    const float most = fminf(v - room, 3.40282347e38f);  // negative where v < room
    const int b = max((int)__float_as_uint(most) >> 16, (int)__float_as_uint(least) >> 16);
    v -= bf16_value((uint32_t)b);
    return (uint32_t)b;
}
// N values h, in pairs, as the P-th plane takes them; `v` holds |h| before the first.
template <int P, int N>
__device__ __forceinline__ void plane_of(uint32_t (&to)[N / 2], const float (&h)[N], float (&v)[N]) {
    uint32_t b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float least = least_plane(h[i]);
        b[i] = P < 2 ? next_plane(v[i], (2 - P) * plane_room(h[i], least), least) : bf16_of(v[i] < least ? least : v[i]);
        b[i] |= __float_as_uint(h[i]) >> 16 & 0x8000u;
    }
#pragma unroll
    for (int k = 0; k < N / 2; ++k) to[k] = b[2 * k] | (b[2 * k + 1] << 16);
}

// A wave-uniform pointer, in scalar registers.
template <class T>
__device__ __forceinline__ const T *uniform(const T *p) {
    const uint64_t b = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<const T *>((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(b >> 32)) << 32 |
                                       (uint32_t)__builtin_amdgcn_readfirstlane((int)b));
}

// One 16-byte global -> LDS load per lane: lane i writes LDS bytes [lds + 16 i, lds + 16 i + 16); `lds` must be
// wave-uniform.  Completion is tracked by hand with vmcnt (the compiler does not see these loads).
__device__ __forceinline__ void dma16(const void *gsrc, uint32_t lds) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "{m0}"(lds), "v"(gsrc) : "memory");
}

// The same from base + off (base wave-uniform).  Where a vector instruction has written the base's registers (readfirstlane),
// five wait states have to pass before a vector load reads them; the compiler does not look inside and places none.
__device__ __forceinline__ void dma16_at(uint32_t off, const void *base, uint32_t lds) {
    asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" : : "{m0}"(__builtin_amdgcn_readfirstlane(lds)), "v"(off), "s"(uniform(static_cast<const char *>(base))) : "memory");
}
// Ends a half phase: nothing moves across, and no wait beside those written out.
__device__ __forceinline__ void half_phase() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" : : : "memory");
    __builtin_amdgcn_sched_barrier(0);
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

// Place of workgroup b in an order of n: workgroups are dealt to the 8 XCDs in turn, and each
// XCD gets a contiguous run of the order.
__device__ __forceinline__ int xcd_run(int b, int n) {
    const int per = n >> 3;
    return b < per * 8 ? (b & 7) * per + (b >> 3) : b;
}
// The tile at place t: groups of kGroup row tiles, row tile fastest, so that a run covers a block of
// about 8 x 4 tiles whose rows and weights stay in its XCD's L2.
constexpr int kGroup = 8;
__device__ __forceinline__ void tile_at(int t, int mtiles, int ntiles, int *mt, int *nt) {
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
    if (g.h_planes == 1) {  // rounded to nearest
        *reinterpret_cast<u32x4 *>(dst) = u32x4{pack2(h[0], h[1]), pack2(h[2], h[3]), pack2(h[4], h[5]), pack2(h[6], h[7])};
        return;
    }
    float v[8];
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fabsf(h[i]);
    const size_t plane = (size_t)g.plane_rows * g.N;
    plane_of<0>(b, h, v);
    *reinterpret_cast<u32x4 *>(dst) = u32x4{b[0], b[1], b[2], b[3]};
    plane_of<1>(b, h, v);
    *reinterpret_cast<u32x4 *>(dst + plane) = u32x4{b[0], b[1], b[2], b[3]};
    plane_of<2>(b, h, v);
    *reinterpret_cast<u32x4 *>(dst + 2 * plane) = u32x4{b[0], b[1], b[2], b[3]};
}

// Split sums.  Parts meet in memory; the XCDs do not share their L2 caches.  THROUGH: they are written and read as
// device-wide atomics, past the L2s, at 4 TB/s for the whole chip, and counted with a relaxed one.  That order is the
// instructions', not the language's (a release would write back the L2, which this is to avoid): vmcnt counts a device-wide
// store once every XCD sees it, all waves have waited for theirs when the counter is raised, and a device-wide load takes
// nothing from a cache that others do not see.  Otherwise the parts are stored as plain values, and a workgroup writes
// back what its L2 holds before it is counted (some 3 us, more with more of them).  So small tiles go through (a row of
// K = 10944 in 4 bits 10.6 -> 7.3 us, 16 rows in bf16 19.3 -> 13.7), those of 4-bit weights with 64 KB a part and the
// tiles for many rows do not (1500 rows, parts of 256 KB: 102 against 116 us).
template <bool THROUGH>
__device__ __forceinline__ void put_part(f32x4 *to, f32x4 v) {
    if constexpr (THROUGH) {
        const u64x2 w = __builtin_bit_cast(u64x2, v);
        uint64_t *const p = reinterpret_cast<uint64_t *>(to);
        __hip_atomic_store(p, w[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(p + 1, w[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    } else {
        *to = v;
    }
}
template <bool THROUGH>
__device__ __forceinline__ f32x4 get_part(const f32x4 *from) {
    if constexpr (THROUGH) {
        const uint64_t *const p = reinterpret_cast<const uint64_t *>(from);
        return __builtin_bit_cast(f32x4, u64x2{__hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT),
                                               __hip_atomic_load(p + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)});
    } else {
        return *from;
    }
}
// Every workgroup of a tile has put its part: true in all threads of the one that comes last, which then gets those of
// the others.  The counter is left as it was found, zero.
template <bool THROUGH>
__device__ __forceinline__ bool last_of_tile(uint32_t *counter, int splits) {
    __shared__ bool last;
    // each wave waits for its own stores, which have then arrived: THROUGH in memory, else in the L2 that the release writes back
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        const uint32_t before = __hip_atomic_fetch_add(counter, 1u, THROUGH ? __ATOMIC_RELAXED : __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        last = before == (uint32_t)splits - 1;
        if (last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(last);  // one branch for the whole wave
}

// sums[b] = the parts' b-th values, part 0 first: the order, and so the result, is the same whoever comes last.  Four
// parts of eight values are in flight at a time; one after the other, each would cost a trip to memory (one CU reads
// some 60 GB/s: the 16 parts of a 64 x 128 tile, half a megabyte, take it 9 us).
template <bool THROUGH, int N>
__device__ __forceinline__ void join_parts(f32x4 (&sums)[N], const f32x4 *parts, size_t stride, int splits) {
    constexpr int C = N < 8 ? N : 8;
    static_assert(N % C == 0, "whole chunks");
#pragma unroll
    for (int b0 = 0; b0 < N; b0 += C) {
        for (int z = 0; z < splits; z += 4) {
            f32x4 v[4][C];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int b = 0; b < C; ++b) v[i][b] = get_part<THROUGH>(parts + (size_t)min(z + i, splits - 1) * stride + (b0 + b) * 64);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (z + i < splits) {
#pragma unroll
                    for (int b = 0; b < C; ++b) sums[b0 + b] = z + i == 0 ? v[i][b] : sums[b0 + b] + v[i][b];
                }
        }
    }
}

// Four consecutive columns of a row.
template <int EPI>
__device__ __forceinline__ void store_four(const GemmArgs &g, f32x4 v, int row, int n) {
    const size_t at = (size_t)row * g.N + n;
    if constexpr (EPI == kStoreF32)
        *reinterpret_cast<f32x4 *>(static_cast<float *>(g.out) + at) = v;
    else
        *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(g.out) + at) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
}
__device__ __forceinline__ void store_h4(const GemmArgs &g, f32x4 gate, f32x4 up, int row, int n) {
    float h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = gated(gate[i], up[i]);
    uint16_t *dst = static_cast<uint16_t *>(g.out) + (size_t)row * g.N + n;
    if (g.h_planes == 1) {
        *reinterpret_cast<u32x2 *>(dst) = u32x2{pack2(h[0], h[1]), pack2(h[2], h[3])};
        return;
    }
    float v[4];
    uint32_t b[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = fabsf(h[i]);
    const size_t plane = (size_t)g.plane_rows * g.N;
    plane_of<0>(b, h, v);
    *reinterpret_cast<u32x2 *>(dst) = u32x2{b[0], b[1]};
    plane_of<1>(b, h, v);
    *reinterpret_cast<u32x2 *>(dst + plane) = u32x2{b[0], b[1]};
    plane_of<2>(b, h, v);
    *reinterpret_cast<u32x2 *>(dst + 2 * plane) = u32x2{b[0], b[1]};
}

// Few rows: the call is bound by reading the weights once, so they go straight from
// memory to registers.  A workgroup takes 16 MB rows and CB blocks of 16 weight rows
// (kGate: the first half gate, the second the same columns of up; half and half of a
// single block); its eight waves share K in slices of 128, a slice ahead in registers,
// and meet in LDS.  Within a slice a lane holds 32 neighbouring k of its row (lane / 16
// picks which), 64 bytes in bf16 or 16 in 4 bits under one scale; the products' order of
// k is that of both operands, so nothing is moved.  The P planes of x meet a weight where
// it is loaded.  gridDim.z cuts K further where the columns are too few for the chip.
//   One block a workgroup is twice as many of them: 2048 x 2048 in 4 bits, one row 4.9 ->
// 3.9 us (2.4 an empty launch), gate and up of 4 x 1408 in bf16 7.3 -> 5.7 (2.0 TB/s);
// two read x half as often: 16 rows of 10944 columns in 4 bits 19.4 against 14.4.  Of many
// columns they read 4.3 to 4.9 TB/s in bf16 (K = 2048, 10944 columns of gate and up).
template <int MB, int CB, bool FOUR, int EPI, int P>
__global__ __launch_bounds__(512) void rows_kernel(const GemmArgs g) {
    constexpr bool kHalves = EPI == kGate && CB == 1;  // rows 0 .. 7 of the block gate, 8 .. 15 the same columns of up
    constexpr int NB = FOUR ? 1 : 4, JB = EPI == kGate && !kHalves ? CB / 2 : CB, UNITS = MB * JB, COLS = kHalves ? 8 : 16 * JB;
    __shared__ f32x4 red[4][MB * CB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), grp = lane >> 4;
    const int n0 = blockIdx.x * COLS, m0 = blockIdx.y * 16 * MB;
    const int total = (g.K + 127) >> 7, step = 8 * g.splits;
    const size_t plane = (size_t)g.plane_rows * g.K;

    const uint16_t *arow[MB], *brow[CB];
    const uint8_t *crow[CB], *srow[CB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) arow[mb] = g.a + (size_t)min(m0 + 16 * mb + (lane & 15), g.M - 1) * g.K;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {  // columns past the end repeat the last one, never stored
        const Weights &w = (kHalves ? (lane & 8) != 0 : EPI == kGate && cb >= JB) ? g.up : g.b;
        const size_t n = min(n0 + 16 * (cb % JB) + (lane & (kHalves ? 7 : 15)), g.N - 1);
        if constexpr (FOUR) {
            crow[cb] = w.codes + n * (g.K / 2);
            srow[cb] = w.scales + n * (g.K / kMxGroup);
        } else {
            brow[cb] = w.w + n * g.K;
        }
    }
    // k of the lane's chunk i: with 4-bit weights 32 neighbouring k, as their codes are loaded; in bf16 the four lanes of a row
    // take 64 neighbouring bytes at a time
    const auto at_k = [&](int k0, int i) { return k0 + (FOUR ? 32 * grp + 8 * i : 32 * i + 8 * grp); };
    struct Slice {
        u32x4 b[CB][NB], a[P][MB][4];
        uint32_t scale[CB];
    };
    // chunks behind the last k are read from the row's start, and dropped in use()
    const auto load = [&](Slice &s, int j) {
        const int k0 = j * 128;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            if constexpr (FOUR) {
                const int k = k0 + 32 * grp, at = k < g.K ? k : 0;
                s.b[cb][0] = *reinterpret_cast<const u32x4 *>(crow[cb] + at / 2);
                s.scale[cb] = srow[cb][at / kMxGroup];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) s.b[cb][i] = *reinterpret_cast<const u32x4 *>(brow[cb] + (at_k(k0, i) < g.K ? at_k(k0, i) : 0));
            }
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 4; ++i) s.a[p][mb][i] = *reinterpret_cast<const u32x4 *>(arow[mb] + p * plane + (at_k(k0, i) < g.K ? at_k(k0, i) : 0));
    };
    f32x4 acc[MB][CB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) acc[mb][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
    const auto use = [&](Slice &s, int j) {
        const int k0 = j * 128;
        if (k0 + 128 > g.K) {
            const u32x4 zero = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = at_k(k0, i) < g.K;
#pragma unroll
                for (int b = 0; b < P * MB; ++b) s.a[b / MB][b % MB][i] = in ? s.a[b / MB][b % MB][i] : zero;
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    if constexpr (!FOUR) s.b[cb][i] = in ? s.b[cb][i] : zero;
                    else if (i == 0) {
                        s.b[cb][0] = in ? s.b[cb][0] : zero;
                        s.scale[cb] = in ? s.scale[cb] : 0u;
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                u32x4 b;
                if constexpr (FOUR) b = mx_values(s.b[cb][0][i], mx_scale(s.scale[cb]));
                else b = s.b[cb][i];
#pragma unroll
                for (int m = 0; m < P * MB; ++m) acc[m % MB][cb] = mfma(b, s.a[m / MB][m % MB][i], acc[m % MB][cb]);
            }
        }
    };
    Slice s0, s1;
    int j = blockIdx.z * 8 + wave;
    if (j < total) load(s0, j);
    while (j < total) {
        if (j + step < total) load(s1, j + step);
        use(s0, j);
        if ((j += step) >= total) break;
        if (j + step < total) load(s0, j + step);
        use(s1, j);
        j += step;
    }

    // the eight waves' sums: (w, w + 4), then 0 .. 3 in order
    if (wave >= 4) {
#pragma unroll
        for (int b = 0; b < MB * CB; ++b) red[wave - 4][b][lane] = acc[b / CB][b % CB];
    }
    __syncthreads();
    if (wave < 4) {
#pragma unroll
        for (int b = 0; b < MB * CB; ++b) red[wave][b][lane] += acc[b / CB][b % CB];
    }
    __syncthreads();
    const int tile = blockIdx.y * gridDim.x + blockIdx.x;
    f32x4 *const parts = reinterpret_cast<f32x4 *>(g.parts) + (size_t)tile * g.splits * (MB * CB * 64) + lane;
    const auto block_sum = [&](int b) { return red[0][b][lane] + red[1][b][lane] + red[2][b][lane] + red[3][b][lane]; };
    if (g.splits > 1) {
        for (int b = wave; b < MB * CB; b += 8) put_part<true>(parts + ((size_t)blockIdx.z * (MB * CB) + b) * 64, block_sum(b));
        if (!last_of_tile<true>(g.counters + tile, g.splits)) return;
    }
    const auto total_sum = [&](int b) {
        if (g.splits == 1) return block_sum(b);
        f32x4 v[1];
        join_parts<true>(v, parts + (size_t)b * 64, MB * CB * 64, g.splits);
        return v[0];
    };
    // D[16 mb + lane % 16][16 jb + 4 (lane / 16) + i]
    for (int u = wave; u < UNITS; u += 8) {
        const int mb = u / JB, jb = u % JB, row = m0 + 16 * mb + (lane & 15), n = n0 + 16 * jb + 4 * grp;
        const f32x4 v = total_sum(mb * CB + jb);
        if constexpr (kHalves) {
            f32x4 up;
#pragma unroll
            for (int i = 0; i < 4; ++i) up[i] = __shfl(v[i], lane ^ 32);
            if (row < g.M && grp < 2) store_h4(g, v, up, row, n);
        } else if constexpr (EPI == kGate) {
            const f32x4 up = total_sum(mb * CB + JB + jb);
            if (row < g.M && n < g.N) store_h4(g, v, up, row, n);
        } else {
            if (row < g.M && n < g.N) store_four<EPI>(g, v, row, n);
        }
    }
}

// A middling number of rows: bound by the weights, which go straight from memory to
// registers as above, or by the products.  WC waves share the rows of x through LDS
// (slices of 128 SL k, one ahead: loaded to registers before a slice's products, stored
// to the other buffer after them) and take CB blocks of 16 weight rows each (kGate:
// the first half gate, the second the same columns of up); KG such groups take K's
// slices in turn and meet in LDS.  gridDim.z cuts K further.
//   Four groups make a short chain where columns are few (48 rows of 2 x 5504 columns, K =
// 2048: 12.9 us, 0.9 TB/s; 64 rows of 5000: 12.9), eight waves side by side read x least
// where they are many (32 rows of 102400 columns: 33 us from the L2s and the memory-side
// cache, 40 from memory, 2.8 TB/s), and 64 x 128 tiles carry up to some 2000 rows (2048 x
// 2048 of K = 5504: 53 us, 870 TFLOP/s).  The chain of a slice bounds it: its rows through
// LDS, 32 conversions a block, then the products.  Planes of x follow each other as a longer
// K, so a weight is loaded and converted once for each of them.
template <int MB, int CB, int WC, int KG, int SL, int EPI>
__global__ __launch_bounds__(64 * WC * KG) void mid_kernel(const GemmArgs g) {
    constexpr int JB = EPI == kGate ? CB / 2 : CB, COLS = 16 * JB * WC;
    constexpr bool kThrough = MB * CB * WC < 64;
    constexpr int CH = 16 * SL;                     // 16-byte chunks of a row's slice
    constexpr int BUF = MB * 16 * CH;               // and of one buffer
    constexpr int LPT = (BUF + 64 * WC - 1) / (64 * WC);
    static_assert(BUF % (64 * WC) == 0 || LPT == 1, "loads of a slice");
    static_assert(KG == 1 || KG * 2 * BUF >= (KG / 2) * WC * MB * CB * 64, "partial sums fit the buffers");
    __shared__ u32x4 sm[KG * 2 * BUF];
    const int tid = threadIdx.x, lane = tid & 63, grp = lane >> 4, l16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wc = wave % WC, kg = wave / WC, gt = tid % (64 * WC);
    int mt, nt;
    tile_at(xcd_run(blockIdx.x, gridDim.x), (g.M + 16 * MB - 1) / (16 * MB), (g.N + COLS - 1) / COLS, &mt, &nt);
    const int m0 = mt * 16 * MB, n0 = nt * COLS + wc * 16 * JB;
    const int ns = (g.K + 128 * SL - 1) / (128 * SL), total = ns * g.a_planes;
    const int j0 = (int)((long long)total * blockIdx.z / g.splits), j1 = (int)((long long)total * (blockIdx.z + 1) / g.splits);
    const int rounds = (j1 - j0 + KG - 1) / KG;
    const size_t plane = (size_t)g.plane_rows * g.K;
    u32x4 *const buf = sm + kg * 2 * BUF;

    // column of block jb that lane l16 loads: pairs of blocks are interleaved (pair_column) so that a lane ends up with 8
    // neighbouring columns
    const auto column = [&](int jb) { return JB % 2 == 0 ? pair_column(lane, jb) : 16 * jb + l16; };
    const uint8_t *crow[CB], *srow[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const Weights &w = EPI == kGate && cb >= JB ? g.up : g.b;
        const size_t n = min(n0 + column(cb % JB), g.N - 1);
        crow[cb] = w.codes + n * (g.K / 2);
        srow[cb] = w.scales + n * (g.K / kMxGroup);
    }
    const uint16_t *arow[LPT];
#pragma unroll
    for (int i = 0; i < LPT; ++i) arow[i] = g.a + (size_t)min(m0 + min((gt + 64 * WC * i) / CH, 16 * MB - 1), g.M - 1) * g.K;

    // Place of a row's chunk 4 SL q + i (the i-th that lanes of quarter q multiply), before the XOR with the row.  A read of 16
    // bytes a lane is served 16 lanes at a time, rows 0 .. 3 and 12 .. 15 of one quarter with rows 4 .. 11 of the next: the
    // quarters of such a pair differ in the lowest bit, so that the XOR leaves them apart (as their chunks lie in memory: 8
    // cycles a read for 4).
    const auto place = [](int q, int i) { return (q & 1) + 2 * i + 8 * SL * (q >> 1); };
    u32x4 areg[LPT];
    const auto load_a = [&](int j) {
        const int p = j / ns, k = (j - p * ns) * (128 * SL) + gt % CH * 8;
#pragma unroll
        for (int i = 0; i < LPT; ++i) areg[i] = *reinterpret_cast<const u32x4 *>(arow[i] + p * plane + (k < g.K ? k : 0));
    };
    const auto put_a = [&](int j, u32x4 *to) {
        const bool in = j % ns * (128 * SL) + gt % CH * 8 < g.K;
#pragma unroll
        for (int i = 0; i < LPT; ++i) {
            const int row = (gt + 64 * WC * i) / CH;
            if (BUF % (64 * WC) == 0 || row < 16 * MB) to[row * CH + (place(gt % CH / (4 * SL), gt % (4 * SL)) ^ (row & 15))] = in ? areg[i] : u32x4{0u, 0u, 0u, 0u};
        }
    };
    // a lane's SL groups of a slice are neighbours, as its codes are loaded; behind the last k they are read from the row's
    // start, and dropped in use()
    struct Slice {
        u32x4 codes[CB][SL];
        uint32_t scales[CB];
    };
    const auto load_b = [&](Slice &s, int j) {
        const int k = j % ns * (128 * SL) + 32 * SL * grp;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
#pragma unroll
            for (int t = 0; t < SL; ++t) s.codes[cb][t] = *reinterpret_cast<const u32x4 *>(crow[cb] + (k + 32 * t < g.K ? k + 32 * t : 0) / 2);
            const uint8_t *const from = srow[cb] + (k < g.K ? k : 0) / kMxGroup;
            if (SL == 1 || k + 32 >= g.K) {
                s.scales[cb] = *from;
            } else {
                uint16_t two;
                __builtin_memcpy(&two, from, 2);
                s.scales[cb] = two;
            }
        }
    };
    f32x4 acc[MB][CB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) acc[mb][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
    const auto use = [&](Slice &s, int j, const u32x4 *from) {
        const int k0 = j % ns * (128 * SL);
        if (k0 + 128 * SL > g.K) {  // groups behind the last k count as zeros, on both sides
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int t = 0; t < SL; ++t)
                    if (k0 + 32 * (SL * grp + t) >= g.K) {
                        s.codes[cb][t] = u32x4{0u, 0u, 0u, 0u};
                        s.scales[cb] &= ~(0xffu << (8 * t));
                    }
        }
#pragma unroll
        for (int i = 0; i < 4 * SL; ++i) {
            u32x4 fa[MB];
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) fa[mb] = from[(16 * mb + l16) * CH + (place(grp, i) ^ l16)];
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                const u32x4 b = mx_values(s.codes[cb][i / 4][i % 4], mx_scale((s.scales[cb] >> (i / 4 * 8)) & 0xffu));
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) acc[mb][cb] = mfma(b, fa[mb], acc[mb][cb]);
            }
        }
    };
    Slice s0, s1;
    int j = j0 + kg;
    if (j < j1) {
        load_a(j);
        load_b(s0, j);
        put_a(j, buf);
    }
    __syncthreads();
    const auto round = [&](Slice &now, Slice &next, u32x4 *from, u32x4 *to) {
        if (j + KG < j1) {
            load_a(j + KG);
            load_b(next, j + KG);
        }
        if (j < j1) use(now, j, from);
        if (j + KG < j1) put_a(j + KG, to);
        __syncthreads();
        j += KG;
    };
    for (int r = 0; r < rounds; r += 2) {
        round(s0, s1, buf, buf + BUF);
        if (r + 1 < rounds) round(s1, s0, buf + BUF, buf);
    }

    // the groups' sums, halved in order
    if constexpr (KG > 1) {
        f32x4 *const part = reinterpret_cast<f32x4 *>(sm);
#pragma unroll
        for (int half = KG / 2; half >= 1; half /= 2) {
            if (kg >= half && kg < 2 * half) {
#pragma unroll
                for (int b = 0; b < MB * CB; ++b) part[(((kg - half) * WC + wc) * MB * CB + b) * 64 + lane] = acc[b / CB][b % CB];
            }
            __syncthreads();
            if (kg < half) {
#pragma unroll
                for (int b = 0; b < MB * CB; ++b) acc[b / CB][b % CB] += part[((kg * WC + wc) * MB * CB + b) * 64 + lane];
            }
            if (half > 1) __syncthreads();
        }
    }
    if (g.splits > 1) {
        const int tile = nt * ((g.M + 16 * MB - 1) / (16 * MB)) + mt;
        constexpr int PART = WC * MB * CB * 64;
        f32x4 *const parts = reinterpret_cast<f32x4 *>(g.parts) + (size_t)tile * g.splits * PART + wc * MB * CB * 64 + lane;
        if (kg == 0) {
#pragma unroll
            for (int b = 0; b < MB * CB; ++b) put_part<kThrough>(parts + (size_t)blockIdx.z * PART + b * 64, acc[b / CB][b % CB]);
        }
        if (!last_of_tile<kThrough>(g.counters + tile, g.splits) || kg > 0) return;
        join_parts<kThrough>(reinterpret_cast<f32x4(&)[MB * CB]>(acc), parts, PART, g.splits);
    }
    if (kg > 0) return;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        const int row = m0 + 16 * mb + l16;
        if (row >= g.M) continue;
#pragma unroll
        for (int jb = 0; jb < JB; jb += JB % 2 == 0 ? 2 : 1) {
            if constexpr (JB % 2 == 0) {
                const int n = n0 + 16 * jb + 8 * grp;
                if (n >= g.N) continue;
                if constexpr (EPI == kGate) store_h(g, acc[mb][jb], acc[mb][jb + 1], acc[mb][JB + jb], acc[mb][JB + jb + 1], row, n);
                else store_eight<EPI>(g, acc[mb][jb], acc[mb][jb + 1], row, n);
            } else {
                const int n = n0 + 16 * jb + 4 * grp;
                if (n >= g.N) continue;
                if constexpr (EPI == kGate) store_h4(g, acc[mb][jb], acc[mb][JB + jb], row, n);
                else store_four<EPI>(g, acc[mb][jb], row, n);
            }
        }
    }
}

// A middling number of rows, bf16 weights: a BM x BN tile on WR x WC waves, K in stages of
// 64 through a ring of D LDS stages that direct global -> LDS loads fill ahead; all P planes
// of x are in a stage, so that the weights are loaded once (64 rows, K = 10944: 26 us, where
// planes one after the other as a longer K took 39).  A stage's operands are read while the
// products of the one before run, so that one barrier a stage is all that the waves wait
// for together: behind it a stage has landed for all of them and the slot of the one before
// is free.  With kGate the BN weight rows are, for each column of waves, 32 rows of the gate
// and the same 32 of the up projection, so that a lane ends up with both products of its
// columns.
//   The loads bound it: a CU takes 18 to 27 ns for each KB of them whatever else it does (a
// stage of 64 x 128: 24 KB, 0.48 us; deeper rings, loads through registers and loads between
// the products are no faster).  544 rows of 2 x 1368 columns, K = 2048: 18.4 us, 330 TFLOP/s.
template <int BM, int BN, int D, int WR, int WC, int EPI, int P>
__global__ __launch_bounds__(64 * WR * WC) void tile_kernel(const GemmArgs g) {
    constexpr int NW = WR * WC, AR = P * BM;
    constexpr int STAGE = (AR + BN) * 8;                      // 16-byte slots per stage
    constexpr int NPW = STAGE / 64 / NW;                      // loads per wave per stage
    constexpr int WM = BM / WR, MB = WM / 16, WN = BN / WC, NB = WN / 16;
    static_assert(STAGE % (64 * NW) == 0 && WN == 64 && MB >= 1 && NB == 4 && D >= 2, "shape");
    __shared__ __attribute__((aligned(1024))) u32x4 ring[D * STAGE];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    constexpr int COLS = EPI == kGate ? BN / 2 : BN;          // output columns of a tile
    int mt, nt;
    tile_at(xcd_run(blockIdx.x, gridDim.x), (g.M + BM - 1) / BM, (g.N + COLS - 1) / COLS, &mt, &nt);
    const int m0 = __builtin_amdgcn_readfirstlane(mt * BM), n0 = __builtin_amdgcn_readfirstlane(nt * COLS);
    const int all = (g.K + kBK - 1) / kBK;
    const int first = (int)((long long)all * blockIdx.z / g.splits), stages = (int)((long long)all * (blockIdx.z + 1) / g.splits) - first;

    // The wave's i-th load fills 8 neighbouring rows of x or the weights: the first one is wave-uniform.  Rows past the end
    // repeat the last one (the widths are multiples of 8: of weight rows all eight exist or none); never stored.
    const char *base[NPW];
    uint32_t off[NPW];
    int kin[NPW];
#pragma unroll
    for (int i = 0; i < NPW; ++i) {
        const int at = 8 * (wave * NPW + i), row = at + (lane >> 3);
        kin[i] = ((lane & 7) ^ (at < AR ? swz_a(row) : swz_b(row - AR))) * 8;
        if (at < AR) {
            const int r = min(m0 + at % BM, g.M - 1);
            base[i] = uniform(reinterpret_cast<const char *>(g.a + ((size_t)(at / BM) * g.plane_rows + r) * g.K));
            off[i] = (uint32_t)min(lane >> 3, g.M - 1 - r) * (uint32_t)g.K * 2u + (uint32_t)kin[i] * 2u;
        } else {
            const int rb = at - AR, n = min(n0 + (EPI == kGate ? (rb >> 6) * 32 + (rb & 31) : rb), g.N - 8);
            base[i] = uniform(reinterpret_cast<const char *>((EPI == kGate && (rb & 32) ? g.up.w : g.b.w) + (size_t)n * g.K));
            off[i] = (uint32_t)(lane >> 3) * (uint32_t)g.K * 2u + (uint32_t)kin[i] * 2u;
        }
    }
    const uint32_t ring_lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ring)) + wave * NPW * 1024;
    int k0 = first * kBK, slot_in = 0;  // of the stage to load next
    const auto issue = [&] {
        const uint32_t dst = ring_lds + (uint32_t)(slot_in * STAGE * 16);
        const bool whole = k0 + kBK <= g.K;
#pragma unroll
        for (int i = 0; i < NPW; ++i) {
            const char *const from = base[i] + (size_t)k0 * 2;
            if (whole) dma16_at(off[i], from, dst + i * 1024);
            else dma16(k0 + kin[i] < g.K ? from + off[i] : reinterpret_cast<const char *>(&kZeros), dst + i * 1024);
        }
        slot_in = slot_in + 1 == D ? 0 : slot_in + 1;
        k0 += kBK;
    };
    f32x4 acc[MB][NB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[mb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int wr = (wave / WC) * WM, wc = (wave % WC) * WN;
    struct Operands {
        u32x4 a[2][P * MB], b[2][NB];
    };
    int at_a[2], at_b[2];  // this lane's slots in a stage for the two steps of 32 k
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int kc = s * 4 + (lane >> 4), ra = wr + (lane & 15), rb = wc + pair_column(lane, 0);
        at_a[s] = ra * 8 + (kc ^ swz_a(ra));
        at_b[s] = (AR + rb) * 8 + (kc ^ swz_b(rb));
    }
    const auto read = [&](Operands &o, int slot) {
        const u32x4 *const cur = ring + slot * STAGE;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int m = 0; m < P * MB; ++m) o.a[s][m] = cur[at_a[s] + (m / MB * BM + m % MB * 16) * 8];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) o.b[s][nb] = cur[at_b[s] + pair_column(0, nb) * 8];  // (rows 4 and 32 on: same swizzle)
        }
    };
    const auto multiply = [&](const Operands &o) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int m = 0; m < P * MB; ++m)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) acc[m % MB][nb] = mfma(o.b[s][nb], o.a[s][m], acc[m % MB][nb]);
    };
#pragma unroll
    for (int st = 0; st < D; ++st)
        if (st < stages) issue();
    wait_stages<NPW, D - 1>(min(D - 1, stages - 1));
    half_phase();
    Operands o0, o1;
    read(o0, 0);
    int slot = 0;
    const auto step = [&](Operands &now, Operands &next, int kt) {
        // stage kt + 1 has landed once no more than the D - 2 stages issued after it are in flight; this wave's operands of
        // stage kt have arrived, behind the barrier those of all waves: its slot is free
        if (kt + 1 < stages) wait_stages<NPW, D - 2>(min(D - 2, stages - 2 - kt));
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
        half_phase();
        if (kt + D < stages) issue();
        slot = slot + 1 == D ? 0 : slot + 1;
        if (kt + 1 < stages) read(next, slot);
        multiply(now);
    };
    for (int kt = 0; kt < stages; kt += 2) {
        step(o0, o1, kt);
        if (kt + 1 < stages) step(o1, o0, kt + 1);
    }

    if (g.splits > 1) {
        const int tile = nt * ((g.M + BM - 1) / BM) + mt;
        f32x4 *const parts = reinterpret_cast<f32x4 *>(g.parts) + (size_t)tile * g.splits * (BM * BN / 4) + (size_t)wave * MB * NB * 64 + lane;
#pragma unroll
        for (int b = 0; b < MB * NB; ++b) put_part<true>(parts + (size_t)blockIdx.z * (BM * BN / 4) + b * 64, acc[b / NB][b % NB]);
        if (!last_of_tile<true>(g.counters + tile, g.splits)) return;
        join_parts<true>(reinterpret_cast<f32x4(&)[MB * NB]>(acc), parts, BM * BN / 4, g.splits);
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

// Many rows: bound by the products.  A tile of 64 Q rows and 256 weight rows on eight
// waves of 32 Q x 64, K in stages of 64, two of them in LDS.  A stage has four regions:
// Ah, the h-th 16 Q rows of both row halves, and Bp, the p-th 32 weight rows of the four
// columns of waves (kGate: B0 gate, B1 up).  Its products are four phases of 4 Q matrix
// instructions:
//     phase   products    reads for them                refills (of two stages on)
//       0      A0 x B0      A0                            A1 (of the next stage)
//       1      A0 x B1      B1                            B0
//       2      A1 x B1      A1                            A0
//       3      A1 x B0      B0 of the next stage          B1
// where a phase first reads and refills, then multiplies.  Waves 4 .. 7 run half a phase
// behind waves 0 .. 3, the other wave of their SIMD, so that one multiplies while the other
// reads: LDS and the matrix unit both are busy all the time.  A region is refilled two
// phases after its last read (a barrier ends every half phase, and a wave's reads have
// arrived when its phase ends) and read six phases after that: a wave waits for all but its
// last five refills, never for all.
//   4-bit weights: B0 and B1 are one region of codes, refilled and read at B0's places.  A
// lane's 16 codes of a stage are 16 neighbouring k under one scale, the operands of both
// 32-k steps (the rows' chunks lie in that order); phases 0 and 1 make them bf16.  The
// scales of up to kRunStages stages wait in LDS from before the first, a longer K is run in
// parts.
//   bf16: 4160 x 2 x 10944 columns of K = 2048 in 310 us, 1200 TFLOP/s (4096 x 4096 of K =
// 16384: 1460; a tile's start and end cost 8 us, its 32 stages 46); 4 bits: 4096 x 8192 of
// K = 2048 in 118 us, 1165 TFLOP/s, the conversions beside the products.
constexpr int kRunStages = 128;
enum Region : int { kB0, kA0, kB1, kA1 };  // in the order that they are filled
// Loads that a wave makes for a region.
template <int Q, bool FOUR>
struct Fills {
    static constexpr int of(Region r) { return r == kA0 || r == kA1 ? Q / 2 : FOUR ? (r == kB0 ? 1 : 0) : 2; }
    static constexpr int all() { return of(kB0) + of(kA0) + of(kB1) + of(kA1); }
    static constexpr int last_five(Region newest) { return all() + of(newest); }
};
template <int Q, bool FOUR, int EPI>
__global__ __launch_bounds__(512) void big_kernel(const GemmArgs g) {
    static_assert(Q == 2 || Q == 4, "whole loads of a region");
    constexpr int BM = 64 * Q;
    using F = Fills<Q, FOUR>;
    // 16-byte slots of the regions and their places in a stage
    constexpr int B0_SLOTS = FOUR ? 512 : 1024, B1_SLOTS = FOUR ? 0 : 1024;
    constexpr int AT_A0 = B0_SLOTS, AT_A1 = AT_A0 + 256 * Q, AT_B1 = AT_A1 + 256 * Q, STAGE = AT_B1 + B1_SLOTS;
    constexpr int SCALE_ROW = kRunStages * 2 + 4;         // bytes of a weight row's scales: 4 beside the banks of the next row
    __shared__ __attribute__((aligned(1024))) u32x4 ring[2 * STAGE];
    __shared__ uint32_t scales[FOUR ? 256 * SCALE_ROW / 4 : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    constexpr int COLS = EPI == kGate ? 128 : 256;
    // the parts of one z follow each other: an XCD's tiles are then at the same stages
    const int mtiles = (g.M + BM - 1) / BM, ntiles = (g.N + COLS - 1) / COLS, tiles = mtiles * ntiles;
    const int place = xcd_run(blockIdx.x, gridDim.x), z = __builtin_amdgcn_readfirstlane(place / tiles);
    int mt, nt;
    tile_at(place - z * tiles, mtiles, ntiles, &mt, &nt);
    const int m0 = __builtin_amdgcn_readfirstlane(mt * BM), n0 = __builtin_amdgcn_readfirstlane(nt * COLS);
    const int nk = (g.K + kBK - 1) / kBK;
    const int wr = wave >> 2, wc = wave & 3, l16 = lane & 15, g4 = lane >> 4;

    // Filling.  A wave's i-th load fills rows 64 i + 8 w .. + 7 of a region, which are neighbours in x or the weights: their first
    // one is wave-uniform, this lane's place behind it is the same for all (with 4-bit weights a load is 32 rows' codes).  Rows
    // past the end repeat the last one; never stored.
    const int at_k = (lane & 7) ^ swz_a(8 * wave + (lane >> 3));
    const int kin_a = (FOUR ? 2 * (at_k & 3) + (at_k >> 2) : at_k) * 8;  // (4-bit: chunk 2 q + s at the place of 4 s + q, which is read conflict-free)
    const int kin_b = FOUR ? ((lane ^ (lane >> 4)) & 1) * 32 : ((lane & 7) ^ swz_b(8 * wave + (lane >> 3))) * 8;
    const uint32_t lane_a = (uint32_t)(lane >> 3) * (uint32_t)g.K * 2u + (uint32_t)kin_a * 2u;
    uint32_t lane_b = (uint32_t)(lane >> 3) * (uint32_t)g.K * 2u + (uint32_t)kin_b * 2u;
    const char *row_b[2][2] = {{nullptr, nullptr}, {nullptr, nullptr}};  // [p][i]; FOUR: [0][0] alone
    const auto column = [&](int rb) {  // of weight row rb of the tile
        return min(n0 + (EPI == kGate ? (rb >> 6) * 32 + (rb & 31) : rb), g.N - 1) - n0;
    };
    if constexpr (FOUR) {
        const uint8_t *const codes = (EPI == kGate && (wave & 1) ? g.up.codes : g.b.codes) + (size_t)n0 * (g.K / 2);
        row_b[0][0] = uniform(reinterpret_cast<const char *>(codes));
        // Codes of 32 rows: those of an operand's 16 rows follow each other, and the two halves of a row change places in
        // every other eight rows, so that 32 lanes read all 64 banks.
        const int at = lane >> 1, row = 8 * ((at >> 2) & 3) + 4 * (at >> 4) + (at & 3);
        lane_b = (uint32_t)column(32 * wave + row) * (uint32_t)(g.K / 2) + (uint32_t)kin_b / 2u;
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = 64 * i + 8 * wave;
#pragma unroll
            for (int p = 0; p < 2; ++p) {  // (widths are multiples of 8: the eight columns exist or none of them)
                const int col = min(n0 + (EPI == kGate ? (r >> 5) * 32 + (r & 31) : (r >> 5) * 64 + 32 * p + (r & 31)), g.N - 8);
                row_b[p][i] = uniform(reinterpret_cast<const char *>((EPI == kGate && p == 1 ? g.up.w : g.b.w) + (size_t)col * g.K));
            }
        }
    }
    const uint32_t ring_lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ring));
    const char *a_run = nullptr;  // rows of x of this run's plane
    int st_run = 0;               // and its first stage
    const auto zeros_or = [](bool in, const char *from) { return in ? from : reinterpret_cast<const char *>(&kZeros); };
    const auto fill = [&](auto region_, int st, int slot) {  // into stage slot `slot`
        constexpr int region = decltype(region_)::value;
        const int k0 = (st_run + st) * kBK;
        const bool whole = k0 + kBK <= g.K;  // (not so: the last stage of a K that is no multiple of 64)
        const uint32_t stage = ring_lds + (uint32_t)slot * (STAGE * 16) + wave * 1024;
        if constexpr (region == kA0 || region == kA1) {
#pragma unroll
            for (int i = 0; i < Q / 2; ++i) {
                const int r = 64 * i + 8 * wave, half = r / (16 * Q);
                const int row = m0 + half * (BM / 2) + (region == kA0 ? 0 : 16 * Q) + r % (16 * Q);
                const uint32_t dst = stage + (region == kA0 ? AT_A0 : AT_A1) * 16 + i * 8192;
                if (whole && row + 8 <= g.M) {
                    dma16_at(lane_a, a_run + ((size_t)row * g.K + k0) * 2, dst);
                } else {
                    const size_t at = (size_t)min(row + (lane >> 3), g.M - 1) * g.K + k0 + kin_a;
                    dma16(zeros_or(k0 + kin_a < g.K, a_run + at * 2), dst);
                }
            }
        } else if constexpr (!FOUR) {
            constexpr int p = region == kB0 ? 0 : 1;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t dst = stage + (p == 0 ? 0 : AT_B1) * 16 + i * 8192;
                const char *base = row_b[p][i] + (size_t)k0 * 2;
                if (whole) dma16_at(lane_b, base, dst);
                else dma16(zeros_or(k0 + kin_b < g.K, base + lane_b), dst);
            }
        } else if constexpr (region == kB0) {
            const char *base = row_b[0][0] + (size_t)k0 / 2;
            if (whole) dma16_at(lane_b, base, stage);
            else dma16(zeros_or(k0 + kin_b < g.K, base + lane_b), stage);
        }
    };

    f32x4 acc[2][Q][4];      // [h][mb][2 p + nb]
    u32x4 fa[Q][2];           // [mb][k step]
    u32x4 fb0[2][2][2], fb1[2][2];  // B0 of two stages (4-bit: of one), B1: [nb][k step]
    typedef uint32_t codes2 __attribute__((ext_vector_type(2)));
    codes2 code[2][2];        // [p][nb]
    uint32_t scale[2][2];
    // this lane's slots in a region for the two k steps
    int at_a[2], at_b[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        at_a[s] = (16 * Q * wr + l16) * 8 + ((4 * s + g4) ^ swz_a(l16));
        at_b[s] = (32 * wc + pair_column(lane, 0)) * 8 + ((4 * s + g4) ^ swz_b(pair_column(lane, 0)));  // (the pair's other block: 4 rows on)
    }
    const auto read_a = [&](int slot, int at) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int mb = 0; mb < Q; ++mb) fa[mb][s] = ring[slot * STAGE + at + mb * 128 + at_a[s]];
    };
    const auto read_b = [&](u32x4(&fb)[2][2], int slot, int at) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int nb = 0; nb < 2; ++nb) fb[nb][s] = ring[slot * STAGE + at + nb * 32 + at_b[s]];
    };
    const auto read_codes = [&](int slot, int st) {
        const codes2 *const from = reinterpret_cast<const codes2 *>(ring + slot * STAGE);
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int nb = 0; nb < 2; ++nb) {
                const int r = 64 * wc + 32 * p + pair_column(lane, nb);
                code[p][nb] = from[(64 * wc + 32 * p + 16 * nb + l16) * 4 + (((g4 >> 1) ^ (l16 >> 3)) * 2 + (g4 & 1))];
                scale[p][nb] = scales[r * (SCALE_ROW / 4) + (st >> 1)];
            }
    };
    const auto convert = [&](u32x4(&fb)[2][2], int p, int st) {
        if constexpr (FOUR) {
#pragma unroll
            for (int nb = 0; nb < 2; ++nb) {
                const float f = mx_scale((scale[p][nb] >> ((st & 1) * 16 + (g4 >> 1) * 8)) & 0xffu);
#pragma unroll
                for (int s = 0; s < 2; ++s) fb[nb][s] = mx_values(code[p][nb][s], f);
            }
        }
    };
    const auto multiply = [&](int h, const u32x4(&fb)[2][2], int p) {
        half_phase();
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int mb = 0; mb < Q; ++mb)
#pragma unroll
                for (int nb = 0; nb < 2; ++nb) acc[h][mb][2 * p + nb] = mfma(fb[nb][s], fa[mb][s], acc[h][mb][2 * p + nb]);
        __builtin_amdgcn_s_setprio(0);
        asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");  // what this phase read has arrived, used already or not
        half_phase();
    };
    const std::integral_constant<int, kB0> B0{};
    const std::integral_constant<int, kB1> B1{};
    const std::integral_constant<int, kA0> A0{};
    const std::integral_constant<int, kA1> A1{};
    // One stage, in slot SLOT; behind it LEFT more (2: any number, which are refilled).
    const auto stage = [&](auto slot_, auto left_, int st) {
        constexpr int SLOT = decltype(slot_)::value, LEFT = decltype(left_)::value, FB = FOUR ? 0 : SLOT;
        read_a(SLOT, AT_A0);
        if constexpr (LEFT >= 1) fill(A1, st + 1, SLOT ^ 1);
        convert(fb0[FB], 0, st);
        wait_vm<LEFT >= 1 ? F::last_five(kA1) : F::of(kA1)>();
        multiply(0, fb0[FB], 0);
        if constexpr (!FOUR) read_b(fb1, SLOT, AT_B1);
        if constexpr (LEFT >= 2) fill(B0, st + 2, SLOT);
        convert(fb1, 1, st);
        wait_vm<LEFT >= 2 ? F::last_five(kB0) : LEFT == 1 ? F::all() : 0>();
        multiply(0, fb1, 1);
        read_a(SLOT, AT_A1);
        if constexpr (LEFT >= 2) fill(A0, st + 2, SLOT);
        if constexpr (LEFT >= 1) wait_vm<LEFT >= 2 ? F::last_five(kA0) : F::all() - F::of(kB0)>();
        multiply(1, fb1, 1);
        if constexpr (LEFT >= 1) {
            if constexpr (FOUR) read_codes(SLOT ^ 1, st + 1);
            else read_b(fb0[FB ^ 1], SLOT ^ 1, 0);
        }
        if constexpr (LEFT >= 2) fill(B1, st + 2, SLOT);
        if constexpr (LEFT >= 1) wait_vm<LEFT >= 2 ? F::last_five(kB1) : F::of(kB1) + F::of(kA1)>();
        multiply(1, fb0[FB], 0);
    };
    // The scales of a run's stages, four (of two stages) a word, 0 behind the last group: two threads a weight row, eight
    // words of a thread in flight.  (One after the other they cost each tile 8 us.)
    const auto load_scales = [&](int stages) {
        const int rb = tid >> 1, groups = g.K / kMxGroup - 2 * st_run, words = (stages + 1) / 2, mine = (words + 1) / 2;
        const uint8_t *const from = (EPI == kGate && (rb & 32) ? g.up.scales : g.b.scales) + ((size_t)n0 + column(rb)) * (g.K / kMxGroup) + 2 * st_run;
        uint32_t *const to = scales + rb * (SCALE_ROW / 4);
        const int rest = groups & 3, full = groups >> 2;
        for (int i0 = 0; i0 < mine; i0 += 8) {
            uint32_t v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int w = (tid & 1) * mine + i0 + i;
                v[i] = 0;
                if (w < full) __builtin_memcpy(&v[i], from + 4 * w, 4);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int w = (tid & 1) * mine + i0 + i;
                if (w == full)
                    for (int k = 0; k < rest; ++k) v[i] |= (uint32_t)from[4 * w + k] << (8 * k);
                if (i0 + i < mine && w < words) to[w] = v[i];
            }
        }
        __syncthreads();
    };
    const auto run = [&](int stages) {
        const int first = stages & 1;  // slot of the first stage: the last but one is in slot 0
        fill(B0, 0, first);
        fill(A0, 0, first);
        fill(B1, 0, first);
        fill(A1, 0, first);
        fill(B0, 1, first ^ 1);
        fill(A0, 1, first ^ 1);
        fill(B1, 1, first ^ 1);
        if constexpr (FOUR) load_scales(stages);
        wait_vm<F::last_five(kB1)>();
        half_phase();
        if constexpr (FOUR) {
            read_codes(first, 0);
        } else {  // into both: a choice between them would put them into memory
            read_b(fb0[0], first, 0);
#pragma unroll
            for (int b = 0; b < 4; ++b) fb0[1][b / 2][b % 2] = fb0[0][b / 2][b % 2];
        }
        if (wr == 1) half_phase();
        int st = 0;
        if (first == 1) stage(std::integral_constant<int, 1>(), std::integral_constant<int, 2>(), st++);
        for (; st < stages - 2; st += 2) {
            stage(std::integral_constant<int, 0>(), std::integral_constant<int, 2>(), st);
            stage(std::integral_constant<int, 1>(), std::integral_constant<int, 2>(), st + 1);
        }
        stage(std::integral_constant<int, 0>(), std::integral_constant<int, 1>(), st);
        stage(std::integral_constant<int, 1>(), std::integral_constant<int, 0>(), st + 1);
        if (wr == 0) half_phase();
    };
    // Stages [s0, s1) of the tile, counted over all planes of x.
    const auto sums = [&](int s0, int s1) {
#pragma unroll
        for (int b = 0; b < 8 * Q; ++b) acc[b / (4 * Q)][b / 4 % Q][b % 4] = f32x4{0.f, 0.f, 0.f, 0.f};
        while (s0 < s1) {
            const int p = s0 / nk, left = min(s1, (p + 1) * nk) - s0;
            // with 4-bit weights at most kRunStages of them: in parts of equal length, so of two stages at least
            const int stages = FOUR ? left / ((left + kRunStages - 1) / kRunStages) : left;
            a_run = uniform(reinterpret_cast<const char *>(g.a + (size_t)p * g.plane_rows * g.K));
            st_run = s0 - p * nk;
            run(stages);
            s0 += stages;
        }
    };
    // K cut into parts: in units of four stages (the last of a plane up to seven), so that none is shorter than two
    const int per_plane = max(nk / kUnitStages, 1), units = per_plane * g.a_planes;
    const auto stage_of = [&](int u) { return u / per_plane * nk + u % per_plane * kUnitStages; };
    sums(__builtin_amdgcn_readfirstlane(stage_of((int)((long long)units * z / g.splits))),
         __builtin_amdgcn_readfirstlane(stage_of((int)((long long)units * (z + 1) / g.splits))));
    if (g.splits > 1) {
        constexpr size_t PART = BM * 64;  // f32x4 of a part
        const int tile = nt * mtiles + mt;
        f32x4 *const parts = reinterpret_cast<f32x4 *>(g.parts) + (size_t)tile * g.splits * PART + (size_t)wave * (8 * Q) * 64 + lane;
#pragma unroll
        for (int b = 0; b < 8 * Q; ++b) put_part<false>(parts + (size_t)z * PART + b * 64, acc[b / (4 * Q)][b / 4 % Q][b % 4]);
        if (!last_of_tile<false>(g.counters + tile, g.splits)) return;
        join_parts<false>(reinterpret_cast<f32x4(&)[8 * Q]>(acc), parts, PART, g.splits);
    }
    // acc[h][mb][2 p + b][i] = C[BM / 2 wr + 16 Q h + 16 mb + lane % 16][column 8 (lane / 16) + 4 b + i of the wave's p-th 32]
    const int cw = n0 + wc * (EPI == kGate ? 32 : 64) + 8 * g4;
#pragma unroll
    for (int b = 0; b < 2 * Q; ++b) {
        const f32x4(&v)[4] = acc[b / Q][b % Q];
        const int row = m0 + BM / 2 * wr + 16 * b + l16;
        if (row >= g.M) continue;
        if constexpr (EPI == kGate) {
            if (cw < g.N) store_h(g, v[0], v[1], v[2], v[3], row, cw);
        } else {
#pragma unroll
            for (int p = 0; p < 2; ++p)
                if (cw + 32 * p < g.N) store_eight<EPI>(g, v[2 * p], v[2 * p + 1], row, cw + 32 * p);
        }
    }
}

template <class... A, class... B>
hipError_t launch_epilogue(Epilogue epi, void (*bf16)(A...), void (*f32)(A...), void (*gate)(A...), dim3 grid, int threads, hipStream_t s, B... args) {
    (epi == kStoreBf16 ? bf16 : epi == kStoreF32 ? f32 : gate)<<<grid, threads, 0, s>>>(args...);
    return hipGetLastError();
}
template <int MB, int CB, int WC, int KG, int SL>
hipError_t launch_mid(const GemmArgs &g, Epilogue epi, dim3 grid, hipStream_t s) {
    return launch_epilogue(epi, mid_kernel<MB, CB, WC, KG, SL, kStoreBf16>, mid_kernel<MB, CB, WC, KG, SL, kStoreF32>, mid_kernel<MB, CB, WC, KG, SL, kGate>,
                           dim3(grid.x * grid.y, 1, grid.z), 64 * WC * KG, s, g);
}
template <int BM, int D, int D3, int WR>
hipError_t launch_tile(const GemmArgs &g, Epilogue epi, dim3 grid, hipStream_t s) {
    return launch_epilogue(epi, tile_kernel<BM, 128, D, WR, 2, kStoreBf16, 1>, tile_kernel<BM, 128, D3, WR, 2, kStoreF32, 3>,
                           tile_kernel<BM, 128, D, WR, 2, kGate, 1>, dim3(grid.x * grid.y, 1, grid.z), 128 * WR, s, g);
}
template <int Q, bool FOUR>
hipError_t launch_big(const GemmArgs &g, Epilogue epi, dim3 grid, hipStream_t s) {  // the tiles of every part, those of a part behind each other
    return launch_epilogue(epi, big_kernel<Q, FOUR, kStoreBf16>, big_kernel<Q, FOUR, kStoreF32>, big_kernel<Q, FOUR, kGate>,
                           dim3(grid.x * grid.y * grid.z), 512, s, g);
}
template <int CB, bool FOUR>
hipError_t launch_rows(const GemmArgs &g, Epilogue epi, dim3 grid, hipStream_t s) {
    constexpr int kAlone = FOUR ? 1 : 3;  // in front of fp32 one plane is a product on its own, which has 4-bit weights
    return launch_epilogue(epi, rows_kernel<1, CB, FOUR, kStoreBf16, 1>, g.a_planes == 3 ? rows_kernel<1, CB, FOUR, kStoreF32, 3> : rows_kernel<1, CB, FOUR, kStoreF32, kAlone>,
                           rows_kernel<1, CB, FOUR, kGate, 1>, grid, 512, s, g);
}

}  // namespace

hipError_t launch_gemm(GemmArgs g, bool four_bit, Epilogue epi, const Shape &t, hipStream_t s) {
    if (!fits(g, four_bit, epi, t) || (t.splits > 1 && (!g.parts || !g.counters))) return hipErrorInvalidValue;
    const Tiles n = tiles_of(g, epi, t.variant);
    g.splits = t.splits;
    const dim3 grid((unsigned)n.n, (unsigned)n.m, (unsigned)t.splits);
    switch (t.variant) {
        case kRows16: return four_bit ? launch_rows<2, true>(g, epi, grid, s) : launch_rows<2, false>(g, epi, grid, s);
        case kRows16Narrow: return four_bit ? launch_rows<1, true>(g, epi, grid, s) : launch_rows<1, false>(g, epi, grid, s);
        case kTile32: return launch_tile<32, 4, 2, 2>(g, epi, grid, s);
        case kTile64: return launch_tile<64, 3, 3, 4>(g, epi, grid, s);
        case kTile128: return launch_tile<128, 4, 2, 4>(g, epi, grid, s);
        case kMid16: return launch_mid<1, 2, 2, 4, 2>(g, epi, grid, s);
        case kMid32: return launch_mid<2, 2, 2, 4, 1>(g, epi, grid, s);
        case kMid48: return launch_mid<3, 2, 2, 4, 1>(g, epi, grid, s);
        case kMid64: return launch_mid<4, 2, 2, 4, 1>(g, epi, grid, s);
        case kMid32Wide: return launch_mid<2, 2, 8, 1, 2>(g, epi, grid, s);
        case kMid64Wide: return launch_mid<4, 4, 4, 1, 1>(g, epi, grid, s);
        case kMid64Cols: return launch_mid<4, 2, 4, 1, 2>(g, epi, grid, s);
        case kMid64Long: return launch_mid<4, 2, 4, 2, 2>(g, epi, grid, s);
        case kBig128: return four_bit ? launch_big<2, true>(g, epi, grid, s) : launch_big<2, false>(g, epi, grid, s);
        case kBig256: return four_bit ? launch_big<4, true>(g, epi, grid, s) : launch_big<4, false>(g, epi, grid, s);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace ffn
