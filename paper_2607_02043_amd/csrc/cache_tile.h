// Tiles of the 8-bit cache (include/mla_cache.h): device code, part of
// mla_kernels.hip (its helpers and namespace).
#pragma once

// Scales are powers of two, handled as exponents where that is cheaper.
constexpr int kMinExp8 = -100, kMaxExp8 = 120;
__device__ __forceinline__ float exp2_bits(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
// The exponent of a stored scale (bf16 bits of a power of two; 128 if it is no number).
__device__ __forceinline__ int scale_exponent(uint32_t bf16) { return (int)((bf16 >> 7) & 0xff) - 127; }

// Four bytes of one lane (the others' land behind them), global -> LDS.
__device__ __forceinline__ void lds_dma4(const void *gsrc, uint32_t lds_base) {
    asm volatile(
        "s_nop 0\n\t"
        "global_load_lds_dword %1, off\n\t"
        :
        : "{m0}"(lds_base), "v"(gsrc)
        : "memory");
}

// Eight e4m3 codes (two words) times a power of two as bf16: exact.
__device__ __forceinline__ u32x4 bf16_of_e4m3x8(uint32_t w0, uint32_t w1, float scale) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true))};
}
// The same as fp16, the two words with scales of their own (rounded to nearest; exact unless below 2^-24).
__device__ __forceinline__ u32x4 f16_of_e4m3x8(uint32_t w0, uint32_t w1, float s0, float s1) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, s0, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w0, s0, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, s1, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w1, s1, true))};
}

// Transposing LDS read of 8-bit elements: inside each 16-lane group, lane i receives
// element (i & 7) of the 8 bytes read by lane 2 j + (i >> 3), j = 0..7: of the 8
// rows of 16 that two lanes each read, lane i gets column i.
__device__ __forceinline__ u32x2 lds_read_tr8(const char *p) {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
    const i32x2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2 *)(p));
    return __builtin_bit_cast(u32x2, v);
}

// NaN codes (0x7f, 0xff) of four to zero.
__device__ __forceinline__ uint32_t finite_e4m3x4(uint32_t w) {
    const uint32_t nan = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;  // bit 7 of every NaN byte
    return w & ~((nan >> 7) * 0xffu);
}

// A tile in LDS: nine quads of 64 dims, each 32 keys of four 16-byte pieces.  Four
// consecutive keys cover the 64 banks at one piece; pieces are xor-swizzled by bits 2
// and 3 of the key so that they spread a score operand, and by bit 4 for the two key
// halves of a value operand.  A score operand's read (piece g of key h for lane
// 16 g + h) is served 16 lanes at a time, {0 .. 3, 12 .. 15, 20 .. 27} and the other
// half of 32: keys 0 .. 3 and 12 .. 15 of one piece with keys 4 .. 11 of the next one,
// which fall on four different pieces with 0, 2, 3, 1 (plain 0, 1, 2, 3, or 0, 2, 1, 3:
// 4 conflict cycles a read).  Piece p of quad 0 of key k is at tile8_off(k, p).
constexpr int kQuad8 = kKeysPerTile * 64;  // 2048 bytes
__device__ __forceinline__ int swz8(int k) { return (((k >> 1) ^ (k >> 2)) & 2) ^ ((k >> 3) & 1) ^ ((k >> 4) & 1); }
__device__ __forceinline__ int tile8_off(int k, int p) { return 64 * k + 16 * (p ^ swz8(k)); }

// DMA of a tile (18 rounds of 1 KB) by four waves, five instructions each.  Round j is keys 16 (j & 1) .. + 15 of quad j / 2;
// wave w takes rounds w, w + 4, ..: a lane has one key, and its source moves by two
// quads a round.  The fifth instruction of waves 2 and 3 loads the scales of key half
// w - 2.  (The instruction offset moves source and destination alike.)
__device__ __forceinline__ int tile8_key(int w, int lane) { return 16 * (w & 1) + (lane >> 2); }
__device__ __forceinline__ int tile8_dims(int w, int lane) {
    return 64 * (w >> 1) + 16 * ((lane & 3) ^ swz8(tile8_key(w, lane)));
}
__device__ __forceinline__ void dma_tile8(const uint8_t *src, uint32_t voff, uint32_t slot, int w) {  // uniform src
    const uint32_t dst = slot + 1024 * w;
#define MLA_DMA8(i) lds_dma16_sbase_imm<128 * (i)>(src, voff, __builtin_amdgcn_readfirstlane(dst + 4096 * (i)))
    MLA_DMA8(0); MLA_DMA8(1); MLA_DMA8(2); MLA_DMA8(3);
    if (w < 2) MLA_DMA8(4);
#undef MLA_DMA8
}
__device__ __forceinline__ void dma_tile8(const uint8_t *src, uint32_t slot, int w) {  // src per lane
    const uint32_t dst = slot + 1024 * w;
#define MLA_DMA8(i) lds_dma16_imm<128 * (i)>(src, __builtin_amdgcn_readfirstlane(dst + 4096 * (i)))
    MLA_DMA8(0); MLA_DMA8(1); MLA_DMA8(2); MLA_DMA8(3);
    if (w < 2) MLA_DMA8(4);
#undef MLA_DMA8
}
// Address of the two scales of a pool slot's block, and their DMA to the four bytes at
// `dst` (one lane: nothing beside them is read, so the array may end there).
__device__ __forceinline__ const char *block_scales8(const AttnArgs &a, size_t pool_slot) {
    return reinterpret_cast<const char *>(a.kv8_scales) + pool_slot / kBlock8 * 4;
}
__device__ __forceinline__ void dma_scales8(const char *src, uint32_t dst, int lane) {
    if (lane == 0) lds_dma4(src, __builtin_amdgcn_readfirstlane(dst));
}
