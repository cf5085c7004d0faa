// Decode rows over the 8-bit cache (include/mla_cache.h): device code, part of
// mla_kernels.hip (its helpers and namespace).
#pragma once

// Index of the pair of scales (4 bytes) of a key in a pool page.
__device__ __forceinline__ size_t scale_entry(const AttnArgs &a, int page, int key) {
    return (size_t)page * (a.page_size / kBlock8) + (size_t)((key & (a.page_size - 1)) / kBlock8);
}

// Eight e4m3 codes (two words) times a power of two as bf16: exact.
__device__ __forceinline__ u32x4 bf16_of_e4m3x8(uint32_t w0, uint32_t w1, float scale) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true))};
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

// A tile in LDS: 32 keys of 36 16-byte pieces, row-major; piece positions are
// xor-swizzled inside aligned groups of four.  Rows are 9 x 64 bytes, so four
// consecutive keys cover the 64 banks at one piece: bits 2 and 3 of the key spread
// the 16 keys of a score operand, bit 4 the two key halves of a value operand.
constexpr int kPieces8 = kDqk / 16;  // 36
__device__ __forceinline__ int swz8(int k) { return ((k >> 2) & 3) ^ ((k >> 3) & 2); }
__device__ __forceinline__ int tile8_off(int k, int c) { return (k * kPieces8 + (c ^ swz8(k))) * 16; }

// A unit (query block or tile: 18 rounds of 1 KB) takes five DMA instructions of
// each wave, so that what is in flight can be counted: rounds wv, wv + 4, ..; the
// fifth of waves 2 and 3 loads the scales of key half wv - 2 (of a query block:
// their first round again).
constexpr int kDma8 = 5;
__device__ __forceinline__ void dma8_offsets(int wv, int lane, uint32_t (&off)[3]) {
#pragma unroll
    for (int w = 0; w < 3; ++w) off[w] = 0;
#pragma unroll
    for (int i = 0; i < kDma8; ++i) {
        const int u = (i * 4 + wv) * 64 + lane, kk = u / kPieces8, c = (u - kk * kPieces8) ^ swz8(kk);
        if (u < kDecKeys * kPieces8) off[i / 2] |= (uint32_t)(kk * kDqk + c * 16) << (16 * (i & 1));
    }
}
// Until only the DMAs of the last `units` units are in flight.  (Loads complete in
// order; a store in between only makes the wait longer.)
__device__ __forceinline__ void wait_dma8(int units) {
    if (units >= 2)
        asm volatile("s_waitcnt vmcnt(10)" ::: "memory");
    else if (units == 1)
        asm volatile("s_waitcnt vmcnt(5)" ::: "memory");
    else
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <int F>
__device__ __forceinline__ void issue_unit8(const AttnArgs &a, const DecSeg &sg, int t, const int *s_pages, uint32_t slot,
                                            uint32_t scale_slot, int wv, int lane, const uint32_t (&off)[3]) {
    const auto lds = [&](int i) { return __builtin_amdgcn_readfirstlane(slot + (i * 4 + wv) * 1024); };
    asm volatile("" : "+v"(lane));  // (nothing of the rare paths is kept across the units)
    if (t < 0) {
        const char *qb = reinterpret_cast<const char *>(a.q + (size_t)sg.row * kHeads * kDqk) + lane * 16;
#pragma unroll
        for (int i = 0; i < kDma8; ++i) {
            const int j = i == 4 && wv >= 2 ? 0 : i;
            lds_dma16(qb + (j * 4 + wv) * 1024, lds(j));
        }
        return;
    }
    const SegKeys<has_window<F>> sk(a, sg);
    const int kbase = sk.key(t * kDecKeys);
    const auto page_of = [&](int key) { return s_pages[min(sk.window_entry(sg, key, a.log2_page), kPageWindow - 1)]; };
    if (a.page_size >= kDecKeys && kbase + kDecKeys - 1 <= sg.p) {
        const int page = __builtin_amdgcn_readfirstlane(page_of(kbase));
        const uint8_t *src = a.kv8 + ((size_t)page * a.page_size + (kbase & (a.page_size - 1))) * kDqk;
#pragma unroll
        for (int i = 0; i < kDma8; ++i)
            if (i < 4 || wv < 2) lds_dma16_sbase(src, (off[i / 2] >> (16 * (i & 1))) & 0xffffu, lds(i));
    } else {
#pragma unroll
        for (int i = 0; i < kDma8; ++i) {
            if (i == 4 && wv >= 2) break;
            const int u = (i * 4 + wv) * 64 + lane, kk = u / kPieces8, c = (u - kk * kPieces8) ^ swz8(kk);
            const int key = min(kbase + kk, sg.p);
            lds_dma16(a.kv8 + ((size_t)page_of(key) * a.page_size + (key & (a.page_size - 1))) * kDqk + c * 16, lds(i));
        }
    }
    if (wv >= 2) {
        const int key = min(kbase + 16 * (wv - 2), sg.p);
        const size_t entry = scale_entry(a, page_of(key), key);
        if (lane == 0)
            lds_dma16(reinterpret_cast<const char *>(a.kv8_scales) + (entry * 4 & ~size_t(15)),
                      __builtin_amdgcn_readfirstlane(scale_slot + 16 * (wv - 2)));
    }
}

// decode_wg over the 8-bit cache.  Half the bytes a key: HBM-bound at 578 B a key,
// so a tile of a group has half the time (1.6 us at 6 TB/s), and it is the chain of
// a tile that has to be short.  Raw tiles pass through a ring of four slots, two to
// three of them in flight.  Keys are converted where the matrix instruction takes
// them (one instruction for two values, the scale of the 16 keys of its rows applied
// on the way: bf16 holds the value exactly), the values of a tile before its score
// barrier, with their scales folded into the probabilities (a power of two, exact).
template <int F>
__device__ void decode8_wg(const AttnArgs &a, int w, char *smem, int (*s_pages_g)[kPageWindow], DecSeg (*s_seg_g)[kMaxSeg],
                           int *s_gbar) {
    const int tid = item_tid(), lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = wv >> 2, gw = wv & 3, gtid = tid & 255;  // wave group, wave and thread inside it
    const int g = lane >> 4, h = lane & 15;
    const int S = a.dec_unit_tiles;
    const int v = 2 * w + grp;  // this group's unit
    const int R0 = v * S, R1 = min(R0 + S, a.dec_total_tiles);
    DecSeg *const s_seg = s_seg_g[grp];
    int *const s_pages = s_pages_g[grp];
    const int nseg = R0 < R1 ? find_unit<F>(a, R0, R1, s_seg, gw == 0) : 0;
    const int n_units = nseg > 0 ? nseg + (R1 - R0) : 0;
    if (tid < 2) s_gbar[tid] = 0;
    TRACE(1);
    __syncthreads();
    uint32_t off[3];
    dma8_offsets(gw, lane, off);
    char *const slots = smem + grp * kDec8GroupBytes;
    char *const s_X = smem + 2 * kDec8GroupBytes + grp * kDec8XBytes;
    char *const s_scale = smem + 2 * (kDec8GroupBytes + kDec8XBytes) + grp * kDec8ScaleBytes;
    const uint32_t ring = lds_addr(slots), scales = lds_addr(s_scale);
    Cursor prod{0, -1, DecSeg{}};
    if (n_units > 0) prod.sg = load_seg(s_seg, 0);
    Cursor cons = prod;
    const auto issue = [&](int u) {
        issue_unit8<F>(a, prod.sg, prod.t, s_pages, ring + (u % kDec8Ring) * kDec8TileBytes, scales + (u % kDec8Ring) * 32, gw, lane, off);
        advance(prod, s_seg, nseg);
    };
    if (n_units > 0) {
        issue(0);  // the first query block
        // page window: entry gtid belongs to the last segment that starts at or before it
        int j = 0;
        for (int k = 1; k < nseg; ++k) j = s_seg[k].pw <= gtid ? k : j;
        const DecSeg sg = s_seg[j];
        const int i = gtid - sg.pw;
        const SegKeys<has_window<F>> sk(a, sg);
        if (i < sk.pages(a, sg)) {
            const int lp = sk.logical_page(sg, i);
            const int pg = lp < a.max_pages ? a.bt[(size_t)sg.r * a.max_pages + lp] : 0;
            const bool ok = (unsigned)pg < (unsigned)a.num_pages;
            if (!ok && page_seen<F>(a, lp, sg.p)) raise_flag(kFlagBadPage);
            s_pages[gtid] = ok ? pg : 0;
        }
    }
    __syncthreads();
    if (n_units == 0) return;  // this group has no unit (the other one may)
    if (n_units > 1) issue(1);
    if (n_units > 2) issue(2);
    int epoch = 0;
    int *const gbar = s_gbar + grp;
    TRACE(2);
    TRACE_VAL(8, 1000000ull * 2 + n_units);

    // This wave's half of the dims, 9 steps of 32: four groups of 64 from gbase on (a lane's 16 dims of a group feed two
    // steps: the dims of a step may be any, as long as keys and queries agree), and 32 from sbase on.
    const int hf = gw >> 1, gbase = hf ? 320 : 0, sbase = hf ? 288 : 256;
    u32x4 qreg[9];
    f32x4 acc[8];
#pragma unroll
    for (int mt = 0; mt < 8; ++mt) acc[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_ref = kNegInf, l_run = 0.f;
    const int kq = 16 * (gw & 1) + (lane & 15);  // key this lane scores
    // value operand: slots 8 g + 4 kt + i of a step hold keys 16 kt + 4 g + i, as the probabilities do
    const int tr = (lane & 15) >> 1, tr_key = 4 * g + (tr & 3) + 16 * (tr >> 2);

    TRACE(3);
    for (int u = 0; u < n_units; ++u) {
        TRACE_TILE(u, 10);
        wait_dma8(min(2, n_units - 1 - u));        // unit u
        group_barrier(gbar, epoch, a.spin_limit);  // landed for all four waves; slot (u + 3) % 4 is free
        if (u + 3 < n_units) issue(u + 3);
        const char *slot = slots + (u % kDec8Ring) * kDec8TileBytes;
        if (cons.t < 0) {  // a new request: its query block
            const char *q = slot + h * kRowBytes;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                qreg[2 * j] = *reinterpret_cast<const u32x4 *>(q + 2 * (gbase + 64 * j + 16 * g));
                qreg[2 * j + 1] = *reinterpret_cast<const u32x4 *>(q + 2 * (gbase + 64 * j + 16 * g) + 16);
            }
            qreg[8] = *reinterpret_cast<const u32x4 *>(q + 2 * (sbase + 8 * g));
            advance(cons, s_seg, nseg);
            continue;
        }
        TRACE_TILE(u, 11);
        const DecSeg sg = cons.sg;
        const SegKeys<has_window<F>> sk(a, sg);
        const int kbase = sk.key(cons.t * kDecKeys);
        // scales of the tile's two key halves
        float sc[2], sr[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const int key = min(kbase + 16 * kt, sg.p);
            const int pg = a.page_size >= 64 ? 0 : s_pages[min(sk.window_entry(sg, key, a.log2_page), kPageWindow - 1)];
            const uint32_t wd = *reinterpret_cast<const uint32_t *>(s_scale + (u % kDec8Ring) * 32 + 16 * kt + 4 * (scale_entry(a, pg, key) & 3));
            // (a half that no row sees may have anything for a scale: 0 times it would be NaN)
            sc[kt] = (wd & 0x7f80u) == 0x7f80u ? 0.f : __uint_as_float(wd << 16);
            sr[kt] = __uint_as_float(wd & 0xffff0000u);
        }
        {
            // partial scores: keys 16 (gw & 1) .. + 16, this wave's dims
            const float kc = (gw & 1) ? sc[1] : sc[0], kr = hf ? ((gw & 1) ? sr[1] : sr[0]) : kc;
            u32x4 av[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) av[j] = *reinterpret_cast<const u32x4 *>(slot + tile8_off(kq, gbase / 16 + 4 * j + g));
            const u32x2 as = *reinterpret_cast<const u32x2 *>(slot + tile8_off(kq, sbase / 16 + (g >> 1)) + 8 * (g & 1));
            f32x4 sa = {0.f, 0.f, 0.f, 0.f}, sb = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float s = j == 3 ? kr : kc;  // (the last group of the upper half: the rope dims)
                sa = mfma_bf16(bf16_of_e4m3x8(av[j][0], av[j][1], s), qreg[2 * j], sa);
                sb = mfma_bf16(bf16_of_e4m3x8(av[j][2], av[j][3], s), qreg[2 * j + 1], sb);
            }
            sa = mfma_bf16(bf16_of_e4m3x8(as[0], as[1], kc), qreg[8], sa);
            *reinterpret_cast<f32x4 *>(s_X + (gw * 64 + lane) * 16) = sa + sb;
        }
        // values of this wave's 128 dims, before the scores are complete
        u32x2 vraw[8];
#pragma unroll
        for (int mt2 = 0; mt2 < 8; ++mt2) vraw[mt2] = lds_read_tr8(slot + tile8_off(tr_key, gw * 8 + mt2) + 8 * (lane & 1));
        u32x4 vop[8];
#pragma unroll
        for (int mt2 = 0; mt2 < 8; ++mt2) vop[mt2] = bf16_of_e4m3x8(vraw[mt2][0], vraw[mt2][1], 1.f);
        group_barrier(gbar, epoch, a.spin_limit);  // partial score blocks complete
        TRACE_TILE(u, 12);
        // full scores of this lane's head: x[kt][i] = key 16 kt + 4 g + i (kt = 0, 1)
        f32x4 x[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
            x[kt] = *reinterpret_cast<const f32x4 *>(s_X + (kt * 64 + lane) * 16) +
                    *reinterpret_cast<const f32x4 *>(s_X + ((kt + 2) * 64 + lane) * 16);
        if (any_not_finite(x)) {
#pragma unroll
            for (int mt2 = 0; mt2 < 8; ++mt2) {
                const u32x2 raw = lds_read_tr8(slot + tile8_off(tr_key, gw * 8 + mt2) + 8 * (lane & 1));
                vop[mt2] = bf16_of_e4m3x8(finite_e4m3x4(raw[0]), finite_e4m3x4(raw[1]), 1.f);
            }
        }
        float mt = kNegInf;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[kt][i] = row_sees<F>(a, kbase + 16 * kt + 4 * g + i, sg.p) ? x[kt][i] * a.scale_log2 : kNegInf;
                mt = fmaxf(mt, x[kt][i]);
            }
        }
        mt = wave_max16(mt);
        // lazy rescale, the same decision in every wave of the group (see decode_wg)
        if (__builtin_amdgcn_ballot_w64(mt > m_ref + 8.f) != 0) {
            const float m_new = fmaxf(m_ref, mt);
            const float alpha = (m_ref == kNegInf) ? 0.f : exp2f(m_ref - m_new);
#pragma unroll
            for (int mt2 = 0; mt2 < 8; ++mt2) acc[mt2] = acc[mt2] * alpha;
            l_run *= alpha;
            m_ref = m_new;
        }
        // probabilities times their keys' value scale as a bf16 pair hi + lo (about 16 bits)
        uint32_t bh[4], bl[4];
        float ps = 0.f;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                float p0 = (x[kt][i] == kNegInf) ? 0.f : exp2f(x[kt][i] - m_ref);
                float p1 = (x[kt][i + 1] == kNegInf) ? 0.f : exp2f(x[kt][i + 1] - m_ref);
                ps += p0 + p1;
                p0 *= sc[kt];
                p1 *= sc[kt];
                const uint32_t h0 = bf16_bits(p0), h1 = bf16_bits(p1);
                bh[kt * 2 + (i >> 1)] = h0 | (h1 << 16);
                bl[kt * 2 + (i >> 1)] = bf16_bits(p0 - bf16_bits_to_float(h0)) |
                                        (bf16_bits(p1 - bf16_bits_to_float(h1)) << 16);
            }
        }
        l_run += ps;
        TRACE_TILE(u, 13);
        const u32x4 opb_h = {bh[0], bh[1], bh[2], bh[3]};
        const u32x4 opb_l = {bl[0], bl[1], bl[2], bl[3]};
#pragma unroll
        for (int mt2 = 0; mt2 < 8; ++mt2) acc[mt2] = mfma_bf16(vop[mt2], opb_h, acc[mt2]);
#pragma unroll
        for (int mt2 = 0; mt2 < 8; ++mt2) acc[mt2] = mfma_bf16(vop[mt2], opb_l, acc[mt2]);

        TRACE_TILE(u, 14);
        const int jseg = cons.j;
        advance(cons, s_seg, nseg);
        if (cons.j != jseg) {  // the segment's last tile: finish it
            const float l_tot = wave_sum16(l_run);
            if (sg.t0 == 0 && sg.t1 == dec_tiles<F>(a, sg.p, 1)) {
                const float inv = 1.f / l_tot;
#pragma unroll
                for (int mt2 = 0; mt2 < 8; ++mt2)
                    store_out4(a, sg.row, h, gw * 128 + mt2 * 16 + 4 * g, acc[mt2] * inv);
                if (a.lse && gw == 0 && g == 0) a.lse[(size_t)sg.row * kHeads + h] = (m_ref + log2f(l_tot)) * kLn2;
            } else if (a.ws_dec_o != nullptr) {
                const size_t slot_id = 2 * (size_t)v + (jseg == 0 ? 0 : 1);
                float *po = a.ws_dec_o + (slot_id * kHeads + h) * kDv;
#pragma unroll
                for (int mt2 = 0; mt2 < 8; ++mt2)
                    *reinterpret_cast<f32x4 *>(po + gw * 128 + mt2 * 16 + 4 * g) = acc[mt2];
                if (gw == 0 && g == 0) {
                    a.ws_dec_ml[(slot_id * kHeads + h) * 2 + 0] = partial_max(m_ref, l_tot);
                    a.ws_dec_ml[(slot_id * kHeads + h) * 2 + 1] = l_tot;
                }
            }
#pragma unroll
            for (int mt2 = 0; mt2 < 8; ++mt2) acc[mt2] = f32x4{0.f, 0.f, 0.f, 0.f};
            m_ref = kNegInf;
            l_run = 0.f;
        }
    }
    TRACE(4);
}
