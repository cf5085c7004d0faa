// Decode rows over the 8-bit cache (include/mla_cache.h): device code, part of
// mla_kernels.hip (its helpers and namespace).
#pragma once

// DMA of one stream unit of a group: a tile with its scales, or (t < 0) a query
// block, 18 rounds too (waves 2 and 3 take their first one twice, for the count).
template <int F>
__device__ __forceinline__ void issue_unit8(const AttnArgs &a, const DecSeg &sg, int t, const int *s_pages, uint32_t slot,
                                            uint32_t scale_slot, int wv, int lane) {
    asm volatile("" : "+v"(lane));  // (no address is kept across the units)
    if (t < 0) {
        const char *qb = reinterpret_cast<const char *>(a.q + (size_t)sg.row * kHeads * kDqk) + lane * 16;
#pragma unroll
        for (int i = 0; i < kDma8; ++i) {
            const int j = (i == 4 && wv >= 2 ? 0 : i) * 4 + wv;
            lds_dma16(qb + j * 1024, __builtin_amdgcn_readfirstlane(slot + j * 1024));
        }
        return;
    }
    const SegKeys<has_window<F>> sk(a, sg);
    const int kbase = sk.key(t * kDecKeys);
    const auto slot_of = [&](int key) {  // pool slot
        const int k = min(key, sg.p);
        return (size_t)s_pages[min(sk.window_entry(sg, k, a.log2_page), kPageWindow - 1)] * a.page_size + (k & (a.page_size - 1));
    };
    if (a.page_size >= kDecKeys && kbase + kDecKeys - 1 <= sg.p) {
        const int page = s_pages[min(sk.window_entry(sg, kbase, a.log2_page), kPageWindow - 1)];
        const size_t first = (size_t)__builtin_amdgcn_readfirstlane(page) * a.page_size + (kbase & (a.page_size - 1));
        dma_tile8(a.kv8 + first * kDqk, tile8_key(wv, lane) * kDqk + tile8_dims(wv, lane), slot, wv);
    } else {
        dma_tile8(a.kv8 + slot_of(kbase + tile8_key(wv, lane)) * kDqk + tile8_dims(wv, lane), slot, wv);
    }
    if (wv >= 2) dma_scales8(a, slot_of(kbase + 16 * (wv - 2)), scale_slot + 16 * (wv - 2), lane);
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
    char *const slots = smem + grp * kDec8GroupBytes;
    char *const s_X = smem + 2 * kDec8GroupBytes + grp * kDec8XBytes;
    char *const s_scale = smem + 2 * (kDec8GroupBytes + kDec8XBytes) + grp * kDec8ScaleBytes;
    const uint32_t ring = lds_addr(slots), scales = lds_addr(s_scale);
    Cursor prod{0, -1, DecSeg{}};
    if (n_units > 0) prod.sg = load_seg(s_seg, 0);
    Cursor cons = prod;
    const auto issue = [&](int u) {
        issue_unit8<F>(a, prod.sg, prod.t, s_pages, ring + (u % kDec8Ring) * kTile8Bytes, scales + (u % kDec8Ring) * 32, gw, lane);
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
        const char *slot = slots + (u % kDec8Ring) * kTile8Bytes;
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
            const uint32_t wd = *reinterpret_cast<const uint32_t *>(s_scale + (u % kDec8Ring) * 32 + 16 * kt + 4 * scale_piece8(a, pg, key));
            // (a half that no row sees may have anything for a scale: 0 times it would be NaN)
            sc[kt] = (wd & 0x7f80u) == 0x7f80u ? 0.f : __uint_as_float(wd << 16);
            sr[kt] = __uint_as_float(wd & 0xffff0000u);
        }
        {
            // partial scores: keys 16 (gw & 1) .. + 16, this wave's dims
            const float kc = (gw & 1) ? sc[1] : sc[0], kr = hf ? ((gw & 1) ? sr[1] : sr[0]) : kc;
            u32x4 av[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) av[j] = *reinterpret_cast<const u32x4 *>(slot + kQuad8 * (gbase / 64 + j) + tile8_off(kq, g));
            const u32x2 as = *reinterpret_cast<const u32x2 *>(slot + kQuad8 * 4 + tile8_off(kq, 2 * hf + (g >> 1)) + 8 * (g & 1));
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
        for (int mt2 = 0; mt2 < 8; ++mt2) vraw[mt2] = lds_read_tr8(slot + kQuad8 * (2 * gw + (mt2 >> 2)) + tile8_off(tr_key, mt2 & 3) + 8 * (lane & 1));
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
                const u32x2 raw = lds_read_tr8(slot + kQuad8 * (2 * gw + (mt2 >> 2)) + tile8_off(tr_key, mt2 & 3) + 8 * (lane & 1));
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
