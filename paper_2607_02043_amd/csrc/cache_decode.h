// Decode rows over the 8-bit cache (include/mla_cache.h): device code, part of
// mla_kernels.hip (its helpers and namespace).
#pragma once

// A stream unit of a group: a segment's query block (t < 0), or two tiles of it, t
// and t + 1 (the last one of a segment may be alone).
struct Cursor8 {
    int j, t;
    DecSeg sg;
};
__device__ __forceinline__ void advance8(Cursor8 &c, const DecSeg *s_seg, int nseg) {
    c.t = c.t < 0 ? c.sg.t0 : c.t + 2;
    if (c.t >= c.sg.t1) {
        ++c.j;
        c.t = -1;
        if (c.j < nseg) c.sg = load_seg(s_seg, c.j);
    }
}

// Sources of a unit's DMAs, found while the unit before it is still computed, so that
// only the DMAs themselves stand in a unit's chain.  A tile's rounds are dealt to the
// waves as dma_tile8 says, with the waves' parts exchanged in the second tile: ten
// instructions of each wave.
struct Source8 {
    const uint8_t *src[2];  // per lane: this wave's part of each tile; of a query block src[0]
    const char *scale;      // of the block of 16 keys whose scales this wave loads (lane 0)
    int tiles;              // 0: a query block
};
template <int F>
__device__ __forceinline__ Source8 find_source8(const AttnArgs &a, const Cursor8 &c, const int *s_pages, int wv, int lane) {
    const DecSeg &sg = c.sg;
    Source8 s;
    s.src[1] = nullptr;
    s.scale = nullptr;
    if (c.t < 0) {
        s.tiles = 0;
        s.src[0] = reinterpret_cast<const uint8_t *>(a.q + (size_t)sg.row * kHeads * kDqk) + wv * 1024 + lane * 16;
        return s;
    }
    const SegKeys<has_window<F>> sk(a, sg);
    s.tiles = min(sg.t1 - c.t, 2);
    const auto slot_of = [&](int key) {  // pool slot
        const int k = min(key, sg.p), page = s_pages[min(sk.window_entry(sg, k, a.log2_page), kPageWindow - 1)];
        return (size_t)page * a.page_size + (k & (a.page_size - 1));
    };
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // (past the segment's end the second tile repeats its last key and is not loaded)
        const int w = wv ^ (2 * h);
        s.src[h] = a.kv8 + slot_of(sk.key((c.t + h) * kDecKeys) + tile8_key(w, lane)) * kDqk + tile8_dims(w, lane);
    }
    const int h = wv >= 2 ? 0 : 1;
    s.scale = block_scales8(a, slot_of(sk.key((c.t + h) * kDecKeys) + 16 * (wv & 1)));
    return s;
}
__device__ __forceinline__ void issue8(const Source8 &s, uint32_t slot, uint32_t scale_slot, int wv, int lane) {
    if (s.tiles == 0) {
#pragma unroll
        for (int i = 0; i < 5; ++i)
            if (i < 4 || wv < 2) lds_dma16(s.src[0] + 4096 * i, __builtin_amdgcn_readfirstlane(slot + 1024 * wv + 4096 * i));
        return;
    }
    dma_tile8(s.src[0], slot, wv);
    if (s.tiles == 2) dma_tile8(s.src[1], slot + kTile8Bytes, wv ^ 2);
    if (wv >= 2 || s.tiles == 2) dma_scales8(s.scale, scale_slot + (wv >= 2 ? 0 : 8) + 4 * (wv & 1), lane);
}

// decode_wg over the 8-bit cache.  Half the bytes a key (578), so a key has half the
// time, and what bounds a group is the chain of a unit: wait, barrier, scores,
// barrier, values.  Hence units of two tiles, 64 keys a barrier pair (256 rows of up
// to 16384 keys, with units of one tile in a ring of four slots 370 us, with two 329);
// each wave scores 16 keys over all dims, takes their probabilities against the
// reference so far and passes those on (the scores passed on instead, whose softmax
// every wave then repeats: 329, so 307), and then accumulates its 128 value dims over
// the 64 keys.  That size now takes 261 us with the merge, 4.9 TB/s.
// Keys are converted at the matrix instruction (two values an instruction, the scale of
// the 16 keys applied on the way: bf16 holds the result exactly).  Values become fp16
// relative to v_ref, the scale of the first blocks (raised, rarely, to what fp16
// holds); probabilities go to the matrix instruction as fp16 hi + lo, taken against a
// reference 2^6 below the max, so that hi + lo keep 22 bits down to 2^-9 of the max and
// 2^-31 of it below.
constexpr float kRef8 = 6.f, kRaise8 = 14.f;  // below the max; raised when a score is further above it (fp16 ends at 2^16)
template <int F>
__device__ void decode8_wg(const AttnArgs &a, int w, char *smem, int (*s_pages_g)[kPageWindow], DecSeg (*s_seg_g)[kMaxSeg],
                           int *s_gbar) {
    const int tid = item_tid(), lane = tid & 63;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = wv >> 2, gw = wv & 3, gtid = tid & 255;  // wave group, wave and thread inside it
    const int g = lane >> 4, h = lane & 15;
    const int S = a.dec_unit_tiles;
    const int v = 2 * w + grp;  // this group's share of the tile list
    const int R0 = v * S, R1 = min(R0 + S, a.dec_total_tiles);
    DecSeg *const s_seg = s_seg_g[grp];
    int *const s_pages = s_pages_g[grp];
    const int nseg = R0 < R1 ? find_unit<F>(a, R0, R1, s_seg, gw == 0) : 0;
    if (tid < 2) s_gbar[tid] = 0;
    TRACE(1);
    __syncthreads();
    char *const slots = smem + grp * kDec8GroupBytes;
    char *const s_X = smem + 2 * kDec8GroupBytes + grp * kDec8XBytes;
    char *const s_scale = smem + 2 * (kDec8GroupBytes + kDec8XBytes) + grp * kDec8ScaleBytes;
    float *const s_stat = reinterpret_cast<float *>(smem + 2 * (kDec8GroupBytes + kDec8XBytes + kDec8ScaleBytes) + grp * kDec8StatBytes);
    int *const s_sign = reinterpret_cast<int *>(s_stat + 4 * kHeads);  // [wave]: 1 a score far above the reference, 2 one not finite
    const uint32_t ring = lds_addr(slots), scales = lds_addr(s_scale);
    Cursor8 prod{0, -1, DecSeg{}};
    if (nseg > 0) prod.sg = load_seg(s_seg, 0);
    Cursor8 cons = prod;
    Source8 next{};  // of unit u + 1 while unit u is computed (if prod is inside the share)
    const auto find_next = [&] { next = find_source8<F>(a, prod, s_pages, gw, lane); };
    const auto issue = [&](int u) {
        issue8(next, ring + (u & 1) * kDec8SlotBytes, scales + (u & 1) * 16, gw, lane);
        advance8(prod, s_seg, nseg);
    };
    if (nseg > 0) {
        find_next();
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
    if (nseg == 0) return;  // this group has no share (the other one may)
    find_next();
    issue(1);
    if (prod.j < nseg) find_next();
    int epoch = 0;
    int *const gbar = s_gbar + grp;
    TRACE(2);
    TRACE_VAL(8, 1000000ull * 2 + nseg + (R1 - R0) / 2);

    u32x4 qreg[18];  // dims 64 (s / 2) + 16 g + 8 (s & 1) .. + 7 of step s: a lane's 16-byte piece of a key feeds two steps
    f32x4 acc[8];
#pragma unroll
    for (int mt = 0; mt < 8; ++mt) acc[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_ref = kNegInf, l_run = 0.f;
    float v_ref = 0.f, v_inv = 0.f;  // 0: no block read yet
    bool first = true;               // the unit to come is the first of its segment
    // value operand: slots 8 g + 4 kt + i of a tile hold keys 16 kt + 4 g + i, as the probabilities do
    const int tr = (lane & 15) >> 1, tr_key = 4 * g + (tr & 3) + 16 * (tr >> 2);

    TRACE(3);
    for (int u = 0; cons.j < nseg; ++u) {
        TRACE_TILE(u, 10);
        wait_dma_all();                            // unit u
        group_barrier(gbar, epoch, a.spin_limit);  // landed for all four waves; the other slot is free
        const char *slot = slots + (u & 1) * kDec8SlotBytes;
        if (cons.t < 0) {  // a new request: its query block
            const char *q = slot + h * kRowBytes + 32 * g;
#pragma unroll
            for (int s = 0; s < 18; ++s) qreg[s] = *reinterpret_cast<const u32x4 *>(q + 128 * (s >> 1) + 16 * (s & 1));
            if (u > 0 && prod.j < nseg) {
                issue(u + 1);
                if (prod.j < nseg) find_next();
            }
            advance8(cons, s_seg, nseg);
            continue;
        }
        TRACE_TILE(u, 11);
        const DecSeg sg = cons.sg;
        const SegKeys<has_window<F>> sk(a, sg);
        const bool two = cons.t + 1 < sg.t1;
        const int kb[2] = {sk.key(cons.t * kDecKeys), sk.key((cons.t + 1) * kDecKeys)};
        // this wave's 16 keys (block gw) and the scales of the unit's four blocks, in flight over the next unit's DMAs
        const char *const kp = slot + (gw >> 1) * kTile8Bytes + tile8_off(16 * (gw & 1) + h, g);
        u32x4 av[9];
#pragma unroll
        for (int j = 0; j < 9; ++j) av[j] = *reinterpret_cast<const u32x4 *>(kp + kQuad8 * j);
        const u32x4 wd = *reinterpret_cast<const u32x4 *>(s_scale + (u & 1) * 16);
        const bool issued = u > 0 && prod.j < nseg;
        if (issued) issue(u + 1);
        // scales of the values, and the largest of the blocks that the row sees (a scale that is no number counts for none: its
        // block is not seen, or its scores are not finite; a tile that is not there has any bits, a sign among them)
        float sc[4], most = 0.f;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            const int first = kb[kt >> 1] + 16 * (kt & 1);
            sc[kt] = __uint_as_float(wd[kt] << 16 & 0x7fffffffu);
            sc[kt] = sc[kt] < INFINITY ? sc[kt] : 0.f;
            const bool seen = (kt < 2 || two) && (!has_window<F> || first + 15 > sg.p - a.band.window || first < a.band.sinks);
            most = fmaxf(most, seen ? sc[kt] : 0.f);
        }
        const uint32_t w_mine = gw == 0 ? wd[0] : gw == 1 ? wd[1] : gw == 2 ? wd[2] : wd[3];
        const float e_mine = __uint_as_float(w_mine << 16), r_mine = __uint_as_float(w_mine & 0xffff0000u);
        // scores x[i]: key 16 gw + 4 g + i of the unit, head h
        f32x4 x, sb = {0.f, 0.f, 0.f, 0.f};
        x = sb;
#pragma unroll
        for (int j = 0; j < 9; ++j) {
            const float s = j < 8 ? e_mine : r_mine;  // (the last quad: the rope dims)
            x = mfma_bf16(bf16_of_e4m3x8(av[j][0], av[j][1], s), qreg[2 * j], x);
            sb = mfma_bf16(bf16_of_e4m3x8(av[j][2], av[j][3], s), qreg[2 * j + 1], sb);
        }
        x = x + sb;
        bool careful = any_not_finite(x);
        float mt = kNegInf;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = kb[gw >> 1] + 16 * (gw & 1) + 4 * g + i;
            x[i] = (gw < 2 || two) && row_sees<F>(a, key, sg.p) ? x[i] * a.scale_log2 : kNegInf;
            mt = fmaxf(mt, x[i]);
        }
        // probabilities of this wave's keys against the reference so far, hi and lo, for all four waves
        float ps = 0.f;
        const auto probabilities = [&] {
            float p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = x[i] == kNegInf ? 0.f : __builtin_amdgcn_exp2f(x[i] - m_ref);
            ps = (p[0] + p[1]) + (p[2] + p[3]);
            const f16x2 h0 = {(_Float16)p[0], (_Float16)p[1]}, h1 = {(_Float16)p[2], (_Float16)p[3]};
            *reinterpret_cast<u32x4 *>(s_X + (gw * 64 + lane) * 16) =
                u32x4{__builtin_bit_cast(uint32_t, h0), __builtin_bit_cast(uint32_t, h1),
                      f16x2_bits(p[0] - (float)h0[0], p[1] - (float)h0[1]), f16x2_bits(p[2] - (float)h1[0], p[3] - (float)h1[1])};
        };
        // the reference for all four waves, from their maxima
        const auto raise = [&] {
            mt = wave_max16(mt);
            if (g == 0) s_stat[gw * kHeads + h] = mt;
            group_barrier(gbar, epoch, a.spin_limit);
            mt = fmaxf(fmaxf(s_stat[h], s_stat[kHeads + h]), fmaxf(s_stat[2 * kHeads + h], s_stat[3 * kHeads + h]));
            return fmaxf(m_ref, mt - kRef8);
        };
        if (first) m_ref = raise();
        probabilities();
        const bool above = !first && __builtin_amdgcn_ballot_w64(mt > m_ref + kRaise8) != 0;
        first = false;
        if (lane == 0) s_sign[gw] = (above ? 1 : 0) | (careful ? 2 : 0);
        // values of this wave's 128 dims, before the probabilities are complete
        u32x2 vraw[2][8];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int m = 0; m < 8; ++m)
                vraw[k][m] = lds_read_tr8(slot + k * kTile8Bytes + kQuad8 * (2 * gw + (m >> 2)) + tile8_off(tr_key, m & 3) + 8 * (lane & 1));
        group_barrier(gbar, epoch, a.spin_limit);  // probabilities complete
        TRACE_TILE(u, 12);
        int signs = s_sign[0] | s_sign[1] | s_sign[2] | s_sign[3];
        u32x4 pb[4];  // of block kt: hi (two words), lo
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) pb[kt] = *reinterpret_cast<const u32x4 *>(s_X + (kt * 64 + lane) * 16);
        signs = __builtin_amdgcn_readfirstlane(signs);
        if ((signs & 1) != 0) {
            // a score far above the reference (rarely): raised, and the probabilities once more
            const float m_new = raise();
            const float alpha = (m_ref == kNegInf) ? 0.f : exp2f(m_ref - m_new);
#pragma unroll
            for (int m = 0; m < 8; ++m) acc[m] = acc[m] * alpha;
            l_run *= alpha;
            m_ref = m_new;
            probabilities();
            group_barrier(gbar, epoch, a.spin_limit);
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) pb[kt] = *reinterpret_cast<const u32x4 *>(s_X + (kt * 64 + lane) * 16);
        }
        l_run += ps;
        if ((signs & 2) != 0) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int m = 0; m < 8; ++m) vraw[k][m] = u32x2{finite_e4m3x4(vraw[k][m][0]), finite_e4m3x4(vraw[k][m][1])};
        }
        // the reference of the values (the same decision in every wave)
        if (__builtin_amdgcn_ballot_w64(most > 128.f * v_ref) != 0) {  // 448 2^7 = 57344
            const float f = v_ref / most;  // (0 at a segment's start)
            v_ref = most;
            v_inv = 1.f / most;
#pragma unroll
            for (int m = 0; m < 8; ++m) acc[m] = acc[m] * f;
        }
        TRACE_TILE(u, 13);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float s0 = fminf(sc[2 * k] * v_inv, 128.f), s1 = fminf(sc[2 * k + 1] * v_inv, 128.f);
            const u32x4 ph = {pb[2 * k][0], pb[2 * k][1], pb[2 * k + 1][0], pb[2 * k + 1][1]};
            const u32x4 pl = {pb[2 * k][2], pb[2 * k][3], pb[2 * k + 1][2], pb[2 * k + 1][3]};
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const u32x4 vop = f16_of_e4m3x8(vraw[k][m][0], vraw[k][m][1], s0, s1);
                acc[m] = mfma_f16(vop, ph, acc[m]);
                acc[m] = mfma_f16(vop, pl, acc[m]);
            }
        }
        if (issued && prod.j < nseg) find_next();  // (beside the last products)

        TRACE_TILE(u, 14);
        const int jseg = cons.j;
        advance8(cons, s_seg, nseg);
        if (cons.j != jseg) {  // the segment's last tile: finish it
            l_run = wave_sum16(l_run);  // of this wave's keys
            if (g == 0) s_stat[gw * kHeads + h] = l_run;
            group_barrier(gbar, epoch, a.spin_limit);
            const float l_tot = (s_stat[h] + s_stat[kHeads + h]) + (s_stat[2 * kHeads + h] + s_stat[3 * kHeads + h]);
            if (sg.t0 == 0 && sg.t1 == dec_tiles<F>(a, sg.p, 1)) {
                const float inv = 1.f / l_tot;
#pragma unroll
                for (int mt2 = 0; mt2 < 8; ++mt2)
                    store_out4(a, sg.row, h, gw * 128 + mt2 * 16 + 4 * g, acc[mt2] * inv * v_ref);
                if (a.lse && gw == 0 && g == 0) a.lse[(size_t)sg.row * kHeads + h] = (m_ref + log2f(l_tot)) * kLn2;
            } else if (a.ws_dec_o != nullptr) {
                const size_t slot_id = 2 * (size_t)v + (jseg == 0 ? 0 : 1);
                float *po = a.ws_dec_o + (slot_id * kHeads + h) * kDv;
                const float inv = inv_sum(l_tot);
#pragma unroll
                for (int mt2 = 0; mt2 < 8; ++mt2)
                    *reinterpret_cast<f32x4 *>(po + gw * 128 + mt2 * 16 + 4 * g) = acc[mt2] * inv * v_ref;
                if (gw == 0 && g == 0) {
                    a.ws_dec_ml[(slot_id * kHeads + h) * 2 + 0] = partial_max(m_ref, l_tot);
                    a.ws_dec_ml[(slot_id * kHeads + h) * 2 + 1] = l_tot;
                }
            }
#pragma unroll
            for (int mt2 = 0; mt2 < 8; ++mt2) acc[mt2] = f32x4{0.f, 0.f, 0.f, 0.f};
            m_ref = kNegInf;
            l_run = 0.f;
            v_ref = 0.f;
            first = true;
        }
    }
    TRACE(4);
}
