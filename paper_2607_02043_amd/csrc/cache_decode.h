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

// DMA of a unit.  Of two tiles every wave issues ten instructions: five of each (see
// dma_tile8), the waves' parts exchanged in the second one.
template <int F>
__device__ __forceinline__ void issue_unit8(const AttnArgs &a, const DecSeg &sg, int t, const int *s_pages, uint32_t slot,
                                            uint32_t scale_slot, int wv, int lane) {
    asm volatile("" : "+v"(lane));  // (no address is kept across the units)
    if (t < 0) {
        const char *qb = reinterpret_cast<const char *>(a.q + (size_t)sg.row * kHeads * kDqk) + lane * 16;
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            const int j = i * 4 + wv;
            if (j < kTile8Bytes / 1024) lds_dma16(qb + j * 1024, __builtin_amdgcn_readfirstlane(slot + j * 1024));
        }
        return;
    }
    const SegKeys<has_window<F>> sk(a, sg);
    const auto page_of = [&](int key) { return s_pages[min(sk.window_entry(sg, key, a.log2_page), kPageWindow - 1)]; };
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (t + h >= sg.t1) break;
        const int kbase = sk.key((t + h) * kDecKeys), w = wv ^ (2 * h);
        const auto slot_of = [&](int key) {  // pool slot
            const int k = min(key, sg.p);
            return (size_t)page_of(k) * a.page_size + (k & (a.page_size - 1));
        };
        if (a.page_size >= kDecKeys && kbase + kDecKeys - 1 <= sg.p) {
            const size_t first = (size_t)__builtin_amdgcn_readfirstlane(page_of(kbase)) * a.page_size + (kbase & (a.page_size - 1));
            dma_tile8(a.kv8 + first * kDqk, tile8_key(w, lane) * kDqk + tile8_dims(w, lane), slot + h * kTile8Bytes, w);
        } else {
            dma_tile8(a.kv8 + slot_of(kbase + tile8_key(w, lane)) * kDqk + tile8_dims(w, lane), slot + h * kTile8Bytes, w);
        }
        if (w >= 2) dma_scales8(a, slot_of(kbase + 16 * (w - 2)), scale_slot + 32 * h + 16 * (w - 2), lane);
    }
}

// decode_wg over the 8-bit cache.  Half the bytes a key (578), so a key has half the
// time, and what bounds a group is the chain of a unit: wait, barrier, scores,
// barrier, softmax, values.  Hence units of two tiles, 64 keys a barrier pair: each
// wave scores 16 keys over all dims (nothing is added across waves) and then
// accumulates its 128 value dims over the 64.  (Units of one tile, in a ring of four
// slots: UNIT_FIGURES.)
// Keys are converted at the matrix instruction (two values an instruction, the scale of
// the 16 keys applied on the way: bf16 holds the result exactly).  Values become fp16
// relative to 2^v_exp, the scale of the first blocks (raised, rarely, to what fp16
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
    const uint32_t ring = lds_addr(slots), scales = lds_addr(s_scale);
    Cursor8 prod{0, -1, DecSeg{}};
    if (nseg > 0) prod.sg = load_seg(s_seg, 0);
    Cursor8 cons = prod;
    const auto issue = [&](int u) {
        issue_unit8<F>(a, prod.sg, prod.t, s_pages, ring + (u & 1) * kDec8SlotBytes, scales + (u & 1) * 64, gw, lane);
        advance8(prod, s_seg, nseg);
    };
    if (nseg > 0) {
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
    issue(1);
    int epoch = 0;
    int *const gbar = s_gbar + grp;
    TRACE(2);
    TRACE_VAL(8, 1000000ull * 2 + nseg + (R1 - R0) / 2);

    u32x4 qreg[18];  // dims 64 (s / 2) + 16 g + 8 (s & 1) .. + 7 of step s: a lane's 16-byte piece of a key feeds two steps
    f32x4 acc[8];
#pragma unroll
    for (int mt = 0; mt < 8; ++mt) acc[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_ref = kNegInf, l_run = 0.f;
    constexpr int kNoExp = -1000;
    int v_exp = kNoExp;
    // value operand: slots 8 g + 4 kt + i of a tile hold keys 16 kt + 4 g + i, as the probabilities do
    const int tr = (lane & 15) >> 1, tr_key = 4 * g + (tr & 3) + 16 * (tr >> 2);

    TRACE(3);
    for (int u = 0; cons.j < nseg; ++u) {
        TRACE_TILE(u, 10);
        wait_dma_all();                            // unit u
        group_barrier(gbar, epoch, a.spin_limit);  // landed for all four waves; the other slot is free
        if (u > 0 && prod.j < nseg) issue(u + 1);
        const char *slot = slots + (u & 1) * kDec8SlotBytes;
        if (cons.t < 0) {  // a new request: its query block
            const char *q = slot + h * kRowBytes + 32 * g;
#pragma unroll
            for (int s = 0; s < 18; ++s) qreg[s] = *reinterpret_cast<const u32x4 *>(q + 128 * (s >> 1) + 16 * (s & 1));
            advance8(cons, s_seg, nseg);
            continue;
        }
        TRACE_TILE(u, 11);
        const DecSeg sg = cons.sg;
        const SegKeys<has_window<F>> sk(a, sg);
        const bool two = cons.t + 1 < sg.t1;
        const int kb[2] = {sk.key(cons.t * kDecKeys), sk.key((cons.t + 1) * kDecKeys)};
        // scales of the unit's four key blocks
        int ec[4], er[4], most = kNoExp;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            const int first = kb[kt >> 1] + 16 * (kt & 1), key = min(first, sg.p);
            const int pg = a.page_size >= 64 ? 0 : s_pages[min(sk.window_entry(sg, key, a.log2_page), kPageWindow - 1)];
            const uint32_t wd = __builtin_amdgcn_readfirstlane(
                *reinterpret_cast<const int *>(s_scale + (u & 1) * 64 + 16 * kt + 4 * scale_piece8(a, pg, key)));
            ec[kt] = scale_exponent(wd);
            er[kt] = scale_exponent(wd >> 16);
            // (a block that the row does not see has no say in the reference)
            const bool seen = (kt < 2 || two) && first <= sg.p && (!has_window<F> || first + 15 > sg.p - a.band.window || first < a.band.sinks);
            if (seen && ec[kt] <= kMaxExp8) most = max(most, ec[kt]);
        }
        {
            // scores of key block gw
            const char *kp = slot + (gw >> 1) * kTile8Bytes + tile8_off(16 * (gw & 1) + h, g);
            const int e0 = gw == 0 ? ec[0] : gw == 1 ? ec[1] : gw == 2 ? ec[2] : ec[3];
            const int e1 = gw == 0 ? er[0] : gw == 1 ? er[1] : gw == 2 ? er[2] : er[3];
            u32x4 av[9];
#pragma unroll
            for (int j = 0; j < 9; ++j) av[j] = *reinterpret_cast<const u32x4 *>(kp + kQuad8 * j);
            f32x4 sa = {0.f, 0.f, 0.f, 0.f}, sb = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < 9; ++j) {
                const float s = exp2_bits(j < 8 ? e0 : e1);  // (the last quad: the rope dims)
                sa = mfma_bf16(bf16_of_e4m3x8(av[j][0], av[j][1], s), qreg[2 * j], sa);
                sb = mfma_bf16(bf16_of_e4m3x8(av[j][2], av[j][3], s), qreg[2 * j + 1], sb);
            }
            *reinterpret_cast<f32x4 *>(s_X + (gw * 64 + lane) * 16) = sa + sb;
        }
        // values of this wave's 128 dims, before the scores are complete
        u32x2 vraw[2][8];
        const auto load_values = [&] {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int mt = 0; mt < 8; ++mt)
                    vraw[k][mt] = lds_read_tr8(slot + k * kTile8Bytes + kQuad8 * (2 * gw + (mt >> 2)) + tile8_off(tr_key, mt & 3) + 8 * (lane & 1));
        };
        load_values();
        group_barrier(gbar, epoch, a.spin_limit);  // scores complete
        TRACE_TILE(u, 12);
        // scores of this lane's head: x[kt][i] = key 16 (kt & 1) + 4 g + i of tile kt / 2
        f32x4 x[4];
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) x[kt] = *reinterpret_cast<const f32x4 *>(s_X + (kt * 64 + lane) * 16);
        if (any_not_finite(x[0] + x[1] + x[2] + x[3])) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int mt = 0; mt < 8; ++mt) vraw[k][mt] = u32x2{finite_e4m3x4(vraw[k][mt][0]), finite_e4m3x4(vraw[k][mt][1])};
        }
        float mt = kNegInf;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = kb[kt >> 1] + 16 * (kt & 1) + 4 * g + i;
                x[kt][i] = (kt < 2 || two) && row_sees<F>(a, key, sg.p) ? x[kt][i] * a.scale_log2 : kNegInf;
                mt = fmaxf(mt, x[kt][i]);
            }
        }
        mt = wave_max16(mt);
        // raise the reference of the probabilities, or that of the values (the same decisions in every wave of the group)
        if (__builtin_amdgcn_ballot_w64(mt > m_ref + kRaise8) != 0) {
            const float m_new = fmaxf(m_ref, mt - kRef8);
            const float alpha = (m_ref == kNegInf) ? 0.f : exp2f(m_ref - m_new);
#pragma unroll
            for (int mt2 = 0; mt2 < 8; ++mt2) acc[mt2] = acc[mt2] * alpha;
            l_run *= alpha;
            m_ref = m_new;
        }
        if (v_exp == kNoExp) {
            v_exp = most;
        } else if (most > v_exp + 7) {  // 448 2^7 = 57344
            const float f = exp2_bits(max(v_exp - most, -126));
            v_exp = most;
#pragma unroll
            for (int mt2 = 0; mt2 < 8; ++mt2) acc[mt2] = acc[mt2] * f;
        }
        u32x4 ph[2], pl[2];
        float ps = 0.f;
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                const float p0 = (x[kt][i] == kNegInf) ? 0.f : __builtin_amdgcn_exp2f(x[kt][i] - m_ref);
                const float p1 = (x[kt][i + 1] == kNegInf) ? 0.f : __builtin_amdgcn_exp2f(x[kt][i + 1] - m_ref);
                ps += p0 + p1;
                const f16x2 hi = {(_Float16)p0, (_Float16)p1};
                ph[kt >> 1][2 * (kt & 1) + (i >> 1)] = __builtin_bit_cast(uint32_t, hi);
                pl[kt >> 1][2 * (kt & 1) + (i >> 1)] = f16x2_bits(p0 - (float)hi[0], p1 - (float)hi[1]);
            }
        }
        l_run += ps;
        TRACE_TILE(u, 13);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float s0 = exp2_bits(min(max(ec[2 * k] - v_exp, -126), 7)), s1 = exp2_bits(min(max(ec[2 * k + 1] - v_exp, -126), 7));
#pragma unroll
            for (int mt2 = 0; mt2 < 8; ++mt2) {
                const u32x4 vop = f16_of_e4m3x8(vraw[k][mt2][0], vraw[k][mt2][1], s0, s1);
                acc[mt2] = mfma_f16(vop, ph[k], acc[mt2]);
                acc[mt2] = mfma_f16(vop, pl[k], acc[mt2]);
            }
        }

        TRACE_TILE(u, 14);
        const int jseg = cons.j;
        advance8(cons, s_seg, nseg);
        if (cons.j != jseg) {  // the segment's last tile: finish it
            const float l_tot = wave_sum16(l_run), out_scale = exp2_bits(max(v_exp, -126));
            if (sg.t0 == 0 && sg.t1 == dec_tiles<F>(a, sg.p, 1)) {
                const float inv = out_scale / l_tot;
#pragma unroll
                for (int mt2 = 0; mt2 < 8; ++mt2)
                    store_out4(a, sg.row, h, gw * 128 + mt2 * 16 + 4 * g, acc[mt2] * inv);
                if (a.lse && gw == 0 && g == 0) a.lse[(size_t)sg.row * kHeads + h] = (m_ref + log2f(l_tot)) * kLn2;
            } else if (a.ws_dec_o != nullptr) {
                const size_t slot_id = 2 * (size_t)v + (jseg == 0 ? 0 : 1);
                float *po = a.ws_dec_o + (slot_id * kHeads + h) * kDv;
#pragma unroll
                for (int mt2 = 0; mt2 < 8; ++mt2)
                    *reinterpret_cast<f32x4 *>(po + gw * 128 + mt2 * 16 + 4 * g) = acc[mt2] * out_scale;
                if (gw == 0 && g == 0) {
                    a.ws_dec_ml[(slot_id * kHeads + h) * 2 + 0] = partial_max(m_ref, l_tot);
                    a.ws_dec_ml[(slot_id * kHeads + h) * 2 + 1] = l_tot;
                }
            }
#pragma unroll
            for (int mt2 = 0; mt2 < 8; ++mt2) acc[mt2] = f32x4{0.f, 0.f, 0.f, 0.f};
            m_ref = kNegInf;
            l_run = 0.f;
            v_exp = kNoExp;
        }
    }
    TRACE(4);
}
