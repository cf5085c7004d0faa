// Appends of the compact latent cache (include/mla_cache.h): device code, part of
// mla_kernels.hip (its helpers and namespace).
#pragma once

// ------------------------------------------------------- rotation on the way
// Sine and cosine of position t times base^(-2 i / 64): the angle in turns, in
// 64 bits, so that only its fraction is rounded to fp32 (2^-25 turns, 2e-7 rad, at
// any position); the rest is fp32.  The turns per position of the 32 pairs come with
// the launch (RopeTable): their powers in 64 bits would be half of a small append.
struct SinCos {
    float sn, cs;
};
__device__ __forceinline__ SinCos rope_angle(int t, double turns) {
    const double a = (double)t * turns;
    const float f = (float)(a - floor(a));
    SinCos r;
    r.sn = sinpif(2.f * f);
    r.cs = cospif(2.f * f);
    return r;
}

// One wavefront a row, as append_kernel; lanes 0 .. 31 rotate a pair each.
// Bound by latency like it: lengths -> page id -> store, with the row's loads and
// the angles beside them (4 tokens 2.0 us, 4160 tokens 4.5 us, 2.1 TB/s).
__global__ __launch_bounds__(kThreads) void append_rope_kernel(AppendArgs a, RopeTable rope) {
    const int lane = threadIdx.x & 63;
    const int row = blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= a.num_rows) return;
    const u32x4 va = reinterpret_cast<const u32x4 *>(a.src + (size_t)row * kDqk)[lane];
    const int i = lane & 31;
    const uint32_t x = *reinterpret_cast<const uint32_t *>(a.src + (size_t)row * kDqk + kDv + 2 * i);
    const int total = a.cu_q[a.num_reqs];
    const int r = find_request(a.cu_q, a.num_reqs, row, lane);
    const int t = a.prefix[r] + (row - a.cu_q[r]);
    const int lp = t >> a.log2_page;
    const int page = row < total && t >= 0 && lp < a.max_pages ? a.bt[(size_t)r * a.max_pages + lp] : -1;
    if ((unsigned)page >= (unsigned)a.num_pages) {
        raise_flag(kFlagBadPage);
        return;
    }
    const SinCos w = rope_angle(t, rope.turns[i]);
    const float x0 = bf16_bits_to_float(x & 0xffffu), x1 = bf16_bits_to_float(x >> 16);
    uint16_t *dst = a.kv + ((size_t)page * a.page_size + (t & (a.page_size - 1))) * kDqk;
    reinterpret_cast<u32x4 *>(dst)[lane] = va;
    if (lane < 32)
        *reinterpret_cast<uint32_t *>(dst + kDv + 2 * i) =
            bf16_bits(x0 * w.cs - x1 * w.sn) | (bf16_bits(x0 * w.sn + x1 * w.cs) << 16);
}

// ------------------------------------------------------------ 8-bit append
// Scales are powers of two, so they are handled as exponents: 2^E with E the
// smallest integer in [kMinExp8, kMaxExp8] for which amax 2^-E <= 448 = 1.75 2^8.
// amax = m 2^e with m in [1, 2) gives E = e - 8, one more if m > 1.75, which is
// when 0x1fffff added to the bits carries into the exponent field.
__device__ __forceinline__ int block_exponent(float amax) {
    const int e = (int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 127 - 8;
    return min(max(e, kMinExp8), kMaxExp8);
}
// |x|, and 0 for NaN and infinities, which do not count for a scale.
__device__ __forceinline__ float finite_abs(float x) {
    const float v = fabsf(x);
    return v < INFINITY ? v : 0.f;
}
// Largest code value at a scale of 2^e: 448, at 2^120 the largest below 2^8 (codes
// from 256 on stand for 2^128 and more there, which neither bf16 nor fp32 holds).
__device__ __forceinline__ float largest_code(int e) { return e < kMaxExp8 ? 448.f : 240.f; }
// Four values to e4m3 (nearest even, none beyond `most`), non-finite ones to NaN.
__device__ __forceinline__ uint32_t pack_e4m3(float x0, float x1, float x2, float x3, float s, float most) {
    const auto f = [&](float x) { return fabsf(x) < INFINITY ? fminf(fmaxf(x * s, -most), most) : NAN; };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f(x0), f(x1), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f(x2), f(x3), w, true);
}

// Blocks of 16 tokens that a request's new tokens p .. p + c - 1 touch.
struct Block8Count {
    __device__ int operator()(int p, int c) const { return c > 0 ? ((p + c - 1) >> 4) - (p >> 4) + 1 : 0; }
};

// Bound by latency: the lengths, then the page id and the rows, then the old scales,
// then the stores, a round trip each (256 tokens of 256 requests 5.2 us, with the
// turns of the rotation found in the kernel 0.4 more).
// One workgroup a block: thread (wave w, lane l) takes the compressed chunk l
// (8 dims) of its rows w, w + 4, .., and the first 128 threads one rope chunk (4
// pairs) each.  The two maxima meet in LDS; then everything is scaled, rounded and
// stored, and a block with earlier tokens whose scale grew rounds those again.
__global__ __launch_bounds__(kThreads) void append8_kernel(Append8Args a, RopeTable rope_table) {
    __shared__ float s_max[4][2];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rr = tid >> 3, rc = tid & 7;  // rope row and chunk of this thread
    double turns[4] = {0.0, 0.0, 0.0, 0.0};
    if (a.rotate) {
#pragma unroll
        for (int k = 0; k < 4; ++k) turns[k] = rope_table.turns[4 * rc + k];
    }
    Located lc;
    if (!locate_item(blockIdx.x, a.num_reqs, ReqLens{a.cu_q, a.prefix, false}, Block8Count{}, lc)) return;
    const int b = (lc.p >> 4) + lc.local;                                     // logical block of the request
    const int t0 = max(lc.p, b * kBlock8), t1 = min(lc.p + lc.c, (b + 1) * kBlock8);  // its new tokens
    const int row0 = lc.row0 + t0 - lc.p, n = t1 - t0;
    if (lc.p < 0 || row0 < 0 || row0 + n > a.num_rows) {  // device lengths that disagree with the host's
        if (tid == 0) raise_flag(kFlagBadPage);
        return;
    }
    // the page id and the new rows in one round of loads
    const int lp = (b * kBlock8) >> a.log2_page;
    const int page = lp < a.max_pages ? a.bt[(size_t)lc.r * a.max_pages + lp] : -1;
    u32x4 vc[4], vr = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        vc[i] = u32x4{0u, 0u, 0u, 0u};
        if (4 * i + wv < n) vc[i] = reinterpret_cast<const u32x4 *>(a.src + (size_t)(row0 + 4 * i + wv) * kDqk)[lane];
    }
    const bool rope = rr < n;  // (n <= 16: threads 0 .. 127)
    if (rope) vr = reinterpret_cast<const u32x4 *>(a.src + (size_t)(row0 + rr) * kDqk + kDv)[rc];
    if ((unsigned)page >= (unsigned)a.num_pages) {
        if (tid == 0) raise_flag(kFlagBadPage);
        return;
    }
    const size_t slot0 = (size_t)page * a.page_size + ((b * kBlock8) & (a.page_size - 1));  // pool slot of the block
    uint8_t *const blk = a.data + slot0 * kDqk;
    uint32_t *const scale = reinterpret_cast<uint32_t *>(a.scales) + slot0 / kBlock8;
    const int held = t0 - b * kBlock8;  // earlier tokens of the block

    const uint32_t old = held > 0 ? *scale : 0u;

    float xr[8], mc = 0.f, mr = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float x0 = bf16_bits_to_float(vr[k] & 0xffffu), x1 = bf16_bits_to_float(vr[k] >> 16);
        xr[2 * k] = x0;
        xr[2 * k + 1] = x1;
        if (a.rotate && rope) {
            const SinCos w = rope_angle(t0 + rr, turns[k]);
            xr[2 * k] = x0 * w.cs - x1 * w.sn;
            xr[2 * k + 1] = x0 * w.sn + x1 * w.cs;
        }
        mr = fmaxf(mr, fmaxf(finite_abs(xr[2 * k]), finite_abs(xr[2 * k + 1])));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            mc = fmaxf(mc, fmaxf(finite_abs(bf16_bits_to_float(vc[i][k] & 0xffffu)), finite_abs(bf16_bits_to_float(vc[i][k] >> 16))));
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        mc = fmaxf(mc, __shfl_xor(mc, off));
        mr = fmaxf(mr, __shfl_xor(mr, off));
    }
    if (lane == 0) {
        s_max[wv][0] = mc;
        s_max[wv][1] = mr;
    }
    __syncthreads();
    int e[2], was[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        e[k] = block_exponent(fmaxf(fmaxf(s_max[0][k], s_max[1][k]), fmaxf(s_max[2][k], s_max[3][k])));
        was[k] = held > 0 ? scale_exponent(old >> (16 * k)) : e[k];
        e[k] = min(max(e[k], was[k]), kMaxExp8);
    }
    if (tid == 0) *scale = (uint32_t)(e[0] + 127) << 7 | (uint32_t)(e[1] + 127) << 23;
    // earlier tokens, if a part's scale grew
    if (held > 0 && (e[0] != was[0] || e[1] != was[1])) {
        for (int u = tid; u < held * (kDqk / 4); u += kThreads) {
            const int k = u % (kDqk / 4) < kDv / 4 ? 0 : 1;
            if (e[k] == was[k]) continue;
            uint32_t *const w = reinterpret_cast<uint32_t *>(blk) + u;
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)*w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)*w, true);
            *w = pack_e4m3(lo[0], lo[1], hi[0], hi[1], exp2_bits(max(was[k] - e[k], -126)), largest_code(e[k]));
        }
    }
    const float sc = exp2_bits(-e[0]), sr = exp2_bits(-e[1]), top_c = largest_code(e[0]), top_r = largest_code(e[1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (4 * i + wv >= n) break;
        float x[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[2 * k] = bf16_bits_to_float(vc[i][k] & 0xffffu);
            x[2 * k + 1] = bf16_bits_to_float(vc[i][k] >> 16);
        }
        reinterpret_cast<u32x2 *>(blk + (size_t)(held + 4 * i + wv) * kDqk)[lane] =
            u32x2{pack_e4m3(x[0], x[1], x[2], x[3], sc, top_c), pack_e4m3(x[4], x[5], x[6], x[7], sc, top_c)};
    }
    if (rope)
        reinterpret_cast<u32x2 *>(blk + (size_t)(held + rr) * kDqk + kDv)[rc] =
            u32x2{pack_e4m3(xr[0], xr[1], xr[2], xr[3], sr, top_r), pack_e4m3(xr[4], xr[5], xr[6], xr[7], sr, top_r)};
}
