// Attention over the 8-bit cache (include/mla_cache.h):
// device code, part of mla_kernels.hip (its helpers and namespace).
#pragma once

// The definition, one workgroup a row: tiles of 16 keys become fp32 in LDS, 256
// threads form the 16 x 16 scores, and each thread accumulates two value dims
// of all heads under a running max and sum per head.  Invisible keys are zeros in
// LDS and never touched in memory.
__global__ __launch_bounds__(kThreads) void rows8_kernel(AttnArgs a) {
    constexpr int kT = 16, kStride = kDqk + 4;
    __shared__ float s_q[kHeads][kStride], s_k[kT][kStride], s_p[kHeads][kT], s_c[kHeads], s_m[kHeads], s_l[kHeads];
    const int tid = threadIdx.x, row = blockIdx.x;
    const int r = find_request(a.cu_q, a.num_reqs, row, tid & 63);
    const int p = a.prefix[r] + row - a.cu_q[r];
    if (p < 0 || row >= a.cu_q[a.num_reqs]) return;
    const int W = a.band.window > 0 ? a.band.window : INT_MAX;
    for (int u = tid; u < kHeads * kDqk; u += kThreads)
        s_q[u / kDqk][u % kDqk] = bf16_bits_to_float(a.q[(size_t)row * kHeads * kDqk + u]);
    if (tid < kHeads) {
        s_m[tid] = kNegInf;
        s_l[tid] = 0.f;
    }
    float acc[kHeads][2] = {};
    const int lo = max(p - W + 1, 0);
    for (int k0 = 0; k0 <= p; k0 += kT) {
        if (k0 >= a.band.sinks && k0 + kT <= lo) {
            k0 = (lo & -kT) - kT;
            continue;
        }
        const auto seen = [&](int key) { return key <= p && (key >= lo || key < a.band.sinks); };
        __syncthreads();
        for (int u = tid; u < kT * kDqk; u += kThreads) {
            const int key = k0 + u / kDqk, d = u % kDqk;
            float v = 0.f;
            if (seen(key)) {
                const int lp = key >> a.log2_page;
                int page = lp < a.max_pages ? a.bt[(size_t)r * a.max_pages + lp] : -1;
                if ((unsigned)page >= (unsigned)a.num_pages) {
                    raise_flag(kFlagBadPage);
                    page = 0;
                }
                const size_t slot = (size_t)page * a.page_size + (key & (a.page_size - 1));
                const float sc = bf16_bits_to_float(a.kv8_scales[slot / kBlock8 * 2 + (d >= kDv)]);
                v = __builtin_amdgcn_cvt_f32_fp8(a.kv8[slot * kDqk + d], 0) * sc;
            }
            s_k[u / kDqk][d] = v;
        }
        __syncthreads();
        {
            const int h = tid >> 4, k = tid & 15;
            float s = 0.f;
            for (int d = 0; d < kDqk; ++d) s += s_q[h][d] * s_k[k][d];
            s = seen(k0 + k) ? s * a.scale_log2 : kNegInf;
            float m = s;
            for (int off = 8; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
            const float m_old = s_m[h], m_new = fmaxf(m_old, m);
            const float pr = s == kNegInf ? 0.f : exp2f(s - m_new);
            float l = pr;
            for (int off = 8; off >= 1; off >>= 1) l += __shfl_xor(l, off);
            s_p[h][k] = pr;
            if (k == 0) {
                s_c[h] = m_old == kNegInf ? 0.f : exp2f(m_old - m_new);
                s_l[h] = s_l[h] * s_c[h] + l;
                s_m[h] = m_new;
            }
        }
        __syncthreads();
        for (int h = 0; h < kHeads; ++h) {
            float o0 = acc[h][0] * s_c[h], o1 = acc[h][1] * s_c[h];
            for (int k = 0; k < kT; ++k) {
                if (s_p[h][k] == 0.f) continue;
                o0 += s_p[h][k] * s_k[k][2 * tid];
                o1 += s_p[h][k] * s_k[k][2 * tid + 1];
            }
            acc[h][0] = o0;
            acc[h][1] = o1;
        }
    }
    __syncthreads();
    for (int h = 0; h < kHeads; ++h) {
        const float inv = 1.f / s_l[h];
        const size_t off = ((size_t)row * kHeads + h) * kDv + 2 * tid;
        if (a.out_bf16)
            *reinterpret_cast<uint32_t *>(reinterpret_cast<uint16_t *>(a.out) + off) =
                bf16_bits(acc[h][0] * inv) | (bf16_bits(acc[h][1] * inv) << 16);
        else
            *reinterpret_cast<float2 *>(reinterpret_cast<float *>(a.out) + off) = float2{acc[h][0] * inv, acc[h][1] * inv};
    }
    if (a.lse && tid < kHeads) a.lse[(size_t)row * kHeads + tid] = (s_m[tid] + log2f(s_l[tid])) * kLn2;
}
