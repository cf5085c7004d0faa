// The compact cache's C entries when host memory runs out: every allocation in them throws, in turn.
// Launch functions and device queries are stubbed as in form_harness.cpp.  Prints "name n" per entry, n the
// allocations that were made to fail (each has to come back as an error with a message), and aborts otherwise.
#define main form_harness_main
#include "form_harness.cpp"
#undef main

#include <cstdio>
#include <cstdlib>
#include <new>

static long long g_fail_at = -1;  // allocations until the one that throws
void *operator new(size_t n) {
    if (g_fail_at >= 0 && g_fail_at-- == 0) throw std::bad_alloc();
    if (void *p = std::malloc(n)) return p;
    throw std::bad_alloc();
}
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, size_t) noexcept { std::free(p); }

template <class Call>
static void run(const char *name, const Call &call) {
    long long n = 0;
    for (;; ++n) {
        mla_debug_set(MLA_DEBUG_CHUNK_KEYS, 64 * (1 + (int)(n % 4)));  // another plan each time
        g_fail_at = n;
        const bool ok = call();
        const bool fired = g_fail_at < 0;
        g_fail_at = -1;
        if (!fired) break;
        if (ok || mla_last_error()[0] == 0) std::abort();
    }
    std::printf("%s %lld\n", name, n);
}

int main() {
    const int32_t q[3] = {1, 40, 1}, p[3] = {700, 90, 5};
    alignas(16) static int32_t dev[64];
    alignas(16) static char mem[1 << 20];
    mla_batch b{};
    b.num_reqs = 3;
    b.page_size = 16;
    b.num_pages = 64;
    b.max_pages_per_req = 64;
    b.q_lens = q;
    b.prefix_lens = p;
    b.cu_q_dev = b.prefix_lens_dev = b.block_table_dev = dev;
    const mla_cache8 c{reinterpret_cast<uint8_t *>(mem), reinterpret_cast<uint16_t *>(mem)};
    const mla_window w{100, 4};
    const uint16_t *x = reinterpret_cast<const uint16_t *>(mem);
    static char ws[64 << 20];
    run("mixed_step_attn8_workspace_bytes", [&] { return mixed_step_attn8_workspace_bytes(&b, &w) != 0; });
    run("mixed_step_attn_window_workspace_bytes", [&] { return mixed_step_attn_window_workspace_bytes(&b, &w) != 0; });
    run("mixed_step_attn8", [&] {
        return mixed_step_attn8(&b, x, &c, &w, 0.1f, mem, MLA_OUT_F32, nullptr, (void *)(((uintptr_t)ws + 255) & ~(uintptr_t)255), sizeof ws - 256, nullptr) == MLA_OK;
    });
    run("mixed_step_attn_window", [&] {
        return mixed_step_attn_window(&b, x, x, &w, 0.1f, mem, MLA_OUT_F32, nullptr, (void *)(((uintptr_t)ws + 255) & ~(uintptr_t)255), sizeof ws - 256, nullptr) == MLA_OK;
    });
    run("append_latent_kv8", [&] { return append_latent_kv8(&b, x, 1e4f, &c, nullptr) == MLA_OK; });
    run("append_latent_kv_rope", [&] { return append_latent_kv_rope(&b, x, 1e4f, reinterpret_cast<uint16_t *>(mem), nullptr) == MLA_OK; });
    return 0;
}
