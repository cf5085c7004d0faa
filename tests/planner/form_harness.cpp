// Host-only harness around the work planner's forms (windows, the 8-bit cache); the launch functions are
// stubbed and the device queries answer for a 256-CU device, as in plan_harness.cpp.  Input on stdin, one batch a line:
//   eight window sinks page_size forced_keys forced_unit forced_first R q_0 p_0 q_1 p_1 ...
// Output, one line a batch, from the planner that consecutive calls share:
//   ok ks n_chunk_items n_dec_items unit_tiles dec_total grid merge_many split_rows split_chunk_rows chunk_merge_wgs rev bytes warm shifts..
// (shifts: band_shift of every request's first row) or "err <status> <message>".
#include <hip/hip_runtime.h>

static hipError_t harness_get_device(int *d) {
    *d = 0;
    return hipSuccess;
}
static hipError_t harness_get_attribute(int *v, hipDeviceAttribute_t, int) {
    *v = 256;
    return hipSuccess;
}
#define hipGetDevice harness_get_device
#define hipDeviceGetAttribute harness_get_attribute
#include "../../paper_2607_02043_amd/csrc/mla_api.cpp"
#undef hipGetDevice
#undef hipDeviceGetAttribute
#include "../../paper_2607_02043_amd/csrc/cache_api.cpp"

#include <iostream>
#include <sstream>
#include <string>

namespace mla {
hipError_t launch_append(const AppendArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_append_rope(const AppendArgs &, const RopeTable &, hipStream_t) { return hipSuccess; }
hipError_t launch_append8(const Append8Args &, const RopeTable &, hipStream_t) { return hipSuccess; }
hipError_t launch_attention(const AttnArgs &, hipStream_t) { return hipSuccess; }
hipError_t launch_combine(const AttnArgs &, hipStream_t) { return hipSuccess; }
hipError_t read_flags(int *flags, bool) {
    *flags = 0;
    return hipSuccess;
}
hipError_t noalloc_scratch(void **ptr) {
    alignas(256) static char fake[256];
    *ptr = fake;
    return hipSuccess;
}
}  // namespace mla

int main() {
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        int eight = 0, P = 0, keys = 0, unit = 0, first = 0, R = 0;
        mla_window w{};
        in >> eight >> w.window >> w.sinks >> P >> keys >> unit >> first >> R;
        std::vector<int32_t> q(R), p(R);
        long long maxk = 1;
        for (int i = 0; i < R; ++i) {
            in >> q[i] >> p[i];
            maxk = std::max<long long>(maxk, (long long)q[i] + p[i]);
        }
        mla_debug_set(MLA_DEBUG_CHUNK_KEYS, keys);
        mla_debug_set(MLA_DEBUG_DEC_UNIT, unit);
        mla_debug_set(MLA_DEBUG_DEC_FIRST, first);
        static const int32_t fake = 0;  // device pointers are never dereferenced by the planner
        mla_batch b{};
        b.num_reqs = R;
        b.page_size = P;
        b.num_pages = 1 << 30;
        b.max_pages_per_req = (int)((maxk + P - 1) / P);
        b.q_lens = q.data();
        b.prefix_lens = p.data();
        b.cu_q_dev = &fake;
        b.prefix_lens_dev = &fake;
        b.block_table_dev = &fake;
        Shape sh;
        Plan pl{};
        mla::Form form;
        int st = check_batch(&b, &sh);
        if (st == MLA_OK && (eight != 0 || w.window > 0)) st = make_form(&b, eight != 0, w.window > 0 ? &w : nullptr, &form);
        if (st == MLA_OK) st = make_plan(&b, sh, &pl, mla::kAbsorbAll, form);
        if (st != MLA_OK) {
            std::cout << "err " << st << " " << g_err << "\n";
            continue;
        }
        std::cout << "ok " << pl.ks_chunk << " " << pl.n_chunk_items << " " << pl.n_dec_units << " " << pl.dec_unit_tiles << " "
                  << pl.dec_total_tiles << " " << pl.grid << " " << (int)pl.merge_many << " " << pl.n_split_rows << " "
                  << pl.n_split_chunk_rows << " " << pl.chunk_merge_wgs << " " << (int)pl.chunk_rev << " " << pl.bytes << " "
                  << (int)pl.warm;
        for (int r = 0; r < R; ++r) std::cout << " " << (w.window > 0 ? mla::band_shift(form.band, p[r]) : 0);
        std::cout << "\n";
    }
    return 0;
}
