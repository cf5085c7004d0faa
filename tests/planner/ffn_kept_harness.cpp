// Host-only harness: how often calls of the feed-forward entry points plan anew (the translation unit
// of their choice is included as is; the device queries answer for a 256-CU device, and the number
// of CUs is asked for once a plan).  Input on stdin, one call per line:
//   what rows in out f32
// (what: 0 product with 4-bit weights, 1 block in bf16, 2 block in 4 bits).  Output, a line for each call:
// the launches that it planned anew, then variant, parts and rows of each launch.
#include <hip/hip_runtime.h>

static int planned = 0;
static hipError_t harness_get_device(int *d) {
    *d = 0;
    return hipSuccess;
}
static hipError_t harness_get_attribute(int *v, hipDeviceAttribute_t, int) {
    ++planned;
    *v = 256;
    return hipSuccess;
}
#define hipGetDevice harness_get_device
#define hipDeviceGetAttribute harness_get_attribute
#include "../../paper_2607_02043_amd/csrc/ffn_api.cpp"
#undef hipGetDevice
#undef hipDeviceGetAttribute

#include <cstdio>
#include <string>

namespace mla {
int set_error(int code, const char *, ...) { return code; }
int hip_error(hipError_t, const char *) { return MLA_ERR_HIP; }
}  // namespace mla
static std::string launches;
namespace ffn {
hipError_t launch_gemm(GemmArgs g, bool, Epilogue, const Shape &t, hipStream_t) {
    launches += " " + std::to_string(t.variant) + "/" + std::to_string(t.splits) + "/" + std::to_string(g.M);
    return hipSuccess;
}
}  // namespace ffn

int main() {
    int what, rows, in, out, f32;
    char *const fake = reinterpret_cast<char *>(size_t(1) << 40);
    const auto u8 = reinterpret_cast<const uint8_t *>(fake);
    const auto u16 = reinterpret_cast<const uint16_t *>(fake);
    while (std::scanf("%d %d %d %d %d", &what, &rows, &in, &out, &f32) == 5) {
        const mla_mx4 m{u8, u8};
        const mla_ffn_weights w{u16, u16, u16, in, out};
        const mla_ffn4_weights w4{m, m, m, in, out};
        const int32_t dtype = f32 ? MLA_OUT_F32 : MLA_OUT_BF16;
        const size_t ws = size_t(1) << 50;
        planned = 0;
        launches.clear();
        if (what == 0) mla_linear4(rows, u16, &m, in, out, fake, dtype, fake, ws, nullptr);
        else if (what == 1) mla_gated_ffn(rows, u16, &w, fake, dtype, fake, ws, nullptr);
        else mla_gated_ffn4(rows, u16, &w4, fake, dtype, fake, ws, nullptr);
        std::printf("%d%s\n", planned, launches.c_str());
    }
}
