// The gated delta rule's scans and triangles on fp32 operands.
#include "delta_scan.h"

namespace dark {
namespace delta {

dark_status launch_prep_f32(const Args& a, bool backward, hipStream_t st) { return launch_prep<float>(a, backward, st); }
dark_status launch_scan_f32(const Args& a, hipStream_t st) { return launch_scan<float>(a, st); }
dark_status launch_back_f32(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st) { return launch_back<float>(a, g_in, g_out, states, st); }

}  // namespace delta
}  // namespace dark
