// The gated delta rule's scans and triangles on bf16 operands.
#include "delta_scan.h"

namespace dark {
namespace delta {

dark_status launch_prep_bf16(const Args& a, bool backward, hipStream_t st) { return launch_prep<unsigned short>(a, backward, st); }
dark_status launch_scan_bf16(const Args& a, hipStream_t st) { return launch_scan<unsigned short>(a, st); }
dark_status launch_back_bf16(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st) { return launch_back<unsigned short>(a, g_in, g_out, states, st); }

}  // namespace delta
}  // namespace dark
