// The gated delta rule's scans and triangles on fp32 operands.
#include "delta_scan.h"

namespace dark {
namespace delta {

dark_status launch_prep_f32(const Args& a, bool backward, hipStream_t st) { return launch_prep<float>(a, backward, st); }
dark_status launch_scan_f32(const Args& a, Pass pass, hipStream_t st) { return launch_scan<float>(a, pass, st); }
dark_status launch_rev_f32(const Args& a, hipStream_t st) { return launch_rev<float>(a, st); }

}  // namespace delta
}  // namespace dark
