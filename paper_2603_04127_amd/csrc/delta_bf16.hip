// The gated delta rule's scans and triangles on bf16 operands.
#include "delta_scan.h"

namespace dark {
namespace delta {

dark_status launch_prep_bf16(const Args& a, bool backward, hipStream_t st) { return launch_prep<unsigned short>(a, backward, st); }
dark_status launch_scan_bf16(const Args& a, Pass pass, hipStream_t st) { return launch_scan<unsigned short>(a, pass, st); }
dark_status launch_rev_bf16(const Args& a, hipStream_t st) { return launch_rev<unsigned short>(a, st); }

}  // namespace delta
}  // namespace dark
