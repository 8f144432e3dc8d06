// The scan of decayed linear attention on bf16 operands.
#include "decay_scan.h"

namespace dark {
namespace decay {

dark_status launch_scan_bf16(const Scans& a, int n, hipStream_t st) { return pick<unsigned short>(a, n, st); }
dark_status launch_state_bf16(const States& a, int n, hipStream_t st) { return pick<unsigned short>(a, n, st); }

}  // namespace decay
}  // namespace dark
