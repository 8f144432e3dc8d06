// The scan of decayed linear attention on fp32 operands (v_mfma_f32_16x16x4_f32: products and sums in fp32).
#include "decay_scan.h"

namespace dark {
namespace decay {

dark_status launch_scan_f32(const Scans& a, int n, hipStream_t st) { return pick<float>(a, n, st); }
dark_status launch_state_f32(const States& a, int n, hipStream_t st) { return pick<float>(a, n, st); }

}  // namespace decay
}  // namespace dark
