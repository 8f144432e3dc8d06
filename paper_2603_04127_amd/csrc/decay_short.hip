// The one-launch scan of decayed linear attention on bf16 operands.
#include "decay_short.h"

namespace dark {
namespace decay {

dark_status launch_short_bf16(const Scans& a, int n, hipStream_t st) { return pick_short<unsigned short>(a, n, st); }

}  // namespace decay
}  // namespace dark
