// The gated delta rule's scans with a wave for each row tile of 16 columns: bf16.
#include "delta_team.h"

namespace dark {
namespace delta {

bool team_bf16(const Args& a) { return teamed<unsigned short>(a); }
bool team_back_bf16(const Args& a, bool states) { return teamed_back<unsigned short>(a, states); }
dark_status launch_team_bf16(const Args& a, hipStream_t st) { return launch_team<unsigned short>(a, st); }
dark_status launch_team_back_bf16(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st) {
  return launch_team_back<unsigned short>(a, g_in, g_out, states, st);
}

}  // namespace delta
}  // namespace dark
