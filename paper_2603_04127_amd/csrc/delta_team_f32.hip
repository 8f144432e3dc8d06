// The gated delta rule's scans with a wave for each row tile of 16 columns: fp32.
#include "delta_team.h"

namespace dark {
namespace delta {

bool team_f32(const Args& a) { return teamed<float>(a); }
bool team_back_f32(const Args& a, bool states) { return teamed_back<float>(a, states); }
dark_status launch_team_f32(const Args& a, hipStream_t st) { return launch_team<float>(a, st); }
dark_status launch_team_back_f32(const Args& a, const float* g_in, float* g_out, bool states, hipStream_t st) {
  return launch_team_back<float>(a, g_in, g_out, states, st);
}

}  // namespace delta
}  // namespace dark
