// The gated delta rule's scans with a wave for each row tile of 16 columns.
#include "delta_team.h"

namespace dark {
namespace delta {

bool team_supported(const Args& a, bool bf16) { return bf16 ? teamed<unsigned short>(a) : teamed<float>(a); }
dark_status launch_team(const Args& a, bool bf16, hipStream_t st) { return bf16 ? launch_team<unsigned short>(a, st) : launch_team<float>(a, st); }
dark_status launch_team_back(const Args& a, bool bf16, const float* g_in, float* g_out, bool states, hipStream_t st) {
  return bf16 ? launch_team_back<unsigned short>(a, g_in, g_out, states, st) : launch_team_back<float>(a, g_in, g_out, states, st);
}

}  // namespace delta
}  // namespace dark
