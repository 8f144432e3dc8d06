// The gated delta rule's scans with four waves for 16 columns.
#include "delta_team.h"

namespace dark {
namespace delta {

bool team_supported(const Args& a) { return teamed(a); }
dark_status launch_team(const Args& a, Pass pass, hipStream_t st) {
  if (a.dk == 64) return pass == kForward ? go_team<64, true>(a, st) : go_team<64, false>(a, st);
  return pass == kForward ? go_team<128, true>(a, st) : go_team<128, false>(a, st);
}
dark_status launch_team_rev(const Args& a, hipStream_t st) { return a.dk == 64 ? go_team_rev<64>(a, st) : go_team_rev<128>(a, st); }

}  // namespace delta
}  // namespace dark
