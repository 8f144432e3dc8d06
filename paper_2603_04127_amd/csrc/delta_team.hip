// The gated delta rule's scans with a wave for each row tile of 16 columns.
#include "delta_team.h"

namespace dark {
namespace delta {

bool team_supported(const Args& a, bool bf16) { return bf16 ? teamed<unsigned short>(a) : teamed<float>(a); }
dark_status launch_team(const Args& a, bool bf16, Pass pass, hipStream_t st) { return bf16 ? launch_team<unsigned short>(a, pass, st) : launch_team<float>(a, pass, st); }
dark_status launch_team_rev(const Args& a, bool bf16, hipStream_t st) { return bf16 ? launch_team_rev<unsigned short>(a, st) : launch_team_rev<float>(a, st); }

}  // namespace delta
}  // namespace dark
