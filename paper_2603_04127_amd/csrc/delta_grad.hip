// The gated delta rule's gradients, for both types.
#include "delta_grad.h"

namespace dark {
namespace delta {

dark_status launch_grad_bf16(const Args& a, hipStream_t st) { return launch_grad<unsigned short>(a, st); }
dark_status launch_grad_f32(const Args& a, hipStream_t st) { return launch_grad<float>(a, st); }

}  // namespace delta
}  // namespace dark
