// The selective state space scan, forward, fp32 storage.
#include "selective_fwd.hpp"

namespace gspn {

hipError_t launch_selective_fwd_f32(const SelectiveProblem &p, hipStream_t s) { return pick<float>(p, s); }

}  // namespace gspn
