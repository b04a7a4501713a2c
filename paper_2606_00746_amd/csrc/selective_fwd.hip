// The selective state space scan, forward, bf16 storage.
#include "selective_fwd.hpp"

namespace gspn {

hipError_t launch_selective_fwd(const SelectiveProblem &p, hipStream_t s)
{
    return p.dtype == 0 ? launch_selective_fwd_f32(p, s) : pick<bf16_t>(p, s);
}

}  // namespace gspn
