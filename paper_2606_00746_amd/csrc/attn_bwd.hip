// Gradient of windowed attention, bf16 storage.
#include "attn_bwd.hpp"

namespace gspn {

hipError_t launch_attn_bwd(const AttnProblem &p, hipStream_t s)
{
    return p.dtype == 0 ? launch_attn_bwd_f32(p, s) : run<bf16_t>(p, s);
}

}  // namespace gspn
