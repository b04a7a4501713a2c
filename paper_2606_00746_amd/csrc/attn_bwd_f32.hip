// Gradient of windowed attention, fp32 storage.
#include "attn_bwd.hpp"

namespace gspn {

hipError_t launch_attn_bwd_f32(const AttnProblem &p, hipStream_t s) { return run<float>(p, s); }

}  // namespace gspn
