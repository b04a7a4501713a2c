// The short causal convolution of channels along the tokens (internal).
#pragma once

#include "attn.hpp"

namespace gspn {

struct ConvProblem {
    Heads x, y, dy, dx;                  // [B][T][C], strides of b and t
    const void *w, *bias;                // [C][K], [C] or null
    const void *state;                   // [B][K - 1][C], or null: zeros
    void *state_out;                     // the same, or null: not wanted
    const void *dstate;                  // gradient of state_out, or null: zeros
    void *dstate_in, *dw, *dbias;        // gradients, null where not wanted
    const int32_t *lens;                 // [B], or null: T
    int B, T, C, K;
    bool silu;
    int dtype;
    Workspace *ws;
};

constexpr int kConvMaxTaps = 8;

hipError_t launch_conv_fwd(const ConvProblem &p, hipStream_t s);
hipError_t launch_conv_bwd(const ConvProblem &p, hipStream_t s);

}  // namespace gspn
