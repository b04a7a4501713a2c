// What joins two sublayers: the norm behind a block, its gate and residual scale, the sum
// with the residual stream and the norm ahead of the next block (internal).
#pragma once

#include "attn.hpp"

namespace gspn {

struct JoinProblem {
    Heads r, f, y, ro;                   // [B][T][C], strides of b and t; f.p and ro.p may be null
    Heads dy, dro, dr, df;               // backward; dro.p and df.p may be null
    const void *w, *w_post, *scale;      // [C] or null
    const void *gate;                    // [B][C] or null
    void *dw, *dw_post, *dscale, *dgate; // null where not wanted
    int B, T, C;
    float eps;
    int dtype, rdtype;                   // of everything else; of r, ro and their gradients
    Workspace *ws;
};

constexpr int kJoinMaxRow = 16384;

hipError_t launch_join_fwd(const JoinProblem &p, hipStream_t s);
hipError_t launch_join_bwd(const JoinProblem &p, hipStream_t s);

}  // namespace gspn
