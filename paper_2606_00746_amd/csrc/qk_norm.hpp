// The norm of query and key heads with the position rotation (internal).
#pragma once

#include "attn.hpp"

namespace gspn {

struct NormProblem {
    Heads q, k, yq, yk;          // forward
    Heads dyq, dyk, dq, dk;      // backward (with q, k)
    const void *wq, *wk;         // [D], or null: ones
    void *dwq, *dwk;             // [D], null where the weight is
    const float *cos, *sin;      // [rows][R / 2]
    const int32_t *positions;    // [B][T] rows of the tables, or null: first + t
    int B, T, Hq, Hk, D, R;
    int rows, first;
    bool adjacent;               // pairs (2 i, 2 i + 1); else (i, R / 2 + i)
    float eps;
    int dtype;
    Workspace *ws;
};

constexpr int kNormMaxHead = 256;

// Heads of a token that a group of lanes of the forward takes: 1 or 4.
int norm_heads_each(const NormProblem &p);
hipError_t launch_norm_rotate_fwd(const NormProblem &p, hipStream_t s);
hipError_t launch_norm_rotate_bwd(const NormProblem &p, hipStream_t s);

}  // namespace gspn
