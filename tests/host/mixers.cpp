// The kernels that the token mixers' calls on stdin take, one call a line:
//   attn B Tq Tk Hq Hkv D left right sinks offset bf16
//   norm B T Hq Hk D R adjacent
// Prints for attention the forward (split, pairs, whole) and the gradient's two kernels
// (fine, pairs, whole), for the norm the heads that a group of lanes takes.
#include <cstdio>
#include <cstring>

#include "qk_norm.hpp"

using namespace gspn;

int main()
{
    char what[16];
    while (scanf("%15s", what) == 1) {
        if (strcmp(what, "attn") == 0) {
            AttnProblem p{};
            int bf16;
            if (scanf("%d %d %d %d %d %d %d %d %d %d %d", &p.B, &p.Tq, &p.Tk, &p.Hq, &p.Hkv, &p.D, &p.left, &p.right, &p.sinks,
                      &p.offset, &bf16) != 11)
                return 1;
            p.dtype = bf16;
            const char *const rows[2] = {"whole", "pairs"};
            const bool fine = bf16 && attn_few_keys(p);
            printf("%s %s %s\n", attn_split_preferred(p) ? "split" : rows[attn_fwd_pairs(p)], fine ? "fine" : rows[attn_dq_pairs(p)],
                   fine ? "fine" : rows[attn_dkv_pairs(p)]);
        } else {
            NormProblem p{};
            int adjacent;
            if (scanf("%d %d %d %d %d %d %d", &p.B, &p.T, &p.Hq, &p.Hk, &p.D, &p.R, &adjacent) != 7)
                return 1;
            p.adjacent = adjacent;
            printf("%d\n", norm_heads_each(p));
        }
    }
    return 0;
}
