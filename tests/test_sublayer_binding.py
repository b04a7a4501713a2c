"""What the state space sublayer's tensor front end refuses before it asks for a GPU."""
import pytest
import torch

import paper_2606_00746_amd as gspn

x = torch.zeros(2, 5, 16)
w, A, B = torch.zeros(16, 4), torch.zeros(16, 8), torch.zeros(2, 5, 1, 8)


@pytest.mark.parametrize("what,call", {
    "on a GPU": lambda: gspn.short_conv_fwd(x, w),
    "on a GPU ": lambda: gspn.selective_scan_fwd(x, x, A, B, B),
    "on a GPU  ": lambda: gspn.residual_norm_fwd(x, x),
    "x must have 3 dimensions": lambda: gspn.short_conv_fwd(x[0], w),
    "w must have 2 dimensions": lambda: gspn.short_conv_fwd(x, w[0]),
    "w must be a contiguous": lambda: gspn.short_conv_fwd(x, w[:8]),
    "bias must be": lambda: gspn.short_conv_fwd(x, w, torch.zeros(8)),
    "lens must be": lambda: gspn.short_conv_fwd(x, w, lens=torch.zeros(2, dtype=torch.int64)),
    "dt must be": lambda: gspn.selective_scan_fwd(x, x[:, :4], A, B, B),
    "dt must have dtype": lambda: gspn.selective_scan_fwd(x, x.bfloat16(), A, B, B),
    "B must have 4 dimensions": lambda: gspn.selective_scan_fwd(x, x, A, B[:, :, 0], B),
    "C must be": lambda: gspn.selective_scan_fwd(x, x, A, B, B[..., :4]),
    "C must be contiguous in its last": lambda: gspn.selective_scan_fwd(x, x, A, B, torch.zeros(2, 5, 1, 16)[..., ::2]),
    "z must be": lambda: gspn.selective_scan_fwd(x, x, A, B, B, z=x[:1]),
    "r must have 3 dimensions": lambda: gspn.residual_norm_fwd(x[0], x[0]),
    "scale must be": lambda: gspn.residual_norm_fwd(x, x, scale=torch.zeros(4)),
    "gate must be": lambda: gspn.residual_norm_fwd(x, x, gate=torch.zeros(16)),
    "w_post must be": lambda: gspn.residual_norm_fwd(x, x.bfloat16(), w_post=torch.zeros(16)),
}.items(), ids=lambda v: v if isinstance(v, str) else "")
def test_refusals(what, call):
    with pytest.raises(ValueError, match=what.strip()):
        call()


def test_types():
    with pytest.raises((TypeError, ValueError)):
        gspn.short_conv_fwd(x.half(), w.half())
