"""What a call of the sublayer could not fill or could not run on is refused (the front end's
own checks, ahead of any GPU)."""
import types

import pytest
import torch

import paper_2606_00746_amd as gspn

x, w, v = torch.zeros(2, 5, 16), torch.zeros(16, 4), torch.zeros(16)
A, B, s = torch.zeros(16, 8), torch.zeros(2, 5, 1, 8), torch.zeros(2, 16, 8)
conv, sel = (x, w, None), (x, x, A, B, B, None, None, None)
reserve = torch.zeros(8, dtype=torch.uint8)


@pytest.mark.parametrize("what,call", {
    "dbias": lambda: gspn.short_conv_bwd(*conv, x, out=(x, w, v, None)),
    "dD": lambda: gspn.selective_scan_bwd_reserve(*sel, x, reserve, out=(x, x, A, B, B, v, None, None, None)),
    "dz": lambda: gspn.selective_scan_bwd_reserve(*sel, x, reserve, out=(x, x, A, B, B, None, x, None, None)),
    "ddt_bias": lambda: gspn.selective_scan_bwd_reserve(*sel, x, reserve, out=(x, x, A, B, B, None, None, v, None)),
    "df": lambda: gspn.residual_norm_bwd(x, None, v, None, None, None, x, out=(x, x, v, None, None, None)),
    "dw": lambda: gspn.residual_norm_bwd(x, x, None, None, None, None, x, out=(x, x, v, None, None, None)),
    "dw_post": lambda: gspn.residual_norm_bwd(x, x, v, None, None, None, x, out=(x, x, v, v, None, None)),
    "dscale": lambda: gspn.residual_norm_bwd(x, x, v, None, None, None, x, out=(x, x, v, None, v, None)),
    "dgate": lambda: gspn.residual_norm_bwd(x, x, v, None, None, None, x, out=(x, x, v, None, None, x[:, 0])),
}.items(), ids=lambda v: v if isinstance(v, str) else "")
def test_a_gradient_of_what_is_not_there(what, call):
    with pytest.raises(ValueError, match=f"{what} is the gradient of"):
        call()


def test_a_stream_of_its_own_without_a_sum():
    """Without f the stream is r; another tensor would be left as it is."""
    with pytest.raises(ValueError, match="r_out"):
        gspn.residual_norm_fwd(x, None, v, out=(x.clone(), x.clone()))
    for same in (x, x.view_as(x), None):
        with pytest.raises(ValueError, match="on a GPU"):      # which is all that these lack
            gspn.residual_norm_fwd(x, None, v, out=(x.clone(), same))


@pytest.mark.parametrize("call", [lambda s: gspn.short_conv_fwd(x, w, stream=s), lambda s: gspn.short_conv_bwd(*conv, x, stream=s),
                                  lambda s: gspn.selective_scan_fwd(*sel, stream=s), lambda s: gspn.selective_scan_fwd_train(*sel, stream=s),
                                  lambda s: gspn.selective_scan_bwd_reserve(*sel, x, reserve, stream=s), lambda s: gspn.residual_norm_fwd(x, stream=s),
                                  lambda s: gspn.residual_norm_bwd(x, None, None, None, None, None, x, stream=s)])
def test_a_stream_of_another_device(call):
    """It would run on the current stream of the tensors' device."""
    with pytest.raises(ValueError, match="stream must be of"):
        call(types.SimpleNamespace(cuda_stream=0, device=torch.device("cuda", 1)))
