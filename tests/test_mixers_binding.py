"""What the tensors' front end of the token mixers refuses before it asks for a GPU."""
import pytest
import torch

import paper_2606_00746_amd as gspn


@pytest.mark.parametrize("value", [1 << 31, 1 << 32, (1 << 40) + 5, -(1 << 33)])
def test_numbers_of_more_than_32_bits(value):
    """ctypes would cut them off: a window of 2**32 keys would be one of 0."""
    x, lse = torch.zeros(1, 4, 1, 64), torch.zeros(1, 1, 4)
    for name in ("left", "right", "sinks", "offset"):
        with pytest.raises(ValueError, match=f"{name} must be between"):
            gspn.window_attn_fwd(x, x, x, **{name: value})
        with pytest.raises(ValueError, match=f"{name} must be between"):
            gspn.window_attn_bwd(x, x, x, x, lse, x, **{name: value})
    for name in ("left", "sinks"):
        with pytest.raises(ValueError, match=f"{name} must be between"):
            gspn.window_attn_decode(x, x, x, **{name: value})
    with pytest.raises(ValueError, match="first must be between"):
        gspn.qk_norm_rotate_fwd(x, x, cos=torch.zeros(9, 32), sin=torch.zeros(9, 32), first=value)
