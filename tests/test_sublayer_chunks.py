"""How many chunks the selective scan cuts its GPU cases into, from the workspace that a call
of these sizes takes (the chunks' states and sums of steps, behind B and C as fp32)."""
import ctypes

import paper_2606_00746_amd as g
import test_selective_chains_gpu as chains
from paper_2606_00746_amd._sublayer import SELECTIVE_FWD_TRAIN


def chunks(B, T, C, G, N):
    out = ctypes.c_int64(-1)
    assert g.load().gspn_selective_scan_workspace_size(SELECTIVE_FWD_TRAIN, B, T, C, G, N, g.F32, ctypes.byref(out)) == 0
    held = max(4, 1 << (N - 1).bit_length())
    return out.value // (B * C * (held + 1) * 4)      # the pieces' alignment adds less than a chunk


def test_chains_of_many_chunks():
    """Sixteen runs of more chunks than a run holds at once."""
    for *sizes, _ in chains.CASES:
        assert chunks(*sizes) > 16 * 16, sizes
    assert chunks(1, 64, 1536, 1, 16) == 0     # one pass
