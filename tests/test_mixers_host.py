"""Which kernels the token mixers' GPU cases take, asked of the library on the CPU."""
import test_mixers_large_gpu as large
from test_host_checks import LINK, _build_and_run


def test_gpu_cases_take_the_kernels_they_name(tmp_path):
    lines, want = [], []
    for cases, kernels in ((large.WHOLE, ("whole", "whole", "whole")), (large.PAIRS, ("pairs", "pairs", "pairs")),
                           (large.SPLIT, ("split", None, None))):
        for c in cases:
            for bf16 in (0, 1):
                lines.append("attn " + " ".join(map(str, (*c[:9], c[10], bf16))))
                want.append(kernels)
    for c in large.NORM:
        lines.append("norm " + " ".join(map(str, (*c[:6], int(c[6] == "adjacent")))))
        want.append(("4",))
    out = _build_and_run(tmp_path, "mixers", *LINK, stdin="\n".join(lines) + "\n").splitlines()
    assert len(out) == len(want)
    for ln, got, names in zip(lines, out, want):
        assert all(w in (None, g) for g, w in zip(got.split(), names)), (ln, got, names)
