"""Which way the selective scan's GPU cases go, asked of the library's own rule on the CPU."""
import test_selective_scan_gpu as scan
from test_host_checks import _build_and_run


def test_gpu_cases_go_both_ways(tmp_path):
    """With and without a reserve, for each number of states that the kernels hold."""
    calls = [(*c[:5], train) for c in scan.CASES for train in (0, 1)]
    out = _build_and_run(tmp_path, "sublayer", stdin="".join(" ".join(map(str, c)) + "\n" for c in calls)).split()
    assert len(out) == len(calls)
    seen = {}
    for (B, T, C, G, N, train), way in zip(calls, out):
        if T > 8 or train:      # fewer run token by token
            held = max(4, 1 << (N - 1).bit_length())
            seen.setdefault(way, set()).add((held, train))
    assert seen["one"] >= {(n, t) for n in (4, 8, 16, 32, 64) for t in (0, 1)}
    assert seen["chunks"] >= {(n, t) for n in (4, 8, 16, 32, 64) for t in (0, 1)}


def test_long_sequences_of_few_channels_go_in_chunks(tmp_path):
    """The sizes whose times the rule was made from."""
    want = {(1, 34225, 2304, 1, 16, 0): "chunks", (8, 4096, 1536, 1, 16, 1): "chunks", (4, 8191, 768, 2, 8, 0): "chunks",
            (64, 64, 768, 1, 16, 0): "one", (1, 64, 1536, 1, 16, 1): "one", (32, 2048, 1536, 1, 16, 0): "one",
            (8, 1024, 1536, 1, 64, 0): "one", (1, 1024, 1536, 1, 64, 0): "chunks", (64, 1024, 1536, 1, 4, 1): "chunks"}
    out = _build_and_run(tmp_path, "sublayer", stdin="".join(" ".join(map(str, c)) + "\n" for c in want)).split()
    assert dict(zip(want, out)) == want
