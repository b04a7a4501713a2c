"""Infinite inputs of the selective scan: what its formula leaves finite stays as it was, bit
for bit, what it makes infinite is so with its sign, and what lies past a sequence's end
is 0.  Signs are chosen so that no sum of the formula adds infinities of both signs."""
import pytest

import paper_2606_00746_amd as gspn
from gpu_util import require_gpu
from test_selective_scan_gpu import GRADS, args, lengths, make, tensors

pytestmark = pytest.mark.gpu
INF = float("inf")

# b, T, C, G, N, lens: token by token, whole sequences in one pass, chunks; numbers of states that
# are held as they are and with room; groups that do and do not fill a wave; ends in a block of 8
CASES = [
    (2, 5, 24, 1, 5, [5, 3]), (1, 7, 16, 1, 16, None),
    (9, 75, 256, 32, 5, [75, 1, 0, 40, 75, 75, 8, 9, 64]), (2, 41, 40, 1, 33, None), (1, 30, 24, 1, 4, [27]),
    (1, 333, 88, 1, 13, [300]), (1, 600, 8, 1, 3, [555]), (1, 333, 128, 1, 16, [301]), (1, 260, 136, 1, 24, None),
    (2, 150, 64, 1, 64, [131, 150]), (1, 270, 128, 2, 7, [266]),
]
TYPES = ["bf16", "f32"]
ids = lambda c: "x".join(map(str, c[:5]))  # noqa: E731


def prepared(case, dtype, seed):
    *sizes, lens = case
    x = make(*sizes, dtype, seed=seed)
    return tensors(x, dtype), lengths(lens), [sizes[1]] * sizes[0] if lens is None else lens


def forwards(t, ln):
    return gspn.selective_scan_fwd(*args(t), state=t["state"], lens=ln)


def both(t, ln):
    y, end, reserve = gspn.selective_scan_fwd_train(*args(t), state=t["state"], lens=ln)
    grads = gspn.selective_scan_bwd_reserve(*args(t), t["dy"], reserve, dstate=t["dend"], state=t["state"], lens=ln)
    return dict(zip(("y", "end", *GRADS), (y, end, *grads)))


def past_the_end_is_zero(got, lens):
    for n in ("y", "dx", "ddt", "dB", "dC", "dz"):
        for i, k in enumerate(lens):
            assert (got[n][i, k:] == 0).all(), (n, i)


def same(got, base, names, lens=(), but=None):
    """Names' values are the base's; `but`(length): a token that is left out."""
    torch = require_gpu()
    for n in names:
        a, b = got[n].clone(), base[n].clone()
        for i, k in enumerate(lens):
            if k > 0:
                a[i, but(k)], b[i, but(k)] = 0, 0
        assert torch.equal(a, b), n


def last(k):
    return k - 1


def first(k):
    return 0


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_an_infinite_last_state(case, dtype):
    """B of the last token: no gradient of A, D, the first state or another token takes it up."""
    t, ln, lens = prepared(case, dtype, 41)
    base = both(t, ln)
    for i, k in enumerate(lens):
        if k > 0:
            t["B"][i, k - 1, :, 0] = INF
    got = both(t, ln)
    same(got, base, ("dA", "dD", "dB", "dstate"))
    same(got, base, ("y", "dx", "ddt", "dC", "dz"), lens, last)
    past_the_end_is_zero(got, lens)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", ["dend", "D"])
@pytest.mark.parametrize("case", [c for c in CASES if c[5]], ids=ids)
def test_past_the_end_of_infinite_gradients(case, name, dtype):
    t, ln, lens = prepared(case, dtype, 42)
    if name == "dend":
        t["dend"][..., 0] = INF
    else:
        t["D"][:] = INF
    past_the_end_is_zero(both(t, ln), lens)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_an_infinite_last_input(case, dtype):
    """x of the last token, with B, C and D above 0: states and y are infinite with x's sign (and
    the gate's), whatever room there is beside the states."""
    torch = require_gpu()
    t, ln, lens = prepared(case, dtype, 43)
    t["D"] = t["D"].abs() + 0.1
    for i, k in enumerate(lens):
        if k > 0:
            for n in ("B", "C"):
                t[n][i, k - 1] = t[n][i, k - 1].abs() + 0.1
    few, base = forwards(t, ln), both(t, ln)
    for i, k in enumerate(lens):
        if k > 0:
            t["x"][i, k - 1] = torch.sign(t["x"][i, k - 1]) * INF
    got = both(t, ln)
    for (y, end), (y0, end0) in ((forwards(t, ln), few), ((got["y"], got["end"]), (base["y"], base["end"]))):
        for i, k in enumerate(lens):
            if k > 0:
                assert torch.equal(y[i, k - 1], t["x"][i, k - 1] * torch.sign(t["z"][i, k - 1])), i
                assert torch.equal(end[i], t["x"][i, k - 1].float()[:, None].expand_as(end[i])), i
                assert torch.equal(y[i, :k - 1], y0[i, :k - 1])
            else:
                assert torch.equal(end[i], end0[i])
    same(got, base, ("dx", "dA", "dstate"))
    same(got, base, ("ddt", "dB", "dC", "dz"), lens, last)
    for i, k in enumerate(lens):
        if k > 0:
            assert torch.isinf(got["ddt"][i, k - 1]).all() and torch.isinf(got["dz"][i, k - 1]).all(), i
    past_the_end_is_zero(got, lens)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_an_infinite_last_step(case, dtype):
    """dt of the last token: all that was is forgotten, what it writes is infinite."""
    torch = require_gpu()
    t, ln, lens = prepared(case, dtype, 44)
    t["D"] = t["D"].abs() + 0.1
    for i, k in enumerate(lens):
        if k > 0:
            for n in ("B", "C", "x"):
                t[n][i, k - 1] = t[n][i, k - 1].abs() + 0.1
            t["dt"][i, k - 1] = INF
    for y, end, *_ in (forwards(t, ln), gspn.selective_scan_fwd_train(*args(t), state=t["state"], lens=ln)):
        for i, k in enumerate(lens):
            if k > 0:
                assert (end[i] == INF).all(), i
                assert torch.equal(y[i, k - 1], torch.sign(t["z"][i, k - 1]) * INF), i


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_an_infinite_step_in_the_middle(case, dtype):
    """Its decay is 0, as that of a step of 200 with these rates: what stands ahead of it does not
    tell them apart, forward or back (an input of 0 there makes NaN of what stands behind)."""
    torch = require_gpu()
    t, ln, lens = prepared(case, dtype, 47)
    t["A"] = -t["A"].abs().clamp(min=1)
    got = []
    for step in (200.0, INF):
        for i, k in enumerate(lens):
            if k > 1:
                t["dt"][i, k // 2], t["x"][i, k // 2] = step, 0
        got.append(both(t, ln))
    for n in ("y", "dx", "ddt", "dB", "dC", "dz"):
        for i, k in enumerate(lens):
            m = k // 2 if k > 1 else k
            assert torch.equal(got[0][n][i, :m], got[1][n][i, :m]), (n, i)
    assert torch.equal(got[0]["dstate"], got[1]["dstate"])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_an_infinite_first_gradient(case, dtype):
    """dy of the first token: what goes back from it is infinite, the tokens behind it know
    nothing of it.  A decay exp(d A) below 2^-120 may be 0 in fp32 (whose normal numbers end at
    2^-126; d A log2 e is off by less than a hundredth there), and 0 times an infinite gradient is
    not a number: states that decay so, and sums that take them, are left out."""
    torch = require_gpu()
    t, ln, lens = prepared(case, dtype, 45)
    t["state"], t["D"] = t["state"].abs() + 0.1, t["D"].abs() + 0.1
    for n in ("B", "C", "z"):
        t[n][:, 0] = t[n][:, 0].abs() + 0.1
    t["x"][:, 0] = -t["x"][:, 0].abs() - 0.1
    base = both(t, ln)
    t["dy"][:, 0] = INF
    got = both(t, ln)
    same(got, base, ("dx", "ddt", "dB", "dC", "dz"), lens, first)
    d = torch.nn.functional.softplus(t["dt"][:, 0].double() + t["bias"].double())
    lasts = d[..., None] * t["A"].double() > -120 * 0.6931471805599453     # [b, C, N]
    assert lasts.double().mean() > 0.9
    for i, k in enumerate(lens):
        if k > 0:
            assert (got["dx"][i, 0] == INF).all() and (got["dB"][i, 0] == -INF).all(), i
            assert (got["ddt"][i, 0] == -INF)[lasts[i].all(-1)].all() and (got["dstate"][i] == INF)[lasts[i]].all(), i
            assert torch.isinf(got["dz"][i, 0]).all(), i
    assert (got["dA"] == INF)[lasts.all(0)].all() and (got["dD"] == -INF).all()
    past_the_end_is_zero(got, lens)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_sums_over_channels_of_infinite_states(case, dtype):
    """C of the first token and B of the last, of one state: dB and dC there are sums over a
    group's channels alone, also where it does not fill the lanes."""
    torch = require_gpu()
    t, ln, lens = prepared(case, dtype, 46)
    for i, k in enumerate(lens):
        if k > 0:
            for n in ("x", "z", "dy"):
                for j, sign in ((0, -1 if n == "x" else 1), (k - 1, 1)):
                    t[n][i, j] = sign * (t[n][i, j].abs() + 0.1)
    base = both(t, ln)
    C0, B1 = t["C"].clone(), t["B"].clone()
    for i, k in enumerate(lens):
        if k > 1:
            C0[i, 0, :, 0], B1[i, k - 1, :, 0] = INF, INF
    up, down = both({**t, "C": C0}, ln), both({**t, "B": B1}, ln)
    for i, k in enumerate(lens):
        if k > 1:
            assert (up["dB"][i, 0, :, 0] == -INF).all(), i
            assert torch.equal(up["dB"][i, 0, :, 1:], base["dB"][i, 0, :, 1:]), i
            assert (down["dC"][i, k - 1, :, 0] == INF).all(), i
            assert torch.equal(down["dC"][i, k - 1, :, 1:], base["dC"][i, k - 1, :, 1:]), i


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("name", ["x", "dy"])
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_nan_goes_one_way(case, name, dtype):
    """NaN of an input goes to its own token's outputs and all behind it, of a gradient to those
    ahead of it, and to nothing on the other side."""
    torch = require_gpu()
    t, ln, lens = prepared(case, dtype, 48)
    base = both(t, ln)
    for i, k in enumerate(lens):
        if k > 0:
            t[name][i, k // 2] = float("nan")
    got = both(t, ln)
    for i, k in enumerate(lens):
        m = k // 2
        if name == "x":
            assert torch.equal(got["y"][i, :m], base["y"][i, :m]) and torch.equal(got["dx"][i], base["dx"][i]), i
            assert torch.equal(got["ddt"][i, :m], base["ddt"][i, :m]) and torch.equal(got["dstate"][i], base["dstate"][i]), i
            assert got["y"][i, m:k].isnan().all() and (k == 0 or got["end"][i].isnan().all()), i
        else:
            assert torch.equal(got["y"][i], base["y"][i]) and torch.equal(got["end"][i], base["end"][i]), i
            for n in ("dx", "ddt", "dB", "dC", "dz"):
                assert torch.equal(got[n][i, m + 1:], base[n][i, m + 1:]), (n, i)
            assert k == 0 or got["dx"][i, :m + 1].isnan().all() and got["dstate"][i].isnan().all(), i
    past_the_end_is_zero(got, lens)
