"""How calls of the state space sublayer meet a program: the whole sublayer, with the
token mixers beside it; results that repeat bit for bit, under a captured graph and on a
stream of the caller's too; workspaces of the caller's; strided tensors whose offsets pass
32 bits; refusals of the tensors' front end; autograd through the training pairs."""
import numpy as np
import pytest

import mixers_ref
import paper_2606_00746_amd as gspn
import sublayer_ref as ref
from gpu_util import require_gpu, to_host
from test_attention_gpu import dev, within

pytestmark = pytest.mark.gpu


def inputs(dtype, B=2, T=150, C=64, N=16, seed=1):
    torch = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def rand(*shape):
        return torch.randn(*shape, device="cuda", generator=g).to(dt)

    def wide(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    return dict(r=wide(B, T, C), f=rand(B, T, C), w=1 + 0.1 * rand(C), wp=1 + 0.1 * rand(C), scale=rand(C), gate=rand(B, C),
                proj=rand(C, 2 * C) / C ** 0.5, small=rand(C, C + 2 * N) / C ** 0.5, taps=rand(C, 4), bias=rand(C), ends=rand(B, 3, C),
                A=-wide(C, N).exp(), D=wide(C), dtb=wide(C) - 2, state=wide(B, C, N), dend=wide(B, C, N), dy=rand(B, T, C), out=rand(C, C) / C ** 0.5,
                lens=torch.tensor([T, T // 3], dtype=torch.int32, device="cuda")[:B])


def everything(x, **kw):
    """A sublayer from one residual joint to the next, its gradients, a single token behind
    it, and the delta rule over the convolution's output; the products between are torch's."""
    torch = require_gpu()
    C, N = x["A"].shape
    y, r = gspn.residual_norm_fwd(x["r"], x["f"], x["w"], x["wp"], x["scale"], x["gate"], **kw)
    xz = y @ x["proj"]
    xc, ends = gspn.short_conv_fwd(xz[..., :C], x["taps"], x["bias"], state=x["ends"], lens=x["lens"], **kw)
    small = xc @ x["small"]
    mats = (small[..., C:C + N].unsqueeze(2), small[..., C + N:].unsqueeze(2))
    sel = (xc, small[..., :C], x["A"], *mats, x["D"], xz[..., C:], x["dtb"])
    s, end, reserve = gspn.selective_scan_fwd_train(*sel, state=x["state"], lens=x["lens"], **kw)
    s2, _ = gspn.selective_scan_fwd(*sel, state=x["state"], lens=x["lens"], **kw)
    f = s @ x["out"]
    y2, r2 = gspn.residual_norm_fwd(r, f, x["w"], **kw)
    dj = gspn.residual_norm_bwd(r, f, x["w"], None, None, None, x["dy"], x["r"], **kw)
    ds = gspn.selective_scan_bwd_reserve(*sel, dj[1] @ x["out"].T.contiguous(), reserve, dstate=x["dend"], state=x["state"], lens=x["lens"], **kw)
    dc = gspn.short_conv_bwd(xz[..., :C], x["taps"], x["bias"], ds[0], dstate=x["ends"], state=x["ends"], lens=x["lens"], **kw)
    d0 = gspn.residual_norm_bwd(x["r"], x["f"], x["w"], x["wp"], x["scale"], x["gate"], dc[0], dj[0], **kw)
    # the next token
    t1, e1 = gspn.short_conv_fwd(xz[:, :1, :C], x["taps"], x["bias"], state=ends, **kw)
    o1, end1 = gspn.selective_scan_fwd(t1, small[:, :1, :C], x["A"], *(m[:, :1] for m in mats), x["D"], xz[:, :1, C:], x["dtb"], state=end, **kw)
    # a recurrence of matrix states over the same convolved channels
    h = xc.view(*xc.shape[:2], 2, C // 2) / 8
    gate = torch.full(h.shape[:3], -0.1, dtype=h.dtype, device="cuda")
    o, e = gspn.delta_rule_fwd(h, h, h, gate, -gate, lens=x["lens"], **kw)
    return [y, r, xc, ends, s, s2, end, y2, r2, *dj[:3], *ds, *dc, *d0, t1, e1, o1, end1, o, e]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_sublayer_step_by_step(dtype):
    """Each operator's output in the run, and in that of its gradients, is its formula's of
    the inputs that it had there (the bounds of its own tests)."""
    torch = require_gpu()
    x = inputs(dtype)
    C, N = x["A"].shape
    h = {n: to_host(t) if t.dtype != torch.int32 else t.cpu().numpy() for n, t in x.items()}
    got = [None if t is None else to_host(t) for t in everything(x)]
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24

    def close(tag, a, want, err, u=half):
        within(tag, a, want, u * np.abs(want) + (1 + u) * err + 1e-37)

    j = ref.join(h["r"], h["f"], h["w"], h["wp"], h["scale"], h["gate"], 1e-6)
    close("y", got[0], j["y"], j["e_y"])
    close("r", got[1], j["r"], j["e_r"], 2.0 ** -24)
    xz = to_host(dev(got[0], dtype) @ x["proj"])
    small = to_host(dev(got[2], dtype) @ x["small"])
    for b, n in enumerate((150, 50)):
        c = ref.conv(xz[b, :, :C], h["taps"], h["bias"], h["ends"][b], n, True)
        close("xc", got[2][b], c["y"], c["e_y"])
        assert np.array_equal(got[3][b], c["end"])
        s = ref.scan(got[2][b], small[b, :, :C], h["A"], *(np.repeat(m[:, None], C, 1) for m in (small[b, :, C:C + N], small[b, :, C + N:])),
                     h["D"], xz[b, :, C:], h["dtb"], h["state"][b], n, True)
        for i in (4, 5):
            close("s", got[i][b], s["y"], s["e_y"])
        close("state", got[6][b], s["end"], s["e_end"], 2.0 ** -24)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_results_repeat(dtype):
    torch = require_gpu()
    x = inputs(dtype)
    first = everything(x)
    for _ in range(3):
        for i, (a, b) in enumerate(zip(first, everything(x))):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_on_a_given_stream(dtype):
    torch = require_gpu()
    x = inputs(dtype)
    want = everything(x)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for s in (side, side.cuda_stream):
        with torch.cuda.stream(side):       # the products between the calls
            got = everything(x, stream=s)
        side.synchronize()
        for i, (a, b) in enumerate(zip(want, got)):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_under_a_graph(dtype):
    """Captured once, replayed on other inputs with eager work in between."""
    torch = require_gpu()
    x = inputs(dtype)
    everything(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything(x)
    for seed in (2, 3, 4):
        new = inputs(dtype, seed=seed)
        for n, t in x.items():
            t.copy_(new[n])
        want = everything(new)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(want, got)):
            assert torch.equal(a, b), (seed, i)


def test_two_streams_at_once():
    """Calls on two streams, each with its own workspace, do not meet."""
    torch = require_gpu()
    xs = [inputs("bf16", T=600, seed=s) for s in (5, 6)]
    want = [everything(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = everything(xs[i])
    torch.cuda.synchronize()
    for w, a in zip(want, got):
        for i, (p, q) in enumerate(zip(w, a)):
            assert torch.equal(p, q), i


def test_workspaces_of_the_caller():
    """One buffer for call after call, whatever it holds, and one that is too small (a new one
    is taken)."""
    torch = require_gpu()
    x = inputs("f32")
    C, N = x["A"].shape
    b = x["dy"].unsqueeze(2)[..., :N]
    sel = (x["dy"], x["f"], x["A"], b, b, x["D"], x["f"], x["dtb"])
    want = [*gspn.selective_scan_fwd(*sel)]
    y, end, reserve = gspn.selective_scan_fwd_train(*sel)
    want += [*gspn.selective_scan_bwd_reserve(*sel, x["dy"], reserve)[:8], *gspn.short_conv_bwd(x["f"], x["taps"], x["bias"], x["dy"])[:3],
             *gspn.residual_norm_bwd(x["r"], x["f"], x["w"], x["wp"], x["scale"], x["gate"], x["dy"])]
    for size in (64, 1 << 26):
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")     # NaN in every word
        got = [*gspn.selective_scan_fwd(*sel, workspace=ws)]
        y, end, reserve = gspn.selective_scan_fwd_train(*sel, reserve=torch.full_like(reserve, 255), workspace=ws)
        got += [*gspn.selective_scan_bwd_reserve(*sel, x["dy"], reserve, workspace=ws)[:8],
                *gspn.short_conv_bwd(x["f"], x["taps"], x["bias"], x["dy"], workspace=ws)[:3],
                *gspn.residual_norm_bwd(x["r"], x["f"], x["w"], x["wp"], x["scale"], x["gate"], x["dy"], workspace=ws)]
        for i, (a, c) in enumerate(zip(want, got)):
            assert torch.equal(a, c), i


def spread(t, tokens):
    """t [B, T, ...] as a view whose tokens stand `tokens` entries apart."""
    torch = require_gpu()
    B, T = t.shape[:2]
    wide = torch.empty(B * T * tokens, dtype=t.dtype, device="cuda")
    v = torch.as_strided(wide, t.shape, (T * tokens, tokens, *t.stride()[2:]))
    return v.copy_(t)


def test_offsets_past_32_bits():
    """Tensors whose entries stand up to 2^32 of them (8 GiB) from the first: the results of
    contiguous ones, bit for bit."""
    torch = require_gpu()
    T, apart = 1100, 1 << 22
    assert T * apart > 2 ** 32
    x = inputs("bf16", B=1, T=T, C=32)
    b = x["dy"][..., :16].contiguous().unsqueeze(2)
    near = dict(x=x["f"], dt=x["dy"], B=b, z=x["f"].flip(1).contiguous())
    far = {n: spread(t, apart) for n, t in near.items()}

    def call(t, y, out):
        sel = (t["x"], t["dt"], x["A"], t["B"], t["B"], x["D"], t["z"], x["dtb"])
        y, end, reserve = gspn.selective_scan_fwd_train(*sel, y=y)
        return [y, end, *gspn.selective_scan_bwd_reserve(*sel, t["dt"], reserve, out=out)[:8]]

    want = call(near, None, None)
    o = [torch.empty_like(t) for t in want[2:]]
    for i in (0, 1, 3, 4, 6):      # dx, ddt, dB, dC, dz
        o[i] = spread(o[i], apart)
    got = call(far, spread(want[0], apart), (*o, None))
    for i, (a, c) in enumerate(zip(want, got)):
        assert torch.equal(a, c), i
    want = [gspn.short_conv_fwd(near["x"], x["taps"])[0], *gspn.short_conv_bwd(near["x"], x["taps"], None, near["dt"])[:2]]
    got = [gspn.short_conv_fwd(far["x"], x["taps"], y=got[0])[0]]
    got += gspn.short_conv_bwd(far["x"], x["taps"], None, far["dt"], out=(o[0], torch.empty_like(x["taps"]), None, None))[:2]
    for a, c in zip(want, got):
        assert torch.equal(a, c)
    v = (x["w"], x["wp"], x["scale"], x["gate"])
    want = [*gspn.residual_norm_fwd(near["x"], near["dt"], *v)]
    want += gspn.residual_norm_bwd(near["x"], near["dt"], *v, near["z"])
    got = [*gspn.residual_norm_fwd(far["x"], far["dt"], *v, out=(o[0], o[1]))]
    got = [t.clone() for t in got]
    got += gspn.residual_norm_bwd(far["x"], far["dt"], *v, far["z"], out=(o[0], o[6], *(torch.empty_like(t) for t in v)))
    for i, (a, c) in enumerate(zip(want, got)):
        assert torch.equal(a, c), i


def test_refusals():
    torch = require_gpu()
    x = inputs("bf16")
    C, N = x["A"].shape
    b = x["dy"].unsqueeze(2)[..., :N]
    sel = (x["dy"], x["f"], x["A"], b, b, x["D"], x["f"], x["dtb"])
    y, end, reserve = gspn.selective_scan_fwd_train(*sel)
    v = (x["w"], x["wp"], x["scale"], x["gate"])
    for what, call in {
        "A must be": lambda: gspn.selective_scan_fwd(*sel[:2], x["A"].bfloat16(), *sel[3:]),
        "D must be": lambda: gspn.selective_scan_fwd(*sel[:5], x["D"].bfloat16()),
        "dt_bias must be": lambda: gspn.selective_scan_fwd(*sel[:7], x["dtb"][1:]),
        "state must be": lambda: gspn.selective_scan_fwd(*sel, state=x["state"].bfloat16()),
        "state_out must be": lambda: gspn.selective_scan_fwd(*sel, state_out=x["state"].mT),
        "z must be on": lambda: gspn.selective_scan_fwd(*sel[:6], x["f"].cpu()),
        "y must have": lambda: gspn.selective_scan_fwd(*sel, y=x["r"]),
        "reserve must": lambda: gspn.selective_scan_bwd_reserve(*sel, x["dy"], x["state"]),
        "smaller than": lambda: gspn.selective_scan_bwd_reserve(*sel, x["dy"], reserve[:64]),
        "workspace": lambda: gspn.selective_scan_fwd(*sel, workspace=x["state"]),
        "lens must be": lambda: gspn.selective_scan_fwd(*sel, lens=x["lens"].long()),
        "contiguous in its last": lambda: gspn.short_conv_fwd(x["f"].mT.contiguous().mT, x["taps"]),
        "w must be": lambda: gspn.short_conv_fwd(x["f"], x["taps"].float()),
        "state must be ": lambda: gspn.short_conv_fwd(x["f"], x["taps"], state=x["ends"][:, 1:]),
        "dy must be": lambda: gspn.short_conv_bwd(x["f"], x["taps"], None, x["dy"][:, 1:]),
        "r_out must": lambda: gspn.residual_norm_fwd(x["r"], x["f"], *v, out=(x["dy"], x["dy"])),
        "f must be": lambda: gspn.residual_norm_fwd(x["r"], x["f"][:, 1:], *v),
        "gate must be": lambda: gspn.residual_norm_fwd(x["r"], x["f"], gate=x["gate"].float()),
        "tensors must be on": lambda: gspn.residual_norm_fwd(x["r"], x["f"].cpu()),
        "dr_out must": lambda: gspn.residual_norm_bwd(x["r"], x["f"], *v, x["dy"], x["dy"]),
    }.items():
        with pytest.raises(ValueError, match=what.strip()):
            call()
    # what the library refuses
    for call in (
        lambda: gspn.selective_scan_fwd(*sel, y=x["dy"]),                                  # an output over an input
        lambda: gspn.short_conv_fwd(x["f"], x["taps"], y=x["f"]),
        lambda: gspn.short_conv_fwd(x["f"], x["taps"][:, :1].contiguous()),                # one tap
        lambda: gspn.short_conv_fwd(x["f"][..., :60], x["taps"][:60]),                     # channels in eights
        lambda: gspn.short_conv_fwd(x["f"][..., 4:60], x["taps"][4:60]),                   # from an odd address
        lambda: gspn.residual_norm_fwd(x["r"], None, x["w"], scale=x["scale"]),            # a block's vector without a block
        lambda: gspn.residual_norm_fwd(x["r"], x["f"], eps=-1.0),
        lambda: gspn.residual_norm_fwd(x["dy"], x["f"].float()),                           # a stream of fewer bits than the block
    ):
        with pytest.raises(gspn.GspnError):
            call()


def test_under_autograd():
    """The pairs as autograd's functions, a leaf used twice: its gradients add up."""
    torch = require_gpu()
    x = inputs("f32")
    N = x["A"].shape[1]

    class Scan(torch.autograd.Function):
        @staticmethod
        def forward(ctx, *a):
            y, _, reserve = gspn.selective_scan_fwd_train(*a)
            ctx.save_for_backward(*a, reserve)
            return y

        @staticmethod
        def backward(ctx, dy):
            *a, reserve = ctx.saved_tensors
            return gspn.selective_scan_bwd_reserve(*a, dy.contiguous(), reserve)[:8]

    class Conv(torch.autograd.Function):
        @staticmethod
        def forward(ctx, *a):
            ctx.save_for_backward(*a)
            return gspn.short_conv_fwd(*a)[0]

        @staticmethod
        def backward(ctx, dy):
            return gspn.short_conv_bwd(*ctx.saved_tensors, dy.contiguous())[:3]

    class Join(torch.autograd.Function):
        @staticmethod
        def forward(ctx, r, f, w):
            y, ro = gspn.residual_norm_fwd(r, f, w)
            ctx.save_for_backward(r, f, w)
            return y, ro

        @staticmethod
        def backward(ctx, dy, dro):
            r, f, w = ctx.saved_tensors
            return gspn.residual_norm_bwd(r, f, w, None, None, None, dy.contiguous(), dro.contiguous())[:3]

    leaves = {n: x[n].clone().requires_grad_() for n in ("r", "f", "w", "taps", "bias", "A", "D", "dtb")}

    def loss(p):
        y, r = Join.apply(p["r"], p["f"], p["w"])
        c = Conv.apply(y, p["taps"], p["bias"])
        b = c[..., :N].unsqueeze(2)
        s = Scan.apply(c, y, p["A"], b, b, p["D"], r, p["dtb"])      # b twice: as B and as C
        y, r = Join.apply(r, s, p["w"])
        return ((y + r).double() * x["dy"].double()).sum()

    grads = torch.autograd.grad(loss(leaves), list(leaves.values()))
    h = 3e-3
    for i, (n, g) in enumerate(zip(leaves, grads)):
        torch.manual_seed(i)
        d = torch.randn_like(g)
        d /= d.norm()
        with torch.no_grad():
            num = float(loss({**leaves, n: leaves[n] + h * d}) - loss({**leaves, n: leaves[n] - h * d})) / (2 * h)
        # the difference's third derivatives, and roundings of the loss's terms over h
        assert abs(num - float((g.double() * d.double()).sum())) <= 2e-2 * float(g.double().norm()) + 1e-2, n
