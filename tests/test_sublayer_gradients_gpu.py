"""The sublayer's gradients against differences along themselves, where a gradient that lacks
anything shows most, and through autograd, each leaf used several times, against autograd
over the formulas in 64 bits.

Along its gradient g an input goes from a to a + s g and a - s g (as fp32 holds them, a step
of d), and the loss, formed in 64 bits from the operator's outputs, changes by g . d but for
* what the outputs are off by, at both ends (`sublayer_ref`, and their rounding to fp32);
* the change's own odd terms: the difference of the loss in 64 bits from g . d in 64 bits;
* what g is off by, times d."""
import numpy as np
import pytest

import paper_2606_00746_amd as gspn
import sublayer_ref as ref
import test_residual_norm_gpu as join
import test_selective_scan_gpu as scan
import test_short_conv_gpu as conv
from gpu_util import require_gpu, to_host
from test_attention_gpu import dev

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def scan64(x):
    return scan.expect(x, None)


def conv64(x):
    return conv.expect(x, None, True)


def join64(x):
    return ref.join(x["r"], x["f"], x["w"], x["w_post"], x["scale"], x["gate"], join.EPS, x["dy"], x["dro"], depth=200)


def scan_gpu(t):
    y, end, reserve = gspn.selective_scan_fwd_train(*scan.args(t), state=t["state"])
    return (y, end), gspn.selective_scan_bwd_reserve(*scan.args(t), t["dy"], reserve, dstate=t["dend"], state=t["state"])


def conv_gpu(t):
    a = t["x"], t["w"], t["bias"]
    return gspn.short_conv_fwd(*a, state=t["state"]), gspn.short_conv_bwd(*a, t["dy"], dstate=t["dend"], state=t["state"])


def join_gpu(t):
    a = [t[n] for n in ("r", "f", "w", "w_post", "scale", "gate")]
    return gspn.residual_norm_fwd(*a, eps=join.EPS), gspn.residual_norm_bwd(*a, t["dy"], t["dro"], eps=join.EPS)


# inputs, both passes on the GPU and in 64 bits, the outputs' names and their gradients', and each
# input's with the name of its gradient, in the order of the calls
OPERATORS = {
    "scan": (lambda: scan.make(1, 50, 16, 1, 4, "f32", 31), scan_gpu, scan64, (("y", "dy"), ("end", "dend")),
             dict(x="dx", dt="ddt", A="dA", B="dB", C="dC", D="dD", z="dz", bias="dbias", state="dstate")),
    "conv": (lambda: conv.make(2, 40, 16, 4, "f32", 31), conv_gpu, conv64, (("y", "dy"), ("end", "dend")),
             dict(x="dx", w="dw", bias="dbias", state="dstate")),
    "join": (lambda: join.make(2, 9, 40, ("f32", "f32"), 31), join_gpu, join64, (("y", "dy"), ("r", "dro")),
             dict(r="dr", f="df", w="dw", w_post="dw_post", scale="dscale", gate="dgate")),
}
STEP = 0.1      # s times the gradient's length: odd terms stay below half a hundredth of the change


def moved(x, name, g, s):
    return {**x, name: np.asarray(x[name] + s * STEP * g / np.linalg.norm(g), np.float32).astype(np.float64)}


def loss(outs, x, ups):
    return sum(float((o * x[u]).sum()) for o, (_, u) in zip(outs, ups))


def expected(op, name, g):
    """The step d; the loss's change in 64 bits, and g . d; what the change may be off by."""
    make, _, f64, ups, grads = OPERATORS[op]
    x = make()
    ends = [moved(x, name, g, s) for s in (1, -1)]
    d = ends[0][name] - ends[1][name]
    want = [f64(e) for e in ends]
    change = [loss([w[o] for o, _ in ups], x, ups) for w in want]
    exact = f64(x)[grads[name]]
    off = sum(float((np.abs(x[u]) * (w.get("e_" + o, 0.0) + U * np.abs(w[o]))).sum()) for w in want for o, u in ups)
    off += float((np.abs(d) * (f64(x)["e_" + grads[name]] + U * np.abs(exact))).sum())
    return ends, d, change[0] - change[1], float((exact * d).sum()), off


CASES = [(op, n) for op in OPERATORS for n in OPERATORS[op][4]]


@pytest.mark.parametrize("op,name", CASES)
def test_along_the_gradient(op, name):
    require_gpu()
    make, gpu, _, ups, grads = OPERATORS[op]

    def on_gpu(x):
        outs, gs = gpu({n: dev(a, "f32") for n, a in x.items()})
        return [to_host(o) for o in outs], dict(zip(grads, map(to_host, gs)))

    g = on_gpu(make())[1][name]
    ends, d, change, along, off = expected(op, name, g)
    got = [loss(on_gpu(e)[0], make(), ups) for e in ends]
    bound = off + abs(change - along)
    print(f"[err] {op} {name}: {abs(got[0] - got[1] - float((g * d).sum())) / bound:.3f} of the bound, {bound / along:.1e} of the change")
    assert bound <= 0.02 * along
    assert abs(got[0] - got[1] - float((g * d).sum())) <= bound


# ---------------------------------------------------------------------------
# through autograd
# ---------------------------------------------------------------------------

def norm64(t):
    return t / (t * t).mean(-1, keepdim=True).add(1e-6).sqrt()


def loss64(p, dy, N):
    """The run below by its formulas, token after token."""
    import torch
    r = p["r"] + p["f"]
    y = norm64(r) * p["w"]
    K = p["taps"].shape[1]
    pad = torch.nn.functional.pad(y, (0, 0, K - 1, 0))
    u = p["bias"] + sum(p["taps"][:, j] * pad[:, j:j + y.shape[1]] for j in range(K))
    c = u * torch.sigmoid(u)
    b = c[..., :N]
    raw = y + p["dtb"]
    d = torch.log1p(torch.exp(-raw.abs())) + raw.clamp(min=0)
    h, s = torch.zeros(*c.shape[::2], N, dtype=torch.float64), []
    for t in range(c.shape[1]):
        h = torch.exp(d[:, t, :, None] * p["A"]) * h + (d[:, t] * c[:, t])[..., None] * b[:, t, None]
        s.append((h * b[:, t, None]).sum(-1))
    s = (torch.stack(s, 1) + p["D"] * c) * r * torch.sigmoid(r)
    r = r + s
    return ((norm64(r) * p["w"] + r) * dy).sum()


def test_shared_leaves():
    """r, f, w and the convolved channels go several ways; every gradient is the sum over them.
    An fp32 step is off by 2^-24 of its result's length; the run is some hundred of them deep
    (150 tokens forward and back, sums over 64 channels and 150 tokens): below 2^12 roundings,
    2.5e-4 of the gradient's length."""
    torch = require_gpu()
    g = torch.Generator().manual_seed(8)
    B, T, C, N = 2, 150, 64, 16
    rand = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x = dict(r=rand(B, T, C), f=rand(B, T, C), w=1 + 0.1 * rand(C), taps=rand(C, 4) / 2, bias=0.1 * rand(C), A=-rand(C, N).exp(),
             D=rand(C), dtb=rand(C) - 2)
    dy = rand(B, T, C)

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
            ctx.save_for_backward(r, f, w)
            return gspn.residual_norm_fwd(r, f, w)

        @staticmethod
        def backward(ctx, dy, dro):
            r, f, w = ctx.saved_tensors
            return gspn.residual_norm_bwd(r, f, w, None, None, None, dy.contiguous(), dro.contiguous())[:3]

    p = {n: t.cuda().requires_grad_() for n, t in x.items()}
    y, r = Join.apply(p["r"], p["f"], p["w"])
    c = Conv.apply(y, p["taps"], p["bias"])
    b = c[..., :N].unsqueeze(2)
    s = Scan.apply(c, y, p["A"], b, b, p["D"], r, p["dtb"])      # b twice: as B and as C
    y2, r2 = Join.apply(r, s, p["w"])
    got = torch.autograd.grad(((y2 + r2) * dy.cuda()).sum(), list(p.values()))
    q = {n: t.double().requires_grad_() for n, t in x.items()}
    want = torch.autograd.grad(loss64(q, dy.double(), N), list(q.values()))
    for n, a, e in zip(x, got, want):
        off = float((a.double().cpu() - e).norm() / e.norm())
        print(f"[err] {n}: {off:.1e}")
        assert off <= 2.0 ** -12, n
