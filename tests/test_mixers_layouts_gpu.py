"""Inputs of the token mixers whose tokens, heads or batch entries share memory (views
that broadcast, and windows that overlap): the results of contiguous copies, bit for
bit, for whole sequences that end inside a tile and for ragged ones."""
import pytest

import paper_2606_00746_amd as gspn
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def views(kind, B, T, H, D, dtype, seed, scale=1.0):
    torch = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def rand(*shape):
        return (scale * torch.randn(*shape, device="cuda", generator=g)).to(dt)

    return {"tokens": lambda: rand(B, 1, H, D).expand(B, T, H, D), "heads": lambda: rand(B, T, 1, D).expand(B, T, H, D),
            "batch": lambda: rand(1, T, H, D).expand(B, T, H, D),
            "all": lambda: rand(D).expand(B, T, H, D),
            # token t's head begins 8 entries behind token t - 1's
            "windows": lambda: torch.as_strided(rand(B * (8 * T + H * D + D)), (B, T, H, D), (8 * T + H * D + D, 8, D, 1))}[kind]()


def same(a, b):
    torch = require_gpu()
    for i, (x, y) in enumerate(zip(a, b)):
        alike = torch.equal(x, y)
        assert alike, i


KINDS = ["tokens", "heads", "batch", "all", "windows"]


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_delta_rule(kind, dtype, ragged):
    torch = require_gpu()
    B, T, Hq, Hv, D = 2, 166, 1, 2, 64
    x = [views(kind, B, T, h, D, dtype, i, s) for i, (h, s) in enumerate(((Hq, 0.1), (Hq, 0.1), (Hv, 1.0), (Hv, 1.0)))]
    gen = torch.Generator(device="cuda").manual_seed(9)
    gates = [(f * torch.rand(B, T, Hv, device="cuda", generator=gen)).to(x[0].dtype) for f in (-0.2, 1.0)]
    kw = dict(state=torch.randn(B, Hv, D, D, device="cuda", generator=gen),
              lens=torch.tensor([T, 37], dtype=torch.int32, device="cuda") if ragged else None)

    def pair(q, k, v, do):
        o, end, reserve = gspn.delta_rule_fwd_train(q, k, v, *gates, **kw)
        few = [t[:, :5] for t in (q, k, v)] + [t[:, :5].contiguous() for t in gates]
        return [o, end, *gspn.delta_rule_bwd_reserve(q, k, v, *gates, do, reserve, dstate=end, **kw),
                *gspn.delta_rule_fwd(*few, state=kw["state"])]

    same(pair(*x), pair(*[t.contiguous() for t in x]))


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("D", [64, 104])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_attention(kind, dtype, D, ragged):
    torch = require_gpu()
    B, T, Hq, Hkv = 2, 550, 2, 1
    x = [views(kind, B, T, h, D, dtype, i) for i, h in enumerate((Hq, Hkv, Hkv, Hq))]
    lens = torch.tensor([T, 37], dtype=torch.int32, device="cuda") if ragged else None
    mask = dict(left=60, right=20, sinks=3, lens=lens)

    def step(q, k, v, do):
        o, lse = gspn.window_attn_fwd(q, k, v, **mask)
        d = gspn.window_attn_decode(q[:, :3], k, v, lens, left=200, sinks=5)
        return [o, lse, *gspn.window_attn_bwd(q, k, v, o, lse, do, **mask), d]

    same(step(*x), step(*[t.contiguous() for t in x]))


@pytest.mark.parametrize("pairs", ["half", "adjacent"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_norm(kind, dtype, pairs):
    torch = require_gpu()
    B, T, Hq, Hk, D = 2, 75, 3, 2, 72
    x = [views(kind, B, T, h, D, dtype, i) for i, h in enumerate((Hq, Hk, Hq, Hk))]
    a = torch.rand(T, 18, device="cuda")
    kw = dict(cos=a.cos(), sin=a.sin(), pairs=pairs)
    w = [1 + 0.1 * torch.randn(D, device="cuda").to(x[0].dtype) for _ in range(2)]

    def both(q, k, dyq, dyk):
        return [*gspn.qk_norm_rotate_fwd(q, k, *w, **kw), *gspn.qk_norm_rotate_bwd(q, k, *w, dyq, dyk, **kw)]

    same(both(*x), both(*[t.contiguous() for t in x]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_token_of_heads_outside_tokens(dtype):
    """One token out of buffers [B, H, T, D], whose heads are a million entries apart."""
    torch = require_gpu()
    H, D, tokens = 12, 128, 8192
    gen = torch.Generator(device="cuda").manual_seed(3)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = [(0.1 * torch.randn(1, H, tokens, D, device="cuda", generator=gen)).to(dt)[:, :, 70:71].transpose(1, 2) for _ in range(4)]
    gates = [(f * torch.rand(1, 1, H, device="cuda", generator=gen)).to(dt) for f in (-0.2, 1.0)]
    cache = [(torch.randn(1, 300, H, D, device="cuda", generator=gen)).to(dt) for _ in range(2)]

    def all_of(q, k, v, do):
        o, lse = gspn.window_attn_fwd(q, k, v)
        r, end, reserve = gspn.delta_rule_fwd_train(q, k, v, *gates)
        return [*gspn.qk_norm_rotate_fwd(q, k), *gspn.qk_norm_rotate_bwd(q, k, None, None, do, v)[:2],
                o, lse, *gspn.window_attn_bwd(q, k, v, o, lse, do), gspn.window_attn_decode(q, *cache), r, end,
                *gspn.delta_rule_bwd_reserve(q, k, v, *gates, do, reserve)[:5], *gspn.delta_rule_fwd(q, k, v, *gates, state=end)]

    same(all_of(*x), all_of(*[t.contiguous() for t in x]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads_first", [False, True])
def test_fused_buffers_by_heads(heads_first, dtype):
    """q, k and v beside each other in every head [B][T][H][3][D], and as heads ahead of
    tokens [B][3 H][T][D]: gradients go into a buffer of that layout, the norm runs in place."""
    torch = require_gpu()
    B, T, H, D = 2, 150, 3, 64
    gen = torch.Generator(device="cuda").manual_seed(8)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def rand(*shape):
        return (0.1 * torch.randn(*shape, device="cuda", generator=gen)).to(dt)

    def slices(f):
        if heads_first:
            return [f[:, i * H:(i + 1) * H].transpose(1, 2) for i in range(3)]
        return [f[:, :, :, i] for i in range(3)]

    fused = rand(B, 3 * H, T, D) if heads_first else rand(B, T, H, 3, D)
    own = [t.contiguous() for t in slices(fused)]
    do, gates = rand(B, T, H, D), [(f * torch.rand(B, T, H, device="cuda", generator=gen)).to(dt) for f in (-0.2, 1.0)]
    o, lse = gspn.window_attn_fwd(*own, left=40, right=8, sinks=2)
    _, _, reserve = gspn.delta_rule_fwd_train(*own, *gates)
    want = [gspn.window_attn_bwd(*own, o, lse, do, left=40, right=8, sinks=2),
            gspn.delta_rule_bwd_reserve(*own, *gates, do, reserve)[:5], gspn.qk_norm_rotate_fwd(*own[:2])]
    grads = torch.full_like(fused, float("nan"))
    gspn.window_attn_bwd(*slices(fused), o, lse, do, left=40, right=8, sinks=2, out=slices(grads))
    same(want[0], slices(grads))
    dg = [torch.empty_like(g) for g in gates]
    gspn.delta_rule_bwd_reserve(*slices(fused), *gates, do, reserve, out=(*slices(grads), *dg, None))
    same(want[1], [*slices(grads), *dg])
    q, k, v = slices(fused)
    gspn.qk_norm_rotate_fwd(q, k, out=(q, k))
    same([*want[2], own[2]], slices(fused))
