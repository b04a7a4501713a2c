"""The token mixers together, in training and in serving.

A causal model of two sublayers over a sequence of tokens, windowed attention with sinks
(its heads normed and rotated) and the gated delta rule, learns to repeat a short random
sequence. Then it continues a prompt token by token, from the attention's cache and
the delta rule's state, and its logits are compared with those of the whole sequence.

    python examples/token_mixers.py [--steps 100]
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_00746_amd as gspn  # noqa: E402

VOCAB, C, HQ, HKV, D = 32, 256, 4, 2, 64
MASK = dict(left=63, right=0, sinks=4)


class NormRotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, wq, wk, cos, sin, first):
        ctx.save_for_backward(q, k, wq, wk, cos, sin)
        ctx.first = first
        return gspn.qk_norm_rotate_fwd(q, k, wq, wk, cos, sin, first=first)

    @staticmethod
    def backward(ctx, dq, dk):
        q, k, wq, wk, cos, sin = ctx.saved_tensors
        return (*gspn.qk_norm_rotate_bwd(q, k, wq, wk, dq, dk, cos, sin, first=ctx.first), None, None, None)


class WindowAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v):
        o, lse = gspn.window_attn_fwd(q, k, v, **MASK)
        ctx.save_for_backward(q, k, v, o, lse)
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, lse = ctx.saved_tensors
        return gspn.window_attn_bwd(q, k, v, o, lse, do.contiguous(), **MASK)


class DeltaRule(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, g, beta):
        o, _, reserve = gspn.delta_rule_fwd_train(q, k, v, g, beta)
        ctx.save_for_backward(q, k, v, g, beta, reserve)
        return o

    @staticmethod
    def backward(ctx, do):
        *x, reserve = ctx.saved_tensors
        return gspn.delta_rule_bwd_reserve(*x, do.contiguous(), reserve)[:5]


class Model(torch.nn.Module):
    def __init__(self, tokens):
        super().__init__()
        self.embed = torch.nn.Embedding(VOCAB, C)
        self.qkv = torch.nn.Linear(C, (HQ + 2 * HKV) * D, bias=False)
        self.wq, self.wk = (torch.nn.Parameter(torch.ones(D)) for _ in range(2))
        self.out = torch.nn.Linear(HQ * D, C, bias=False)
        self.delta = torch.nn.Linear(C, 3 * HQ * D + 2 * HQ, bias=False)
        self.delta_out = torch.nn.Linear(HQ * D, C, bias=False)
        self.head = torch.nn.Linear(C, VOCAB, bias=False)
        a = torch.arange(tokens)[:, None] * 10000.0 ** (-torch.arange(D // 2) * 2 / D)
        self.register_buffer("cos", a.cos())
        self.register_buffer("sin", a.sin())

    def forward(self, ids, serve=None):
        """Logits of ids [B, T]; serve: the cache of a sequence that goes on behind them."""
        B, T = ids.shape
        first = 0 if serve is None else serve["len"]
        bf = torch.bfloat16
        x = self.embed(ids)
        fused = self.qkv(F.rms_norm(x, (C,))).to(bf).view(B, T, HQ + 2 * HKV, D)
        q, k, v = fused.split((HQ, HKV, HKV), 2)        # slices: the kernels take strides
        q, k = NormRotate.apply(q, k, self.wq.to(bf), self.wk.to(bf), self.cos, self.sin, first)
        if serve is None:
            o = WindowAttention.apply(q, k, v)
        else:
            serve["k"][:, first:first + T], serve["v"][:, first:first + T] = k, v
            lens = torch.full((B,), first + T, dtype=torch.int32, device=ids.device)
            o = gspn.window_attn_decode(q, serve["k"], serve["v"], lens, left=MASK["left"], sinks=MASK["sinks"])
        x = x + self.out(o.flatten(2).float())
        y = self.delta(F.rms_norm(x, (C,)))
        q, k, v = y[..., :3 * HQ * D].view(B, T, 3, HQ, D).unbind(2)
        q, k, v = F.normalize(q, dim=-1).to(bf), F.normalize(k, dim=-1).to(bf), v.to(bf)
        g, beta = -F.softplus(y[..., -2 * HQ:-HQ] - 3).to(bf), torch.sigmoid(y[..., -HQ:]).to(bf)
        if serve is None:
            o = DeltaRule.apply(q, k, v, g, beta)
        else:
            o, serve["state"] = gspn.delta_rule_fwd(q, k, v, g, beta, state=serve["state"], state_out=serve["state"])
            serve["len"] += T
        return self.head(F.rms_norm(x + self.delta_out(o.flatten(2).float()), (C,)))

    def cache(self, B, tokens):
        """An empty cache and state for B sequences of up to `tokens` tokens."""
        dev = self.cos.device
        k, v = (torch.zeros(B, tokens, HKV, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
        return dict(k=k, v=v, len=0, state=torch.zeros(B, HQ, D, D, device=dev))


def batch(B, part, gen):
    """Sequences of a random part and the same part again."""
    ids = torch.randint(VOCAB, (B, part), device="cuda", generator=gen)
    return torch.cat((ids, ids), 1)


def main(steps=100, B=16, part=40, quiet=False):
    """(first loss, last loss, largest difference of served logits from the whole forward's)."""
    torch.manual_seed(0)
    gen = torch.Generator(device="cuda").manual_seed(0)
    model = Model(2 * part).cuda()
    opt = torch.optim.AdamW(model.parameters(), lr=2e-3)
    losses = []
    for step in range(steps):
        ids = batch(B, part, gen)
        logits = model(ids[:, :-1])
        loss = F.cross_entropy(logits[:, part - 1:].flatten(0, 1), ids[:, part:].flatten())
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
        if not quiet and (step % 20 == 0 or step == steps - 1):
            print(f"step {step}: loss {losses[-1]:.3f}", flush=True)
    with torch.no_grad():
        ids = batch(B, part, gen)
        whole = model(ids)
        serve = model.cache(B, 2 * part)
        got = [model(ids[:, :part], serve)]              # the prompt, then a token at a time
        for t in range(part, 2 * part):
            got.append(model(ids[:, t:t + 1], serve))
        got = torch.cat(got, 1)
    off = (got - whole).abs().max().item()
    if not quiet:
        hits = (got[:, part - 1:-1].argmax(-1) == ids[:, part:]).float().mean().item()
        print(f"served: {100 * hits:.1f}% of the repeated tokens right, logits within {off:.3f} of the whole forward's")
    return losses[0], losses[-1], off


if __name__ == "__main__":
    p = argparse.ArgumentParser()
    p.add_argument("--steps", type=int, default=100)
    main(p.parse_args().steps)
