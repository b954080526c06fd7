"""A layer with a linear test-time memory, trained on associative recall and then served.

    python examples/linear_memory.py [--steps 60] [--batch 16] [--pairs 64]

A sequence writes (key, value) pairs, keys reused with new values, and asks for the newest value of
a key in between.  The layer projects a token to queries, keys, values, a decay and a write strength;
the gated delta rule (``tnt.delta_forward`` / ``tnt.delta_backward``) is its memory; the projection
matrices are updated by orthogonalised momenta (``tnt.orthogonalise``), the gates by plain momentum.
The trained layer then answers the same sequences token by token (``tnt.delta_step``) after a prompt
through the chunked forward, with the states of the batch in a pool.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2511_07343_amd import tnt  # noqa: E402

D, H, DK, DV, KEYS = 128, 4, 64, 64, 24  # width, heads, head sizes, distinct keys
DEV = "cuda"


class DeltaRule(torch.autograd.Function):
    """The gated delta rule as a differentiable call on [B][H][L][..] tensors."""

    @staticmethod
    def forward(ctx, cfg, q, k, v, g, lr):
        x = dict(q=q, k=k, v=v, g=g, lr=lr)
        o, saved, _ = tnt.delta_forward(cfg, x)
        ctx.cfg = cfg
        ctx.save_for_backward(q, k, v, g, lr, saved)
        return o

    @staticmethod
    def backward(ctx, dO):
        q, k, v, g, lr, saved = ctx.saved_tensors
        d = tnt.delta_backward(ctx.cfg, dict(q=q, k=k, v=v, g=g, lr=lr), dO.contiguous(), saved=saved)
        return None, d["dq"], d["dk"], d["dv"], d["dg"], d["dlr"]


def config(B, L):
    return tnt.DeltaConfig(B=B, H=H, L=L, dk=DK, dv=DV, dtype=tnt.BF16, scale=1.0)


class Layer:
    def __init__(self, gen):
        r = lambda *s: torch.randn(*s, device=DEV, generator=gen)
        self.mats = {n: (r(D, m) / D ** 0.5).requires_grad_() for n, m in
                     (("q", H * DK), ("k", H * DK), ("v", H * DV))}
        self.mats["o"] = (r(H * DV, D) / (H * DV) ** 0.5).requires_grad_()
        self.gates = {"g": (0.1 * r(D, H)).requires_grad_(), "lr": (0.1 * r(D, H)).requires_grad_()}

    def inputs(self, x):
        """What the memory sees of tokens x [B][L][D]: views that keep the tokens first."""
        heads = lambda t, d: t.unflatten(-1, (H, d)).transpose(1, 2)
        unit = lambda t: t / (t.norm(dim=-1, keepdim=True) + 1e-6)
        q, k = (unit(heads(x @ self.mats[n], DK)).to(torch.bfloat16) for n in "qk")
        v = heads(x @ self.mats["v"], DV).to(torch.bfloat16)
        g = -torch.nn.functional.softplus((x @ self.gates["g"]).transpose(1, 2) - 6.0)
        lr = torch.sigmoid((x @ self.gates["lr"]).transpose(1, 2))
        return dict(q=q, k=k, v=v, g=g, lr=lr)

    def out(self, o):
        return o.transpose(1, 2).flatten(2).float() @ self.mats["o"]


class Updates:
    """Momentum; of the matrices, orthogonalised (one call a shape)."""

    def __init__(self, layer, rate, gate_rate, decay=0.9):
        self.layer, self.rate, self.gate_rate, self.decay = layer, rate, gate_rate, decay
        self.m = {id(w): torch.zeros_like(w) for w in (*layer.mats.values(), *layer.gates.values())}
        self.cfgs = {}

    @torch.no_grad()
    def step(self, grads):
        shapes = {}
        for w, d in grads:
            m = self.m[id(w)].mul_(self.decay).add_(d)
            if any(w is p for p in self.layer.mats.values()):
                shapes.setdefault(tuple(w.shape), []).append((w, m))
            else:
                w -= self.gate_rate * m
        for (r, c), group in shapes.items():
            cfg = self.cfgs.setdefault((r, c, len(group)), tnt.OrthConfig(n=len(group), rows=r, cols=c))
            u = tnt.orthogonalise(cfg, torch.stack([m for _, m in group]))
            for (w, _), du in zip(group, u):
                w -= self.rate * du


def batch(gen, B, pairs, keys, values):
    """Tokens [B][2 pairs][D] (a write and a question in turn), answers, which tokens ask."""
    L = 2 * pairs
    ids = torch.randint(0, KEYS, (B, pairs), device=DEV, generator=gen)
    vals = torch.randint(0, values.shape[0], (B, pairs), device=DEV, generator=gen)
    at = torch.arange(pairs, device=DEV)
    asked = ids.gather(1, (torch.rand(B, pairs, device=DEV, generator=gen) * (at + 1)).long())
    # the newest write of the asked key, up to the question
    hit = (ids[:, None] == asked[..., None]) & (at <= at[:, None])
    newest = (hit * (at + 1)).amax(-1) - 1
    x = torch.zeros(B, L, D, device=DEV)
    x[:, 0::2, :D // 2] = keys[ids]
    x[:, 0::2, D // 2:] = values[vals]
    x[:, 1::2, :D // 2] = keys[asked]
    target = torch.zeros(B, L, D, device=DEV)
    target[:, 1::2, D // 2:] = values[vals.gather(1, newest)]
    return x, target


def serve(layer, x, prompt):
    """The layer on x [B][L][D]: a prompt through the chunked forward, then token by token."""
    B, L, _ = x.shape
    z = {n: t.detach() for n, t in layer.inputs(x).items()}
    cut = lambda a, b: {n: t[:, :, a:b] for n, t in z.items()}
    o, _, fin = tnt.delta_forward(config(B, prompt), cut(0, prompt), save=False, final_state=True)
    slots = torch.arange(B, device=DEV, dtype=torch.int32).flip(0) + 1  # anywhere in a pool
    pool = torch.zeros(B + 2, H, DK, DV, device=DEV)
    pool[slots.long()] = fin
    outs, one = [o], config(B, 1)
    for t in range(prompt, L):
        outs.append(tnt.delta_step(one, cut(t, t + 1), pool, slots=slots))
    return layer.out(torch.cat(outs, 2))


def main(steps=60, B=16, pairs=64, seed=0, verbose=True, rate=0.1, gate_rate=2.0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    unit = lambda t: t / t.norm(dim=-1, keepdim=True)
    keys = unit(torch.randn(KEYS, D // 2, device=DEV, generator=gen))
    values = unit(torch.randn(16, D // 2, device=DEV, generator=gen))
    layer = Layer(gen)
    updates = Updates(layer, rate, gate_rate)
    params = [*layer.mats.values(), *layer.gates.values()]
    cfg, losses = config(B, 2 * pairs), []
    for s in range(steps):
        x, target = batch(gen, B, pairs, keys, values)
        y = layer.out(DeltaRule.apply(cfg, *layer.inputs(x).values()))
        loss = ((y - target)[:, 1::2] ** 2).sum(-1).mean()
        updates.step(list(zip(params, torch.autograd.grad(loss, params))))
        losses.append(loss.item())
        if verbose and s % 10 == 0:
            print(f"step {s:3d}  loss {losses[-1]:.4f}", flush=True)
    with torch.no_grad():
        x, target = batch(gen, B, pairs, keys, values)
        y = layer.out(DeltaRule.apply(cfg, *layer.inputs(x).values()))
        served = serve(layer, x, prompt=pairs + 3)
        answer = lambda t: (t[:, 1::2, D // 2:] @ values.T).argmax(-1)
        right = (answer(y) == answer(target)).float().mean().item()
        gap = ((y - served).norm() / y.norm()).item()
    if verbose:
        print(f"final loss {losses[-1]:.4f}, answers right {right:.3f}, "
              f"served token by token against chunked {gap:.1e}")
    return losses, right, gap


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--pairs", type=int, default=64)
    a = ap.parse_args()
    main(a.steps, a.batch, a.pairs)
