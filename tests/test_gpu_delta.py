"""The gated delta rule on the GPU against the fp64 recurrence: forward, every gradient, packed
sequences, shared heads, strides, carried states and the token-by-token form.

Bounds (max |x - y| / max |y| per tensor), from the arithmetic: fp32 tensors come from sums of
products kept to 2^-24 over at most 64 + 128 terms a product and a few products in a row, 2^-24 *
sqrt(200) * 8 < 1e-5; bf16 tensors are those rounded once: bf16 keeps 8
significant bits, so half a unit in the last place is up to 2^-8 of an element, and the same.
"""
import math

import pytest
import torch

from oracle import linear_oracle as O
from paper_2511_07343_amd import tnt
from parity_log import check_err

pytestmark = pytest.mark.gpu
TOL = {torch.float32: 1e-5, torch.bfloat16: 2.0 ** -8 + 1e-5}
DEV = "cuda:0"


def make(B, H, L, dk, dv, Hk=0, dtype=torch.bfloat16, n=None, seed=0, S0=False, gmean=-3.0,
         lr=None, g=None):
    """Seeded inputs on the CPU, in the call's types."""
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)
    unit = lambda t: t / t.norm(dim=-1, keepdim=True)
    Hk = Hk or H
    x = dict(q=unit(r(B, Hk, L, dk)).to(dtype), k=unit(r(B, Hk, L, dk)).to(dtype),
             v=r(B, H, L, dv).to(dtype),
             g=-torch.nn.functional.softplus(r(B, H, L) + gmean) if g is None else g(B, H, L, gen),
             lr=torch.sigmoid(r(B, H, L)) if lr is None else lr(B, H, L, gen))
    x["dO"] = r(B, H, L, dv).to(dtype)
    if S0:
        x["S0"] = 0.5 * r(n or B, H, dk, dv)
        x["dfinal"] = 0.5 * r(n or B, H, dk, dv)
    return x


def err(a, b):
    b = b.double()
    d = (a.detach().double().cpu() - b).abs().max().item() if b.numel() else 0.0
    m = b.abs().max().item() if b.numel() else 0.0
    return d / m if m else d


def compare(case, got, want):
    bad = []
    for n, w in want.items():
        assert got[n].shape == w.shape, (n, got[n].shape, w.shape)
        e = err(got[n], w)
        if not check_err(case, n, e, TOL[got[n].dtype]):
            bad.append((n, e))
    assert not bad, bad


def gpu(x, tokens_first=False):
    out = {}
    for n, t in x.items():
        t = t.to(DEV)
        if tokens_first and n in ("q", "k", "v", "g", "lr", "dO"):
            t = t.transpose(1, 2).contiguous().transpose(1, 2)
        out[n] = t
    return out


def both(cfg, x, starts=None, tokens_first=False, save=True, train=True):
    """(got, want) of a forward and a backward."""
    d = gpu(x, tokens_first)
    if starts is not None:
        d["seq_start"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    x64 = {n: t.double() for n, t in x.items()}
    o, fin, grads = O.delta_rule_grads({n: t for n, t in x64.items() if n not in ("dO", "dfinal")},
                                       x64["dO"], cfg.scale, starts, x64.get("dfinal"))
    go, saved, gfin = tnt.delta_forward(cfg, d, save=save, final_state=True)
    got, want = dict(o=go, state=gfin), dict(o=o, state=fin)
    if train:
        got.update(tnt.delta_backward(cfg, d, d["dO"], saved=saved, dfinal=d.get("dfinal")))
        want.update(grads)
    torch.cuda.synchronize()
    return got, want


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("L", [1, 2, 16, 63, 64, 65, 130])
def test_lengths(L, dtype):
    """One token to a few chunks, ends inside and at the edge of a chunk and of a 16-row tile."""
    x = make(1, 2, L, 64, 64, dtype=dtype, seed=L, S0=True)
    cfg = tnt.DeltaConfig(B=1, H=2, L=L, dk=64, dv=64, dtype=int(dtype == torch.bfloat16), scale=0.125)
    compare(f"delta L{L} {dtype}", *both(cfg, x))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dk,dv", [(8, 8), (16, 40), (32, 16), (40, 128), (64, 128), (96, 80),
                                   (128, 64), (128, 128)])
def test_head_sizes(dk, dv, dtype):
    """Padded key sizes, odd numbers of value tiles, keys narrower and wider than values."""
    x = make(2, 2, 100, dk, dv, dtype=dtype, seed=dk + dv, S0=True)
    cfg = tnt.DeltaConfig(B=2, H=2, L=100, dk=dk, dv=dv, dtype=int(dtype == torch.bfloat16), scale=0.3)
    compare(f"delta {dk}x{dv} {dtype}", *both(cfg, x))


@pytest.mark.parametrize("H,Hk", [(4, 1), (6, 2), (3, 3)])
@pytest.mark.parametrize("tokens_first", [False, True])
def test_shared_heads_and_strides(H, Hk, tokens_first):
    """Value heads that share keys: dq and dk are summed over them; views of tokens-first memory."""
    x = make(2, H, 77, 64, 48, Hk=Hk, seed=H, S0=True)
    cfg = tnt.DeltaConfig(B=2, H=H, Hk=Hk, L=77, dk=64, dv=48)
    compare(f"delta H{H}/{Hk} tf{tokens_first}", *both(cfg, x, tokens_first=tokens_first))


@pytest.mark.parametrize("starts", [[0, 0, 1, 1, 70, 134, 134, 200], [0, 200], [0, 64, 128, 192, 200],
                                    [0, 0, 0, 200, 200]])
def test_packed(starts):
    """Empty sequences, single tokens, lengths of whole chunks, one sequence alone."""
    n = len(starts) - 1
    x = make(1, 2, 200, 64, 64, Hk=1, n=n, seed=n, S0=True)
    cfg = tnt.DeltaConfig(B=1, H=2, Hk=1, L=200, dk=64, dv=64, n_seq=n)
    compare(f"delta packed {starts}", *both(cfg, x, starts=starts))


def test_packed_many_sequences():
    """More sequences than one pass of the plan's scan takes, most of one or two tokens."""
    gen = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 3, (1500,), generator=gen).tolist()
    starts = [0]
    for m in lens:
        starts.append(starts[-1] + m)
    n, L = len(lens), starts[-1]
    x = make(1, 1, L, 16, 16, n=n, seed=9, S0=True, dtype=torch.float32)
    cfg = tnt.DeltaConfig(B=1, H=1, L=L, dk=16, dv=16, n_seq=n, dtype=0)
    compare("delta packed 1500", *both(cfg, x, starts=starts))


def test_offsets_out_of_order_stay_inside():
    """Offsets below 0, past L and decreasing are clamped and made non-decreasing."""
    x = make(1, 1, 100, 32, 32, n=4, seed=5)
    cfg = tnt.DeltaConfig(B=1, H=1, L=100, dk=32, dv=32, n_seq=4)
    d = gpu(x)
    d["seq_start"] = torch.tensor([-7, 60, 30, 1000, 2000], dtype=torch.int32, device=DEV)
    o, _, fin = tnt.delta_forward(cfg, d, final_state=True)
    d["seq_start"] = torch.tensor([0, 60, 60, 100, 100], dtype=torch.int32, device=DEV)
    o2, _, fin2 = tnt.delta_forward(cfg, d, final_state=True)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(fin, fin2)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_extreme_gates(dtype):
    """No decay, decays that forget everything (-inf, far below the clamp), write strengths of zero
    and one, mixed token by token: finite everywhere and equal to the recurrence."""
    def g(B, H, L, gen):
        pick = torch.randint(0, 5, (B, H, L), generator=gen)
        vals = torch.tensor([0.0, -1e-6, -0.7, -300.0, -math.inf])
        return vals[pick]

    def lr(B, H, L, gen):
        return torch.tensor([0.0, 1.0, 0.5])[torch.randint(0, 3, (B, H, L), generator=gen)]

    x = make(2, 2, 150, 64, 64, dtype=dtype, seed=2, S0=True, g=g, lr=lr)
    cfg = tnt.DeltaConfig(B=2, H=2, L=150, dk=64, dv=64, dtype=int(dtype == torch.bfloat16))
    # below the clamp the kernel's dg is a factor e^-80 times a state, the oracle's zero
    compare(f"delta gates {dtype}", *both(cfg, x))


def test_repeated_keys():
    """Every key of the sequence the same, lr 1: the triangular system's worst conditioned case,
    where powers of its matrix would grow like binomials."""
    x = make(1, 1, 128, 32, 32, dtype=torch.float32, seed=4, S0=True,
             g=lambda B, H, L, gen: torch.zeros(B, H, L), lr=lambda B, H, L, gen: torch.ones(B, H, L))
    k = torch.zeros(1, 1, 128, 32)
    k[..., 3] = 1.0
    x["k"] = k
    cfg = tnt.DeltaConfig(B=1, H=1, L=128, dk=32, dv=32, dtype=0)
    compare("delta repeated keys", *both(cfg, x))


def test_broadcast_inputs():
    """Heads that share one gate and values expanded over heads: gradients per element, which the
    caller sums."""
    x = make(2, 3, 70, 32, 32, dtype=torch.float32, seed=6)
    x["v"] = x["v"][:, :1].expand(2, 3, 70, 32)
    x["lr"] = x["lr"][:, :1].expand(2, 3, 70)
    cfg = tnt.DeltaConfig(B=2, H=3, L=70, dk=32, dv=32, dtype=0)
    d = gpu({n: t for n, t in x.items() if n not in ("v", "lr")})
    d["v"] = x["v"][:, :1].to(DEV).expand(2, 3, 70, 32)
    d["lr"] = x["lr"][:, :1].to(DEV).expand(2, 3, 70)
    o, saved, _ = tnt.delta_forward(cfg, d)
    got = dict(o=o, **tnt.delta_backward(cfg, d, d["dO"], saved=saved))
    x64 = {n: t.double().contiguous() for n, t in x.items()}
    ro, _, grads = O.delta_rule_grads({n: t for n, t in x64.items() if n != "dO"}, x64["dO"])
    compare("delta broadcast", got, dict(o=ro, **grads))


@pytest.mark.parametrize("n", [0, 5])
def test_decay_of_a_zero_state_has_no_gradient(n):
    """A single token without a carried state decays zeros: its dg is zero, not rounding."""
    x = make(1, 2, n or 1, 64, 64, n=n, seed=n)
    cfg = tnt.DeltaConfig(B=1, H=2, L=n or 1, dk=64, dv=64, n_seq=n)
    d = gpu(x)
    if n:
        d["seq_start"] = torch.arange(n + 1, dtype=torch.int32, device=DEV)
    _, saved, _ = tnt.delta_forward(cfg, d)
    g = tnt.delta_backward(cfg, d, d["dO"], saved=saved)
    torch.cuda.synchronize()
    assert (g["dg"] == 0).all() and (g["dlr"] != 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_chunks(dtype):
    """A chain of 34 chunks: against the recurrence, and the recomputing backward and graph replays
    bit for bit."""
    B, L = 2, 32 * 64 + 130
    x = make(B, 1, L, 16, 16, dtype=dtype, seed=31, S0=True)
    cfg = tnt.DeltaConfig(B=B, H=1, L=L, dk=16, dv=16, dtype=int(dtype == torch.bfloat16))
    compare(f"delta parts {dtype}", *both(cfg, x))
    d = gpu(x)

    def step(save):
        o, saved, fin = tnt.delta_forward(cfg, d, save=save, final_state=True)
        return dict(o=o, fin=fin, **tnt.delta_backward(cfg, d, d["dO"], saved=saved, dfinal=d["dfinal"]))

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        ref = {n: t.clone() for n, t in step(True).items()}
        again = step(False)
    torch.cuda.synchronize()
    assert all(torch.equal(ref[n], again[n]) for n in ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        out = step(True)
    for _ in range(3):
        for t in out.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], ref[n]) for n in ref)
        with torch.cuda.stream(st):
            step(True)
        torch.cuda.synchronize()


def test_recompute_equals_saved():
    """A backward that recomputes the states runs the same kernels: bitwise equal gradients."""
    x = make(2, 2, 150, 64, 64, seed=7, S0=True)
    cfg = tnt.DeltaConfig(B=2, H=2, L=150, dk=64, dv=64)
    d = gpu(x)
    _, saved, _ = tnt.delta_forward(cfg, d)
    a = tnt.delta_backward(cfg, d, d["dO"], saved=saved, dfinal=d["dfinal"])
    b = tnt.delta_backward(cfg, d, d["dO"], saved=None, dfinal=d["dfinal"])
    torch.cuda.synchronize()
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_directional_differences():
    """The gradients against central differences of the kernels' own fp32 forward."""
    x = make(1, 2, 90, 32, 32, dtype=torch.float32, seed=8, S0=True)
    cfg = tnt.DeltaConfig(B=1, H=2, L=90, dk=32, dv=32, dtype=0)
    d = gpu(x)

    def loss(z):
        o, _, fin = tnt.delta_forward(cfg, z, save=False, final_state=True)
        return (o.double() * d["dO"].double()).sum() + (fin.double() * d["dfinal"].double()).sum()

    _, saved, _ = tnt.delta_forward(cfg, d)
    grads = tnt.delta_backward(cfg, d, d["dO"], saved=saved, dfinal=d["dfinal"])
    gen = torch.Generator().manual_seed(1)
    for n in ("q", "k", "v", "g", "lr", "S0"):
        u = torch.randn(d[n].shape, generator=gen).to(DEV)
        h = 2e-3
        up, dn = dict(d), dict(d)
        up[n], dn[n] = d[n] + h * u, d[n] - h * u
        num = ((loss(up) - loss(dn)) / (2 * h)).item()
        ana = (grads["d" + n].double() * u.double()).sum().item()
        size = (grads["d" + n].double().norm()).item()  # of a random direction's derivative
        # the difference's own error: h^2 times the third derivative, and fp32 outputs over 2h
        assert check_err("delta differences", "d" + n, abs(num - ana) / size, 5e-3), (n, num, ana)


def test_empty():
    """No tokens: the final state is S0, and its adjoint passes through."""
    cfg = tnt.DeltaConfig(B=2, H=2, L=0, dk=32, dv=32)
    x = gpu(make(2, 2, 0, 32, 32, S0=True, seed=1))
    o, saved, fin = tnt.delta_forward(cfg, x, final_state=True)
    g = tnt.delta_backward(cfg, x, x["dO"], saved=saved, dfinal=x["dfinal"])
    torch.cuda.synchronize()
    assert o.shape == (2, 2, 0, 32) and torch.equal(fin, x["S0"]) and torch.equal(g["dS0"], x["dfinal"])


def test_nan_stays_in_its_sequence():
    """A NaN token poisons its own head from there on, and nothing before or beside it; what lies
    past a sequence's end is not read."""
    x = make(1, 2, 200, 64, 64, n=3, seed=3)
    cfg = tnt.DeltaConfig(B=1, H=2, L=200, dk=64, dv=64, n_seq=3)
    starts = torch.tensor([0, 70, 130, 200], dtype=torch.int32, device=DEV)
    d = dict(gpu(x), seq_start=starts)
    clean, _, fclean = tnt.delta_forward(cfg, d, final_state=True)
    d["v"] = d["v"].clone()
    d["v"][0, 1, 100] = float("nan")
    o, _, fin = tnt.delta_forward(cfg, d, final_state=True)
    torch.cuda.synchronize()
    assert torch.equal(o[:, 0], clean[:, 0]) and torch.equal(o[0, 1, :70], clean[0, 1, :70])
    assert torch.equal(o[0, 1, 130:], clean[0, 1, 130:])
    assert torch.isnan(o[0, 1, 100:130]).all() and torch.isnan(fin[1, 1]).all()
    assert torch.equal(fin[[0, 2]], fclean[[0, 2]])


def test_workspace_garbage_and_stream():
    """Nothing is read from a workspace or saved buffer that the call has not written (both filled
    with NaN), and a call on a side stream equals one on the current one, bit for bit."""
    x = make(2, 2, 77, 64, 40, seed=12, S0=True)
    cfg = tnt.DeltaConfig(B=2, H=2, L=77, dk=64, dv=40)
    d = gpu(x)
    o, saved, fin = tnt.delta_forward(cfg, d, final_state=True)
    g = tnt.delta_backward(cfg, d, d["dO"], saved=saved, dfinal=d["dfinal"])
    nan = lambda n: torch.full((n,), 255, dtype=torch.uint8, device=DEV)
    ws, wb = nan(cfg.size(tnt.TNT_WS_FWD)), nan(cfg.size(tnt.TNT_WS_BWD))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o2, saved2, fin2 = tnt.delta_forward(cfg, d, final_state=True, workspace=ws)
        g2 = tnt.delta_backward(cfg, d, d["dO"], saved=saved2, dfinal=d["dfinal"], workspace=wb)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(fin, fin2) and all(torch.equal(g[n], g2[n]) for n in g)


def test_graph_replays():
    """Forward and backward captured into a HIP graph, replayed between eager calls."""
    x = make(1, 2, 200, 64, 64, n=3, seed=13, S0=True)
    cfg = tnt.DeltaConfig(B=1, H=2, L=200, dk=64, dv=64, n_seq=3)
    d = dict(gpu(x), seq_start=torch.tensor([0, 70, 130, 200], dtype=torch.int32, device=DEV))

    def step():
        o, saved, fin = tnt.delta_forward(cfg, d, final_state=True)
        return dict(o=o, fin=fin, **tnt.delta_backward(cfg, d, d["dO"], saved=saved, dfinal=d["dfinal"]))

    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ref = {n: t.clone() for n, t in step().items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        out = step()
    for _ in range(3):
        for t in out.values():
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], ref[n]) for n in ref)
        with torch.cuda.stream(st):
            step()
        torch.cuda.synchronize()


# ------------------------------------------------------------------------ token by token
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dk,dv,T", [(64, 64, 1), (128, 128, 1), (16, 8, 3), (96, 80, 2), (40, 104, 5)])
def test_step(dk, dv, T, dtype):
    """Sequences in slots of a pool, out of order, one row of padding; untouched slots stay."""
    B, H, Hk = 5, 4, 2
    x = make(B, H, T, dk, dv, Hk=Hk, dtype=dtype, seed=dk)
    cfg = tnt.DeltaConfig(B=B, H=H, Hk=Hk, L=T, dk=dk, dv=dv, dtype=int(dtype == torch.bfloat16), scale=0.5)
    pool = torch.randn(7, H, dk, dv, generator=torch.Generator().manual_seed(1))
    slots = [6, 0, -1, 3, 1]
    d = gpu(x, tokens_first=True)
    state = pool.to(DEV)
    o = tnt.delta_step(cfg, d, state, slots=torch.tensor(slots, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    live = [i for i, s in enumerate(slots) if s >= 0]
    x64 = {n: t.double()[live] for n, t in x.items() if n != "dO"}
    ro, rS = O.delta_rule(**x64, S0=pool[[slots[i] for i in live]].double(), scale=0.5)
    want_o, want_s = torch.zeros(B, H, T, dv).double(), pool.double().clone()
    want_o[live] = ro
    want_s[[slots[i] for i in live]] = rS
    compare(f"delta step {dk}x{dv} T{T} {dtype}", dict(o=o, state=state), dict(o=want_o, state=want_s))
    assert torch.equal(state[[2, 4, 5]].cpu(), pool[[2, 4, 5]])


def test_step_continues_forward():
    """A prompt through the chunked forward, then token by token: the whole sequence's outputs."""
    B, H, L, n = 2, 2, 100, 9
    x = make(B, H, L + n, 64, 64, dtype=torch.float32, seed=21)
    d = gpu(x)
    cut = lambda a, b: {k: t[:, :, a:b].contiguous() for k, t in d.items()}
    cfg = tnt.DeltaConfig(B=B, H=H, L=L, dk=64, dv=64, dtype=0)
    o, _, state = tnt.delta_forward(cfg, cut(0, L), save=False, final_state=True)
    one = tnt.DeltaConfig(B=B, H=H, L=1, dk=64, dv=64, dtype=0)
    outs = [o] + [tnt.delta_step(one, cut(t, t + 1), state) for t in range(L, L + n)]
    x64 = {k: t.double() for k, t in x.items() if k != "dO"}
    ro, rS = O.delta_rule(**x64)
    compare("delta prompt then steps", dict(o=torch.cat(outs, 2), state=state), dict(o=ro, state=rS))


def test_step_slot_out_of_range_is_padding():
    x = make(2, 1, 1, 32, 32, seed=2)
    cfg = tnt.DeltaConfig(B=2, H=1, L=1, dk=32, dv=32)
    state = torch.ones(3, 1, 32, 32, device=DEV)
    o = tnt.delta_step(cfg, gpu(x), state, slots=torch.tensor([3, 1 << 30], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert torch.equal(o, torch.zeros_like(o)) and torch.equal(state, torch.ones_like(state))


def test_slices_of_a_sequence():
    """Tokens cut out of a longer sequence, gates that begin at any element, slots and offsets inside
    longer lists: the same bits as from copies."""
    B, H, L, d = 2, 2, 100, 64
    x = gpu(make(B, H, L, d, d, seed=41))
    pool = torch.randn(5, H, d, d, generator=torch.Generator().manual_seed(2)).to(DEV)
    one = tnt.DeltaConfig(B=B, H=H, L=1, dk=d, dv=d)
    slots = torch.tensor([9, 4, 1], dtype=torch.int32, device=DEV)[1:]
    for t in range(4):
        cut = {n: z[:, :, t:t + 1] for n, z in x.items()}
        a, b = pool.clone(), pool.clone()
        got = tnt.delta_step(one, cut, a, slots=slots)
        want = tnt.delta_step(one, {n: z.clone() for n, z in cut.items()}, b, slots=slots.clone())
        assert torch.equal(got, want) and torch.equal(a, b) and not torch.equal(a, pool)
    for first in (1, 2, 3):
        cfg = tnt.DeltaConfig(B=1, H=H, L=L - first, dk=d, dv=d, n_seq=2)
        cut = {n: z[:1, :, first:] for n, z in x.items()}
        cut["seq_start"] = torch.tensor([7, 0, 60, L - first], dtype=torch.int32, device=DEV)[1:]
        whole = {n: z.clone() for n, z in cut.items()}
        o, saved, _ = tnt.delta_forward(cfg, cut)
        wo, wsaved, _ = tnt.delta_forward(cfg, whole)
        g = tnt.delta_backward(cfg, cut, cut["dO"], saved=saved)
        w = tnt.delta_backward(cfg, whole, whole["dO"], saved=wsaved)
        assert torch.equal(o, wo) and all(torch.equal(g[n], w[n]) for n in w)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_growing_states(dtype):
    """g above 0: the state grows by e^g, in the chunked forward, the backward and token by token."""
    def g(B, H, L, gen):
        x = 0.03 * torch.randn(B, H, L, generator=gen)
        x[:, 1] = 0.02
        return x

    x = make(1, 2, 150, 64, 64, dtype=dtype, seed=51, S0=True, g=g)
    cfg = tnt.DeltaConfig(B=1, H=2, L=150, dk=64, dv=64, dtype=int(dtype == torch.bfloat16))
    got, want = both(cfg, x)
    compare(f"delta growing {dtype}", got, want)
    d = gpu(x)
    state = d["S0"].clone()
    o = tnt.delta_step(cfg, {n: d[n] for n in ("q", "k", "v", "g", "lr")}, state)
    torch.cuda.synchronize()
    compare(f"delta growing steps {dtype}", dict(o=o, state=state), dict(o=want["o"], state=want["state"]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dk,dv", [(16, 24), (32, 32), (64, 64), (96, 80), (128, 128)])
def test_shared_heads_of_every_size(dk, dv, dtype):
    """Value heads that share keys at every padded key size and type, over three chunks, packed rows from
    carried states among them."""
    flag = int(dtype == torch.bfloat16)
    x = make(2, 6, 150, dk, dv, Hk=2, dtype=dtype, seed=dk, S0=True)
    cfg = tnt.DeltaConfig(B=2, H=6, Hk=2, L=150, dk=dk, dv=dv, dtype=flag, scale=0.3)
    compare(f"delta shared {dk}x{dv} {dtype}", *both(cfg, x, tokens_first=True))
    starts = [0, 0, 67, 68, 150]
    x = make(1, 4, 150, dk, dv, Hk=1, dtype=dtype, n=4, seed=dv, S0=True)
    cfg = tnt.DeltaConfig(B=1, H=4, Hk=1, L=150, dk=dk, dv=dv, n_seq=4, dtype=flag)
    compare(f"delta shared packed {dk}x{dv} {dtype}", *both(cfg, x, starts=starts))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dk,dv,L", [(128, 128, 390), (104, 64, 448), (64, 128, 390), (32, 16, 384)])
def test_several_chunks_of_every_size(dk, dv, L, dtype):
    """Six and seven chunks: every turn of the chains' buffers, an even and an odd number of chunks."""
    x = make(1, 2, L, dk, dv, dtype=dtype, seed=dk + L, S0=True)
    cfg = tnt.DeltaConfig(B=1, H=2, L=L, dk=dk, dv=dv, dtype=int(dtype == torch.bfloat16), scale=0.2)
    compare(f"delta chunks {dk}x{dv} L{L} {dtype}", *both(cfg, x))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dk,dv", [(40, 24), (128, 128)])
def test_saved_buffer_and_workspaces_of_nan(dk, dv, dtype):
    """Nothing is read that the calls have not written: saved buffer, forward's and both backwards'
    workspaces filled with NaN beforehand."""
    x = make(1, 4, 200, dk, dv, Hk=2, n=3, dtype=dtype, seed=61, S0=True)
    cfg = tnt.DeltaConfig(B=1, H=4, Hk=2, L=200, dk=dk, dv=dv, n_seq=3, dtype=int(dtype == torch.bfloat16))
    d = dict(gpu(x), seq_start=torch.tensor([0, 70, 71, 200], dtype=torch.int32, device=DEV))
    o, saved, fin = tnt.delta_forward(cfg, d, final_state=True)
    g = tnt.delta_backward(cfg, d, d["dO"], saved=saved, dfinal=d["dfinal"])
    nan = lambda kind: torch.full((cfg.size(kind),), 255, dtype=torch.uint8, device=DEV)
    o2, fin2, saved2 = torch.empty_like(o), torch.empty_like(fin), nan("saved")
    assert tnt.tnt_delta_fwd(cfg, None, d["q"], d["k"], d["v"], d["g"], d["lr"], d["seq_start"], d["S0"], o2, fin2,
                             saved2, nan(tnt.TNT_WS_FWD)) == 0
    for kept, kind in ((saved2, tnt.TNT_WS_BWD), (None, tnt.TNT_WS_BWD_RECOMPUTE)):
        g2 = tnt.delta_backward(cfg, d, d["dO"], saved=kept, dfinal=d["dfinal"], workspace=nan(kind))
        torch.cuda.synchronize()
        assert all(torch.equal(g[n], g2[n]) for n in g)
    assert torch.equal(o, o2) and torch.equal(fin, fin2)


@pytest.mark.parametrize("d", [32, 64, 128])
def test_errors_of_both_signs(d):
    """Sums of positive terms in fp32, o = S0^T q.  What the three terms of an operand leave out is below
    2^-23 of a product and of either sign, and so are the sums' roundings, at most 2^-24 each: over the
    2048 outputs and more their mean is far below 2^-26, where products left out with one sign have
    2^-25."""
    gen = torch.Generator().manual_seed(3)
    r = lambda *s: torch.rand(*s, generator=gen) + 0.1
    x = dict(q=r(1, 64, 1, d), k=r(1, 64, 1, d), v=r(1, 64, 1, d), g=torch.zeros(1, 64, 1),
             lr=torch.zeros(1, 64, 1), S0=r(1, 64, d, d))
    want = (x["q"][:, :, 0, :, None].double() * x["S0"].double()).sum(2)
    o, _, _ = tnt.delta_forward(tnt.DeltaConfig(B=1, H=64, L=1, dk=d, dv=d, dtype=0), gpu(x), save=False)
    mean = ((o[:, :, 0].double().cpu() - want) / want).mean().item()
    assert check_err("delta mean error", f"o {d}", abs(mean), 2.0 ** -26), mean
