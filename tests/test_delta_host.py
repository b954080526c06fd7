"""Host-side checks of the gated delta rule's calls: refusals before anything is enqueued, buffer
sizes, the binding's argument checks, and the fp64 recurrence against finite differences."""
import ctypes

import pytest
import torch

from oracle import linear_oracle as O
from paper_2511_07343_amd import tnt

P = 256  # an aligned address that is never read


def cfg(**kw):
    base = dict(B=2, H=4, Hk=2, L=100, dk=64, dv=64)
    base.update(kw)
    return tnt.DeltaConfig(**base)


def fwd(c, strides=None, ptr=P, ws=1 << 40, saved=None, saved_bytes=0, seq=None, S0=None):
    return tnt.tnt_delta_fwd(c, strides, ptr, ptr, ptr, ptr, ptr, seq, S0, ptr, None, saved, ptr,
                             ws_bytes=ws, stream=0, saved_bytes=saved_bytes)


def bwd(c, strides=None, ptr=P, ws=1 << 40, saved=None, saved_bytes=0):
    return tnt.tnt_delta_bwd(c, strides, ptr, ptr, ptr, ptr, ptr, None, None, ptr, None, saved, ptr, ptr,
                             ptr, ptr, ptr, None, ptr, ws_bytes=ws, stream=0, saved_bytes=saved_bytes)


def step(c, ptr=P, n_slots=8, slots=None):
    return tnt.tnt_delta_step(c, None, ptr, ptr, ptr, ptr, ptr, ptr, n_slots, slots, ptr, stream=0)


@pytest.mark.parametrize("bad,code", [
    (dict(B=0), 2), (dict(H=0), 2), (dict(H=3), 2), (dict(L=-1), 2), (dict(dk=0), 2),
    (dict(n_seq=-1), 2), (dict(n_seq=3), 2),            # packed: one row
    (dict(dk=60), 3), (dict(dk=136), 3), (dict(dv=4), 3), (dict(dv=256), 3),
    (dict(dtype=2), 7), (dict(B=1 << 20, L=1 << 20), 3),
])
def test_shapes_refused(bad, code):
    c = cfg(**bad)
    assert fwd(c) == code and bwd(c) == code
    assert tnt.tnt_delta_workspace_size(c, 0) == 0 and tnt.tnt_delta_saved_size(c) == 0


def test_null_alignment_workspace_refused():
    c = cfg()
    assert fwd(c, ptr=0) == 1 and bwd(c, ptr=0) == 1 and step(c, ptr=0) == 1
    assert fwd(c, ptr=264) == 5 and bwd(c, ptr=264) == 5 and step(c, ptr=264) == 5
    assert fwd(c, ws=c.size(tnt.TNT_WS_FWD) - 1) == 4
    assert fwd(c, saved=P, saved_bytes=c.size("saved") - 1) == 4
    assert bwd(c, ws=c.size(tnt.TNT_WS_BWD_RECOMPUTE) - 1) == 4
    assert bwd(c, saved=P, saved_bytes=c.size("saved"), ws=c.size(tnt.TNT_WS_BWD) - 1) == 4
    assert fwd(cfg(B=1, n_seq=2), seq=None) == 1
    assert tnt.lib().tnt_delta_fwd(None, None, *([P] * 10), 0, P, 1 << 40, None) == 1


def test_strides_refused():
    c = cfg()
    good = []
    for name in ("q", "k", "v", "v", "g", "g", "v", "q", "k", "v", "g", "g"):
        s = torch.empty(c.shape(name), device="meta").stride()
        good += s[:3]
    for at, code in ((2, 5), (5, 5), (8, 5)):  # tokens of q, k, v not 16 bytes apart
        bad = list(good)
        bad[at] = 65
        assert fwd(c, tnt.tnt_delta_strides(*bad)) == code
    for at in (9, 10, 11):  # an output with two elements in one place
        bad = list(good)
        bad[at] = 0
        assert fwd(c, tnt.tnt_delta_strides(*bad)) == 7
    for at in range(21, 36):
        bad = list(good)
        bad[at] = 0
        assert bwd(c, tnt.tnt_delta_strides(*bad)) == 7


def test_step_refused():
    assert step(cfg(B=1, n_seq=2)) == 2
    assert step(cfg(), n_slots=0) == 2
    assert step(cfg(), n_slots=1) == 2          # fewer states than rows, without slots
    assert step(cfg(L=0), ptr=0) == 0           # nothing to do


def test_sizes():
    c = cfg()
    assert c.size("saved") == 2 * 2 * 4 * (64 * 64 + 64 * 64) * 4  # chunks x heads x (errors, states)
    assert c.size(tnt.TNT_WS_BWD_RECOMPUTE) == c.size(tnt.TNT_WS_BWD) + c.size("saved")
    assert c.size(tnt.TNT_WS_FWD) > c.size("saved")
    assert tnt.tnt_delta_workspace_size(c, 9) == 0


def test_binding_checks():
    c = cfg(B=1, H=2, Hk=1, L=3, dk=8, dv=8)
    x = {n: torch.zeros(c.shape(n), dtype=c.io if n in "qkv" else torch.float32)
         for n in ("q", "k", "v", "g", "lr")}
    for n, t in (("q", torch.zeros(1, 2, 3, 8, dtype=torch.bfloat16)), ("v", torch.zeros(c.shape("v"))),
                 ("g", torch.zeros(1, 2, 4)), ("lr", torch.zeros(1, 2, 3, dtype=torch.float64)),
                 ("k", torch.zeros(1, 1, 8, 3, dtype=torch.bfloat16).transpose(2, 3)),
                 ("S0", torch.zeros(1, 2, 8, 9))):
        with pytest.raises(ValueError, match=n):
            tnt.delta_forward(c, {**x, n: t})
    with pytest.raises(ValueError, match="seq_start"):
        tnt.delta_forward(cfg(B=1, H=2, Hk=1, L=3, dk=8, dv=8, n_seq=2), x)
    with pytest.raises(ValueError, match="slots"):
        tnt.delta_step(c, x, torch.zeros(4, 2, 8, 8), slots=torch.zeros(1, dtype=torch.int64))


def test_oracle_gradients_against_differences():
    gen = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    x = dict(q=r(1, 1, 7, 3), k=0.5 * r(1, 1, 7, 3), v=r(1, 2, 7, 4), g=-r(1, 2, 7).abs(),
             lr=torch.sigmoid(r(1, 2, 7)), S0=r(2, 2, 3, 4))
    dO, dfin, starts = r(1, 2, 7, 4), r(2, 2, 3, 4), [0, 3, 7]
    _, _, g = O.delta_rule_grads(x, dO, 0.7, starts, dfin)

    def loss(z):
        o, fin = O.delta_rule(z["q"], z["k"], z["v"], z["g"], z["lr"], z["S0"], 0.7, starts)
        return (o * dO).sum() + (fin * dfin).sum()

    for n in x:
        u, h = r(*x[n].shape), 1e-6
        num = (loss({**x, n: x[n] + h * u}) - loss({**x, n: x[n] - h * u})) / (2 * h)
        ana = (g["d" + n] * u).sum()
        assert abs(num - ana) <= 1e-7 * max(1.0, abs(ana)), n


def test_oracle_without_decay_solves_recall():
    """One key, lr 1, no decay: the state recalls the last value written, exactly."""
    k = torch.zeros(1, 1, 4, 3, dtype=torch.float64)
    k[..., 1] = 1.0
    v = torch.arange(8, dtype=torch.float64).reshape(1, 1, 4, 2)
    o, S = O.delta_rule(k, k, v, torch.zeros(1, 1, 4, dtype=torch.float64),
                        torch.ones(1, 1, 4, dtype=torch.float64))
    assert torch.equal(o, v) and torch.equal(S[0, 0, 1], v[0, 0, -1])


def test_strides_layout_matches_header():
    assert ctypes.sizeof(tnt.tnt_delta_strides) == 12 * 3 * 8
    assert ctypes.sizeof(tnt.tnt_delta_config) == 36


def test_host_tensors_are_refused(monkeypatch):
    """Tensors in host memory never reach the library, given workspaces and saved buffers among them."""
    c = cfg(B=1, H=2, Hk=1, L=3, dk=8, dv=8)
    x = {n: torch.zeros(c.shape(n), dtype=c.io if n in "qkv" else torch.float32)
         for n in ("q", "k", "v", "g", "lr")}
    dO, state = torch.zeros(c.shape("v"), dtype=c.io), torch.zeros(4, 2, 8, 8)
    size = lambda kind: torch.empty(c.size(kind), dtype=torch.uint8)

    def reached(*a, **kw):
        raise AssertionError("the library was called")

    for n in ("tnt_delta_fwd", "tnt_delta_bwd", "tnt_delta_step"):
        monkeypatch.setattr(tnt, n, reached)
    for call in (lambda s: tnt.delta_forward(c, x, stream=s),
                 lambda s: tnt.delta_forward(c, x, workspace=size(tnt.TNT_WS_FWD), stream=s),
                 lambda s: tnt.delta_backward(c, x, dO, stream=s),
                 lambda s: tnt.delta_backward(c, x, dO, saved=size("saved"), workspace=size(tnt.TNT_WS_BWD), stream=s),
                 lambda s: tnt.delta_step(c, x, state, stream=s)):
        for stream in (None, 0):
            with pytest.raises(ValueError, match="GPU"):
                call(stream)


@pytest.mark.parametrize("n", ["g", "lr", "dg", "dlr", "seq_start", "slots"])
@pytest.mark.parametrize("off,ok", [(4, True), (8, True), (2, False)])
def test_element_wise_tensors_at_any_element(n, off, ok):
    """Gates, their gradients, offsets and slots are read and written one element at a time: they may
    begin anywhere, as slices of longer tensors do.  (The calls end at their workspace or at a
    broadcast output.)"""
    at = lambda name: P + off if name == n else P
    seq = cfg(B=1, n_seq=2) if n == "seq_start" else cfg()
    start = at("seq_start") if seq.n_seq else None
    want = 4 if ok else 5
    if n in ("g", "lr", "seq_start"):
        assert tnt.tnt_delta_fwd(seq, None, P, P, P, at("g"), at("lr"), start, None, P, None, None, P,
                                 ws_bytes=0, stream=0) == want
    if n != "slots":
        assert tnt.tnt_delta_bwd(seq, None, P, P, P, at("g"), at("lr"), start, None, P, None, None, P, P, P,
                                 at("dg"), at("dlr"), None, P, ws_bytes=0, stream=0) == want
    if n in ("g", "lr", "slots"):
        c, s = cfg(), []
        for name in ("q", "k", "v", "v", "g", "g"):
            s += torch.empty(c.shape(name), device="meta").stride()[:3]
        s[9] = 0
        got = tnt.tnt_delta_step(c, tnt.tnt_delta_strides(*s), P, P, P, at("g"), at("lr"), P, 8, at("slots"), P,
                                 stream=0)
        assert got == (7 if ok else 5)


def test_strides_that_are_not_read():
    """The backward has no output o, so whatever stands in its strides is not looked at."""
    c, s = cfg(), []
    for name in ("q", "k", "v", "v", "g", "g", "v", "q", "k", "v", "g", "g"):
        s += torch.empty(c.shape(name), device="meta").stride()[:3]
    for junk in (0, -3, 65, 1 << 40):
        s[9:12] = [junk] * 3
        assert bwd(c, tnt.tnt_delta_strides(*s), ws=0) == 4
        assert fwd(c, tnt.tnt_delta_strides(*s), ws=0) in (3, 5, 7)


def test_launches_past_the_grid_are_refused():
    """A launch holds fewer than 2^32 threads: more (sequence, head) tiles or chunks are refused before
    anything is enqueued."""
    c, s = cfg(B=1 << 20, H=31, Hk=31, L=1, dk=128, dv=128), []
    for name in ("q", "k", "v", "v", "g", "g"):
        s += torch.empty(c.shape(name), device="meta").stride()[:3]
    s[9] = 0  # (a broadcast output: the call would end there)
    assert tnt.tnt_delta_step(c, tnt.tnt_delta_strides(*s), P, P, P, P, P, P, 1 << 20, None, P, stream=0) == 3
    for big in (dict(B=1 << 20, H=31, Hk=31, L=0, dk=64, dv=16), dict(B=1 << 20, H=17, Hk=17, L=1, dk=8, dv=8)):
        assert fwd(cfg(**big), ws=0) == 3 and bwd(cfg(**big), ws=0) == 3
    assert fwd(cfg(B=1 << 19, H=16, Hk=16, L=1, dk=8, dv=8), ws=0) == 4


def test_saved_buffer_of_another_configuration(monkeypatch):
    """A saved buffer of another size was written for other shapes, a larger one too."""
    monkeypatch.setattr(tnt, "_elsewhere", lambda stream, dev: False)
    monkeypatch.setattr(tnt, "_current", lambda dev: 0)
    monkeypatch.setattr(tnt, "tnt_delta_bwd", lambda *a, **kw: 0)
    c = cfg(B=1, H=2, Hk=1, L=70, dk=8, dv=8)
    x = {n: torch.zeros(c.shape(n), dtype=c.io if n in "qkv" else torch.float32)
         for n in ("q", "k", "v", "g", "lr")}
    dO = torch.zeros(c.shape("v"), dtype=c.io)
    saved = lambda k: torch.empty(k.size("saved"), dtype=torch.uint8)
    tnt.delta_backward(c, x, dO, saved=saved(c))
    for other in (dict(L=200), dict(L=60), dict(dk=40), dict(dv=40), dict(H=4)):
        with pytest.raises(ValueError, match="saved"):
            tnt.delta_backward(c, x, dO, saved=saved(cfg(**{**dict(B=1, H=2, Hk=1, L=70, dk=8, dv=8), **other})))
