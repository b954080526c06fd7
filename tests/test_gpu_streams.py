"""The ``stream`` argument of the layer's, the linear memory's and the update's calls: their buffers belong to that
stream, and the results equal the calls' on the current stream, bit for bit, whatever the current
stream is given meanwhile."""
import pytest
import torch

from paper_2511_07343_amd import inputs, tnt

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def calls():
    gen = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=gen)
    unit = lambda t: t / t.norm(dim=-1, keepdim=True)
    B, H, L, d = 2, 2, 150, 64
    x = dict(q=unit(r(B, H, L, d)).bfloat16(), k=unit(r(B, H, L, d)).bfloat16(), v=r(B, H, L, d).bfloat16(),
             g=-r(B, H, L).abs(), lr=torch.sigmoid(r(B, H, L)), S0=r(B, H, d, d))
    x = {n: t.to(DEV) for n, t in x.items()}
    dO, G, pool = r(B, H, L, d).bfloat16().to(DEV), r(3, 200, 260).to(DEV), r(B, H, d, d).to(DEV)
    cfg = tnt.DeltaConfig(B=B, H=H, L=L, dk=d, dv=d)
    orth = tnt.OrthConfig(n=3, rows=200, cols=260)
    saved = tnt.delta_forward(cfg, x)[1]
    torch.cuda.synchronize()

    def step(stream):
        state = pool.clone()
        if stream is not None:  # the state's copy is made on the current stream
            torch.cuda.synchronize()
        return tnt.delta_step(cfg, x, state, stream=stream), state

    layer = inputs.WORKLOADS[0]
    z = tnt.device_inputs(inputs.make_inputs(layer, 0), layer, device=DEV)
    kept = tnt.forward(layer, z)[1]
    torch.cuda.synchronize()
    return dict(
        layer=lambda s: tnt.forward(layer, z, final_state=True, stream=s)[::2],
        layer_backward=lambda s: tuple(tnt.backward(layer, z, z["dO"], saved=kept, stream=s).values()),
        layer_recompute=lambda s: tuple(tnt.backward(layer, z, z["dO"], stream=s).values()),
        layer_steps=lambda s: tnt.step_forward(layer, z, [100, 1, 60], stream=s)[:1],
        forward=lambda s: tnt.delta_forward(cfg, x, final_state=True, stream=s)[::2],
        backward=lambda s: tuple(tnt.delta_backward(cfg, x, dO, saved=saved, stream=s).values()),
        recompute=lambda s: tuple(tnt.delta_backward(cfg, x, dO, stream=s).values()),
        step=step,
        update=lambda s: (tnt.orthogonalise(orth, G, stream=s),))


@pytest.mark.parametrize("name", ["forward", "backward", "recompute", "step", "update", "layer", "layer_backward",
                                  "layer_recompute", "layer_steps"])
@pytest.mark.parametrize("raw", [False, True])
def test_a_given_stream(name, raw, monkeypatch):
    call = calls()[name]
    want = [t.clone() for t in call(None)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    made = []
    empty = tnt._bytes
    monkeypatch.setattr(tnt, "_bytes", lambda n, dev: made.append(torch.cuda.current_stream().cuda_stream) or empty(n, dev))
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)  # the call's kernels wait behind this
    got = call(side.cuda_stream if raw else side)
    # memory that the call has dropped must not come back to the current stream yet
    held = [torch.full((1 << 16,), float("nan"), device=DEV) for _ in range(200)]
    torch.cuda.synchronize()
    assert all(s == side.cuda_stream for s in made) and (made or name == "step")
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.cuda.current_stream() == torch.cuda.default_stream() and len(held) == 200


@pytest.mark.parametrize("name", ["forward", "backward", "step", "update", "layer", "layer_backward", "layer_steps"])
def test_another_current_device(name, monkeypatch):
    """Tensors of a device that is not the current one: the library's launches go to the current device,
    so the tensors' is made current first."""
    call = calls()[name]
    want = [t.clone() for t in call(None)]
    seen, entered, real = [], [], torch.cuda.stream
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0 if entered else 1)

    class entering:
        def __init__(self, s):
            self.s, self.inner = s, real(s)

        def __enter__(self):
            entered.append(self.s)
            seen.append(self.s.device)
            return self.inner.__enter__()

        def __exit__(self, *e):
            entered.pop()
            return self.inner.__exit__(*e)

    monkeypatch.setattr(torch.cuda, "stream", entering)
    got = call(None)
    torch.cuda.synchronize(DEV)
    assert seen == [torch.device(DEV)] and all(torch.equal(a, b) for a, b in zip(got, want))
