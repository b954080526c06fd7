"""The orthogonalised update on the GPU against the fp64 form.

Bounds on |x - y|_F / |y|_F.  fp32: an operand of 22 bits, 2^-22 of the product's norm, in three
products a step and five steps, and a singular value far below the norm is amplified with its
noise, measured in 64-bit emulation at up to 25 times that: 25 * 15 * 2^-22 < 1e-4.  bf16: 11-bit
operands of the products with X, the same with 2^-11 and independent roundings (sqrt(15) in place
of 15, and 2 in place of 25: the last two steps' errors are not amplified, and only theirs last), and
the result's own 2^-8: sqrt(2^-16 + 60 * 2^-22) < 6e-3.
"""
import pytest
import torch

from oracle import linear_oracle as O
from paper_2511_07343_amd import tnt
from parity_log import check_err

pytestmark = pytest.mark.gpu
TOL = {torch.float32: 1e-4, torch.bfloat16: 6e-3}
DEV = "cuda:0"
MUON = (3.4445, -4.7750, 2.0315)


def matrices(n, r, c, dtype, seed=0, scale=1e-3):
    gen = torch.Generator().manual_seed(seed)
    rank = max(1, min(r, c) // 16)
    strong = torch.randn(n, r, rank, generator=gen) @ torch.randn(n, rank, c, generator=gen)
    return (scale * (torch.randn(n, r, c, generator=gen) + strong)).to(dtype)


def check(case, got, G, coef, eps=1e-7, scale=1.0):
    bad = []
    for i in range(G.shape[0]):
        want = O.orthogonalise(G[i], coef, eps, scale)
        e = ((got[i].double().cpu() - want).norm() / want.norm()).item()
        if not check_err(case, f"out[{i}]", e, TOL[got.dtype]):
            bad.append((i, e))
    assert not bad, bad


def run(G, **kw):
    cfg = tnt.OrthConfig(n=G.shape[0], rows=G.shape[1], cols=G.shape[2],
                         dtype=int(G.dtype == torch.bfloat16), **kw)
    out = tnt.orthogonalise(cfg, G)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,r,c", [
    (1, 1, 1), (3, 1, 7), (2, 5, 3), (2, 16, 16), (3, 33, 20), (2, 32, 300), (2, 700, 31),
    (4, 64, 256), (4, 256, 64), (2, 65, 300), (1, 64, 1024), (2, 512, 128), (2, 128, 512), (1, 127, 129),
    (1, 129, 129), (2, 130, 200), (1, 64, 1025), (1, 513, 128), (2, 300, 257), (1, 1, 3000), (1, 384, 640)])
def test_sizes(n, r, c, dtype):
    """One element to several tiles, both orientations, both forms and the sizes between them."""
    G = matrices(n, r, c, dtype, seed=r + c)
    check(f"orth {n}x{r}x{c} {dtype}", run(G.to(DEV)), G, [MUON] * 5)


@pytest.mark.parametrize("r,c", [(40, 100), (150, 200)])
def test_coefficients_steps_scale(r, c):
    """Other coefficients each step, other step counts, eps, an output scale."""
    G = matrices(2, r, c, torch.float32, seed=1)
    coef = [(4.0, -6.0, 2.5), (2.0, -1.5, 0.5), (1.5, -0.5, 0.0)]
    check("orth coef", run(G.to(DEV), steps=3, coef=coef, scale=0.2, eps=1e-3), G, coef, 1e-3, 0.2)
    check("orth one step", run(G.to(DEV), steps=1), G, [MUON])


@pytest.mark.parametrize("r,c", [(64, 250), (128, 512), (129, 300), (7, 1000)])
def test_number_format(r, c):
    """One step with (1, 0, 0) is the scaling alone: every element to the 22 bits of its two
    terms (2^-22, and twice that for the products on the way), none off by a term."""
    G = matrices(1, r, c, torch.float32, seed=8)
    out = run(G.to(DEV), steps=1, coef=(1.0, 0.0, 0.0)).double().cpu()[0]
    want = G[0].double() / (G[0].double().norm() + 1e-7)
    big = want.abs() > 2.0 ** -12 * want.abs().max()
    assert ((out - want).abs() / want.abs())[big].max() <= 2.0 ** -20


@pytest.mark.parametrize("r,c", [(24, 60), (140, 160)])
def test_converges_to_an_orthogonal_factor(r, c):
    """The cubic iteration converges: rows orthonormal, singular vectors kept."""
    G = matrices(1, r, c, torch.float32, seed=2)
    G += 0.05 * torch.eye(r, c)
    out = run(G.to(DEV), steps=16, coef=(1.5, -0.5, 0.0)).double().cpu()[0]
    U, S, V = torch.linalg.svd(G[0].double(), full_matrices=False)
    grown = S / S.norm()
    for _ in range(16):
        grown = 1.5 * grown - 0.5 * grown ** 3
    assert (out - (U * grown) @ V).norm() <= 1e-4 * grown.norm()


@pytest.mark.parametrize("scale", [1e-30, 1e25])
@pytest.mark.parametrize("r,c", [(30, 50), (140, 150)])
def test_any_scale(r, c, scale):
    """Squares that leave the range of fp32: the norm is summed in 64 bits."""
    G = matrices(1, r, c, torch.float32, seed=3, scale=scale)
    check(f"orth scale {scale}", run(G.to(DEV), eps=0.0), G, [MUON] * 5, 0.0)


@pytest.mark.parametrize("r,c", [(40, 60), (140, 150)])
def test_zero_and_nan_matrices(r, c):
    """A zero matrix gives zeros; NaN and infinity spoil their own matrix alone."""
    G = matrices(4, r, c, torch.float32, seed=4)
    clean = run(G.to(DEV))
    G[1] = 0.0
    G[2, r // 2, c // 2] = float("nan")
    G[3, 0, 0] = float("inf")
    out = run(G.to(DEV))
    assert torch.equal(out[0], clean[0]) and torch.equal(out[1], torch.zeros_like(out[1]))
    assert torch.isnan(out[2]).any() and torch.isnan(out[3]).any()


@pytest.mark.parametrize("r,c", [(40, 60), (150, 140)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_in_place(r, c, dtype):
    """Rows further apart than their length and off any alignment, transposed views, out = G."""
    G = matrices(2, r, c, dtype, seed=5)
    want = run(G.to(DEV))
    wide = torch.zeros(2, r + 1, c + 3, dtype=dtype, device=DEV)
    wide[:, :r, :c] = G.to(DEV)
    view = wide[:, :r, :c]
    cfg = tnt.OrthConfig(n=2, rows=r, cols=c, dtype=int(dtype == torch.bfloat16))
    out = torch.full((2, r + 2, c + 5), 7.0, dtype=dtype, device=DEV)
    tnt.orthogonalise(cfg, view, out=out[:, :r, :c])
    assert torch.equal(out[:, :r, :c], want)
    assert (out[:, r:] == 7).all() and (out[:, :, c:] == 7).all()
    t = G.to(DEV).transpose(1, 2).contiguous().transpose(1, 2)
    check("orth transposed", tnt.orthogonalise(cfg, t), G, [MUON] * 5)
    tnt.orthogonalise(cfg, view, out=view)
    torch.cuda.synchronize()
    assert torch.equal(view, want) and (wide[:, r:] == 0).all() and (wide[:, :, c:] == 0).all()


@pytest.mark.parametrize("r,c", [(64, 200), (200, 260)])
def test_repeats_graph_and_workspace(r, c):
    """Bitwise the same from a workspace full of NaN, on a side stream and in graph replays."""
    G = matrices(3, r, c, torch.float32, seed=6).to(DEV)
    want = run(G)
    cfg = tnt.OrthConfig(n=3, rows=r, cols=c)
    ws = torch.full((max(16, cfg.size),), 255, dtype=torch.uint8, device=DEV)
    out = torch.empty_like(G)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        tnt.orthogonalise(cfg, G, out=out, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        tnt.orthogonalise(cfg, G, out=out, workspace=ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        run(G)


def test_batch_of_initial_weights():
    """Every memory and head of the deep memories' weight gradients [M][H][hid][d] in one call."""
    G = matrices(6, 256, 64, torch.float32, seed=7)
    check("orth memories", run(G.view(2, 3, 256, 64).to(DEV).flatten(0, 1)), G, [MUON] * 5)


def test_no_matrices():
    cfg = tnt.OrthConfig(n=0, rows=8, cols=8)
    assert tnt.orthogonalise(cfg, torch.empty(0, 8, 8, device=DEV)).shape == (0, 8, 8)


@pytest.mark.parametrize("n,r,c", [(2, 64, 250), (1, 64, 1024), (1, 64, 1025), (2, 130, 200), (2, 300, 257),
                                   (1, 512, 128), (1, 1030, 700)])
def test_bf16_is_the_result_rounded_once(n, r, c):
    """In both forms.  With an error e of the norm before it (the fp32 bound), a rounding goes the other
    way for a part e / ulp of the elements, by an ulp: sqrt(e * ulp) of the norm, ulp at most 2^-7."""
    G = matrices(n, r, c, torch.bfloat16, seed=r)
    out = run(G.to(DEV)).double().cpu()
    for i in range(n):
        want = O.orthogonalise(G[i], [MUON] * 5).to(torch.bfloat16).double()
        e = ((out[i] - want).norm() / want.norm()).item()
        assert check_err(f"orth rounded {n}x{r}x{c}", f"out[{i}]", e, (1e-4 * 2.0 ** -7) ** 0.5), (i, e)


def test_rows_far_apart():
    """Rows 2^21 elements apart, past the 32-bit offsets of the form for one workgroup."""
    G = matrices(1, 8, 12, torch.float32, seed=9)
    far = torch.empty_strided((1, 8, 12), (1 << 24, 1 << 21, 1), device=DEV)
    far.copy_(G)
    out = torch.empty(1, 8, 12, device=DEV)
    tnt.orthogonalise(tnt.OrthConfig(n=1, rows=8, cols=12), far, out=out)
    torch.cuda.synchronize()
    check("orth far rows", out, G, [MUON] * 5)


@pytest.mark.parametrize("r,c", [(40, 60), (150, 140)])
def test_transposed_batch(r, c):
    """[rows][matrices][cols] memory: the same results in the same layout, in place too."""
    G = matrices(3, r, c, torch.float32, seed=10)
    want = run(G.to(DEV))
    side = G.to(DEV).transpose(0, 1).contiguous().transpose(0, 1)
    cfg = tnt.OrthConfig(n=3, rows=r, cols=c)
    out = tnt.orthogonalise(cfg, side)
    assert out.stride() == side.stride() and torch.equal(out, want)
    tnt.orthogonalise(cfg, side, out=side)
    torch.cuda.synchronize()
    assert torch.equal(side, want)


@pytest.mark.parametrize("r,c", [(40, 64), (136, 144)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_first_element_anywhere(r, c, dtype):
    """Matrices that begin inside a buffer, their rows whole 16-byte pieces all the same."""
    G = matrices(2, r, c, dtype, seed=11)
    cfg = tnt.OrthConfig(n=2, rows=r, cols=c, dtype=int(dtype == torch.bfloat16))
    for off in (1, 3):
        src, dst = (torch.full((2 * r * c + 8,), 7.0, dtype=dtype, device=DEV) for _ in range(2))
        g, out = (t[off:off + 2 * r * c].view(2, r, c) for t in (src, dst))
        g.copy_(G)
        tnt.orthogonalise(cfg, g, out=out)
        torch.cuda.synchronize()
        check("orth offset", out, G, [MUON] * 5)
        assert (dst[:off] == 7).all() and (dst[off + 2 * r * c:] == 7).all()


@pytest.mark.parametrize("scale", [1e-36, 1e-37, 1e-39])
@pytest.mark.parametrize("r,c", [(30, 50), (140, 150)])
def test_norms_near_the_smallest_numbers(r, c, scale):
    """A norm whose reciprocal leaves fp32 (entries with few bits left, but exact as given), without
    and with an eps as small."""
    G = matrices(1, r, c, torch.float32, seed=12, scale=scale)
    check(f"orth scale {scale}", run(G.to(DEV), eps=0.0), G, [MUON] * 5, 0.0)
    tiny = torch.tensor(1e-39).item()
    check(f"orth scale {scale} eps", run(G.to(DEV), eps=tiny), G, [MUON] * 5, tiny)
    assert torch.equal(run(torch.zeros(2, r, c, device=DEV), eps=tiny), torch.zeros(2, r, c, device=DEV))


@pytest.mark.parametrize("n,r,c", [(49, 64, 1024), (50, 33, 513), (52, 700, 50), (1, 64, 1000), (2, 600, 33)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_longer_sides_of_513_to_1024(n, r, c, dtype):
    """Both sides of the rule: many matrices in a workgroup each, a few of them in tiles."""
    G = matrices(n, r, c, dtype, seed=n + r)
    check(f"orth {n}x{r}x{c} {dtype}", run(G.to(DEV)), G, [MUON] * 5)


@pytest.mark.parametrize("n,r,c", [(4, 64, 256), (2, 300, 31), (2, 65, 300), (3, 500, 510), (1, 1030, 700), (2, 129, 640)])
def test_fp32_accuracy(n, r, c):
    """Operands of 22 bits, each product's rounding independent: 2^-23 of its norm, sqrt(15) of them, the
    amplification of 25; one term less anywhere is 2^-12 in its place."""
    G = matrices(n, r, c, torch.float32, seed=n * r)
    out = run(G.to(DEV))
    for i in range(n):
        want = O.orthogonalise(G[i], [MUON] * 5)
        e = ((out[i].double().cpu() - want).norm() / want.norm()).item()
        assert check_err(f"orth fp32 {n}x{r}x{c}", f"out[{i}]", e, 25 * 15 ** 0.5 * 2.0 ** -23), (i, e)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_matrices_of_many_tiles(dtype):
    """Ragged sides of several tiles, more workgroups than the card takes at once; matrices at the ends and
    in between."""
    G = matrices(64, 500, 510, dtype, seed=13)
    out = run(G.to(DEV))
    pick = [0, 7, 31, 63]
    check(f"orth many {dtype}", out[pick], G[pick], [MUON] * 5)
