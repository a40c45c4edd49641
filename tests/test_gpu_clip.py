"""Gradient norm and clipping against 64 bits.

The squares and sums are fp64, so the norm is rounded once (2^-24, and far
less from the sums); the factor is max_norm / norm rounded once; an output is
a rounded product of the gradient and the rounded factor: for fp32 within
2 * 2^-24 of the exact one, for a 16-bit type within u more (subnormal results:
within half of the smallest one)."""
import math

import pytest
import torch

import paper_2608_11368_amd as pair
from tests.gpu_util import DEV, log

pytestmark = pytest.mark.gpu
U = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pair.lib()
    yield
    torch.cuda.synchronize()


def make(sizes, dtypes, scale, seed=0, offset=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = torch.empty(n + offset, device=DEV).normal_(generator=g).mul_(scale)
        out.append(t.to(dtypes[i % len(dtypes)])[offset:])
    return out


def check(grads, r, outs, max_norm):
    exact = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    assert int(r["status"].item()) == 0
    assert abs(float(r["norm"].item()) - exact) <= 1.01 * 2.0 ** -24 * exact
    coef = max_norm / exact if exact > max_norm else 1.0
    assert abs(float(r["coef"].item()) - coef) <= 1.01 * 2.0 ** -24 * coef
    for g, o in zip(grads, outs):
        want = g.double() * coef
        bar = want.abs() * (2.01 * 2.0 ** -24 + U[o.dtype]) + TINY[o.dtype]
        assert bool(((o.double() - want).abs() <= bar).all()), (g.numel(), o.dtype)


F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
SIZES = [
    [1], [7], [8], [0, 9, 0], [4095], [4096], [4097], [8192 + 13], [1, 2, 3, 4, 5, 6, 7, 8, 9],
    [100_003, 1, 4096, 12_288, 5], [2_000_001], list(range(1, 330)), [17] * 700,
]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("types", [[F32], [BF16], [F16], [BF16, F32, F16]], ids=str)
def test_out_of_place_and_in_place(sizes, types):
    log(f"clip: {len(sizes)} tensors up to {max(sizes)} {types}")
    for scale, max_norm in ((1.0, 0.25), (1e-3, 1e6)):
        grads = make(sizes, types, scale)
        outs = [torch.full_like(g, 5.0) for g in grads]
        r = pair.clip_grads(grads, max_norm, out=outs)
        torch.cuda.synchronize()
        check(grads, r, outs, max_norm)
        wide = [torch.full(g.shape, 5.0, device=DEV) for g in grads]
        r = pair.clip_grads(grads, max_norm, out=wide)
        torch.cuda.synchronize()
        check(grads, r, wide, max_norm)
        mine = [g.clone() for g in grads]
        r2 = pair.clip_grads(mine, max_norm)
        torch.cuda.synchronize()
        assert torch.equal(r2["norm"], r["norm"])
        for a, b in zip(mine, outs):
            assert torch.equal(a, b)


@pytest.mark.parametrize("offset", [1, 3])
def test_views_at_any_element(offset):
    """Views that start inside a vector, into a flat buffer at odd places."""
    log(f"clip: views {offset} elements in")
    sizes = [1000, 33, 4096, 5, 70_001]
    for types in ([F32], [BF16], [F16]):
        grads = make(sizes, types, 1.0, seed=offset, offset=offset)
        flat = torch.full((sum(sizes) + offset + 9,), 7.0, device=DEV)
        views = list(torch.split(flat[offset:offset + sum(sizes)], sizes))
        r = pair.clip_grads(grads, 0.5, out=views)
        torch.cuda.synchronize()
        check(grads, r, views, 0.5)
        assert bool((flat[:offset] == 7).all()) and bool((flat[offset + sum(sizes):] == 7).all())


def test_extremes():
    """Squares beyond fp32's range, zeros, and the bound itself."""
    log("clip: large, small and zero gradients")
    big = [torch.full((1000,), 1e30, device=DEV), torch.full((3,), -2e30, device=DEV)]
    outs = [torch.empty_like(g) for g in big]
    r = pair.clip_grads(big, 1.0, out=outs)
    torch.cuda.synchronize()
    check(big, r, outs, 1.0)
    small = [torch.full((1000,), 1e-30, device=DEV)]
    r = pair.clip_grads(small, 1e-30, out=[torch.empty_like(small[0])])
    torch.cuda.synchronize()
    check(small, r, r["out"], float(torch.tensor(1e-30)))
    zero = [torch.zeros(5000, device=DEV)]
    r = pair.clip_grads(zero, 1.0)
    torch.cuda.synchronize()
    assert float(r["norm"].item()) == 0.0 and float(r["coef"].item()) == 1.0
    exact = [torch.tensor([3.0, 4.0], device=DEV)]
    r = pair.clip_grads(exact, 5.0)
    torch.cuda.synchronize()
    assert float(r["coef"].item()) == 1.0 and exact[0].tolist() == [3.0, 4.0]
    empty = [torch.empty(0, device=DEV)]
    r = pair.clip_grads(empty, 5.0)
    torch.cuda.synchronize()
    assert float(r["norm"].item()) == 0.0


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_non_finite_gradients_stay(bad):
    log(f"clip: a gradient of {bad}")
    grads = make([5000, 40], [BF16], 10.0)
    grads[0][4321] = bad
    outs = [torch.zeros_like(g) for g in grads]
    r = pair.clip_grads(grads, 1.0, out=outs)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == pair.ST_NONFINITE and float(r["coef"].item()) == 1.0
    norm = float(r["norm"].item())
    assert math.isnan(norm) if math.isnan(bad) else norm == math.inf
    for g, o in zip(grads, outs):
        assert torch.equal(g.view(torch.int16), o.view(torch.int16))
    mine = [g.clone() for g in grads]
    pair.clip_grads(mine, 1.0)
    torch.cuda.synchronize()
    for a, b in zip(mine, grads):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_norm_alone():
    log("clip: the norm alone")
    grads = make([70_000, 3], [F32], 100.0)
    before = [g.clone() for g in grads]
    r = pair.clip_grads(grads, math.inf)
    torch.cuda.synchronize()
    check(grads, r, before, math.inf)
    for a, b in zip(grads, before):
        assert torch.equal(a, b)


def test_gradient_of_the_estimator_on_a_stream_and_in_a_graph():
    """The batch-mean gradient and its clipped form, on a side stream and
    replayed from a graph on new scores, against the eager calls' bits."""
    log("clip: after the batch-mean gradient, side stream and graph")
    B, G, D = 6, 8, 5000
    off = torch.arange(0, (B + 1) * G, G, device=DEV)
    scores = torch.randn((B * G, D), device=DEV)
    coeff = torch.randn(B * G, device=DEV)
    grad, out = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
    norm, coef = torch.empty(1, device=DEV), torch.empty(1, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(pair.pair_clip_grads_workspace_bytes(2), dtype=torch.uint8, device=DEV)

    def step():
        pair.pair_weighted_grad(B, B * G, off, scores, coeff, grad, 1, st)
        pair.pair_clip_grads([grad[:3000], grad[3000:]], 1.0, norm, coef, ws,
                             [out[:3000], out[3000:]], st)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for k in range(3):
        scores.copy_(torch.randn((B * G, D), device=DEV) * (0.001 if k == 1 else 1.0))
        g.replay()
        torch.cuda.synchronize()
        mean = pair.weighted_grad(off, scores, coeff, reduce=True, stream=side)["out"]
        r = pair.clip_grads([mean[:3000], mean[3000:]], 1.0, stream=side)
        side.synchronize()
        assert int(st.item()) == 0
        assert torch.equal(norm, r["norm"]) and torch.equal(coef, r["coef"])
        assert torch.equal(out, mean)


def test_refusals():
    g = torch.randn(10, device=DEV)
    for error, kw in (
            (ValueError, dict(grads=[])), (ValueError, dict(grads=[g.cpu()])),
            (TypeError, dict(grads=[g.double()])), (ValueError, dict(grads=[g[::2]])),
            (ValueError, dict(grads=[g], out=[g[:5].clone()])), (ValueError, dict(grads=[g], out=[])),
            (pair.PairError, dict(grads=[g], out=[g.half()])),
            (pair.PairError, dict(grads=[g], max_norm=0.0)),
            (pair.PairError, dict(grads=[g], max_norm=float("nan")))):
        with pytest.raises(error):
            pair.clip_grads(**{"max_norm": 1.0, **kw})
    torch.cuda.synchronize()
