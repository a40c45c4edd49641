"""What autograd is told of the paged calls and the clipping."""
import pytest
import torch

import paper_2608_11368_amd as pair

DEV = "cuda:0"


def test_written_counts():
    """One write for each tensor, of a view also for what it looks into; nothing
    for what has no count."""
    written = pair._native().written
    base = torch.zeros(8)
    view, other, half = base[2:5], torch.zeros(3), torch.zeros(2).half()
    with torch.inference_mode():
        fixed = torch.zeros(2)
    written()
    written(view, [other, half, None, 3], None, fixed, [])
    assert (base._version, view._version, other._version, half._version) == (1, 1, 1, 1)
    x = torch.ones(3, requires_grad=True)
    y = (x * other).sum()
    written(other)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


@pytest.fixture
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def paged(dtype=torch.bfloat16):
    """Two requests of 40 and 9 keys in 16-token pages, a token each."""
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    k, v = (torch.randn((5, 16, 2, 64), generator=g, device=DEV).to(dtype) for _ in range(2))
    q = torch.randn((2, 4, 64), generator=g, device=DEV).to(dtype)
    table = torch.tensor([[3, 0, 4], [1, -1, -1]], dtype=torch.int32, device=DEV)
    return dict(q=q, k_cache=k, v_cache=v, table=table, q_offsets=torch.arange(3, device=DEV),
                lens=torch.tensor([40, 9], dtype=torch.int32, device=DEV), max_q=1, max_len=40)


@pytest.mark.gpu
def test_values_saved_for_a_gradient(gpu):
    """Gradients, caches and an output that are written in place after a product
    has saved them: its backward pass refuses instead of using the new values."""
    a = paged()
    slots = torch.tensor([5, 70], device=DEV)
    new = torch.randn((2, 2, 64), device=DEV).bfloat16()
    out = torch.zeros_like(a["q"])
    grads = [torch.randn(50, device=DEV), torch.randn(7, device=DEV)]
    flat = torch.randn(57, device=DEV)
    calls = [
        (grads[1], lambda: pair.clip_grads(grads, 1e-3)),
        (flat, lambda: pair.clip_grads(grads, 1e-3, out=[flat[:50], flat[50:]])),
        (a["k_cache"], lambda: pair.cache_store(new, new, slots, a["k_cache"], a["v_cache"])),
        (a["v_cache"], lambda: pair.cache_store(new, new, slots, a["k_cache"], a["v_cache"])),
        (out, lambda: pair.paged_attention(**a, out=out)),
    ]
    for saved, call in calls:
        w = torch.ones(saved.shape, dtype=saved.dtype, device=DEV, requires_grad=True)
        y = (w * saved).sum()
        call()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_a_plan_counts_its_table(gpu):
    def i32(*x):
        return torch.tensor(x, dtype=torch.int32, device=DEV)

    table = torch.full((2, 2), -1, dtype=torch.int32, device=DEV)
    before = table._version
    r = pair.page_plan(i32(0, 0), i32(3, 4), table, i32(5, 6, 7),
                       torch.tensor([3], device=DEV), 16, 7)
    torch.cuda.synchronize()
    assert table._version == before + 1 and r["table"] is table
    with torch.inference_mode():
        pair.page_plan(i32(3, 4), i32(0, 0), table.clone(), r["free_pages"], r["free_count"], 16, 7)
        pair.clip_grads([torch.ones(3, device=DEV)], 0.5)
    torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("wants", ["q", "k_cache", "v_cache"])
def test_attention_is_not_cut_from_the_graph_in_silence(gpu, wants):
    """A backward pass that comes to the attention's results fails; the results
    are the same, and under no_grad or on a given output nothing changes."""
    a = paged()
    want = pair.paged_attention(**a, want_lse=True)
    assert not want["out"].requires_grad
    a[wants] = a[wants].detach().requires_grad_()
    for lse in (False, True):
        r = pair.paged_attention(**a, want_lse=lse)
        assert torch.equal(r["out"], want["out"]) and int(r["status"].item()) == 0
        assert (r["lse"] is None) if not lse else torch.equal(r["lse"], want["lse"])
        for x in (r["out"], r["lse"]) if lse else (r["out"],):
            with pytest.raises(NotImplementedError, match="no gradient"):
                x.float().sum().backward()
        assert not r["status"].requires_grad
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r = pair.paged_attention(**a, stream=side)
    side.synchronize()
    assert torch.equal(r["out"], want["out"]) and r["out"].requires_grad
    with torch.no_grad():
        assert not pair.paged_attention(**a)["out"].requires_grad
    with torch.inference_mode():
        assert not pair.paged_attention(**a)["out"].requires_grad
    out = torch.empty_like(want["out"])
    r = pair.paged_attention(**a, out=out)
    torch.cuda.synchronize()
    assert r["out"] is out and not out.requires_grad and torch.equal(out, want["out"])
