"""The allocating helpers of the paged calls and the clipping in a captured graph:
outputs, workspaces and status words belong to the graph, and every replay
gives what an eager call gives on the inputs that it finds."""
import pytest
import torch

import paper_2608_11368_amd as pair
from tests.gpu_util import DEV, log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pair.lib()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("new", [1, 40])
def test_a_step_of_helpers(new):
    log(f"paged helpers in a graph, {new} new tokens")
    n, page, heads, kv, dim, pages = 3, 16, 4, 2, 64, 40
    rows = n * new
    cached = torch.tensor([100, 7, 33], dtype=torch.int32, device=DEV)
    fresh = torch.full((n,), new, dtype=torch.int32, device=DEV)
    mask = torch.ones(n, dtype=torch.uint8, device=DEV)
    table = torch.full((n, 12), -1, dtype=torch.int32, device=DEV)
    held = [7, 1, 3]
    for r in range(n):
        table[r, :held[r]] = torch.arange(held[r], device=DEV) + sum(held[:r])
    free = torch.full((pages,), -1, dtype=torch.int32, device=DEV)
    free[:pages - 11] = torch.arange(11, pages, device=DEV)
    count = torch.tensor([pages - 11], device=DEV)
    first = [x.clone() for x in (table, mask)]
    k_cache, v_cache = (torch.randn((pages, page, kv, dim), device=DEV).bfloat16() for _ in range(2))
    qkv = torch.randn((rows, heads + 2 * kv, dim), device=DEV).bfloat16()
    grads = [torch.randn(5000, device=DEV), torch.randn(33, device=DEV)]
    outs = [torch.zeros_like(g) for g in grads]

    def step():
        p = pair.page_plan(cached, fresh, table, free, count, page, rows, mask=mask)
        q, k, v = qkv.split([heads, kv, kv], dim=1)
        s = pair.cache_store(k, v, p["slots"], k_cache, v_cache)
        a = pair.paged_attention(q, k_cache, v_cache, table, p["q_offsets"], p["lens"], new, 200,
                                 want_lse=True)
        c = pair.clip_grads(grads, 1.0, out=outs)
        return {**{"plan_" + x: y for x, y in p.items()}, "store": s["status"], **a,
                "norm": c["norm"], "coef": c["coef"], "clip": c["status"]}

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    status = ("plan_status", "store", "status", "clip")
    for i in range(4):
        table.copy_(first[0])
        mask.copy_(first[1])
        mask[i % n] = 0 if i < n else 1
        qkv.copy_(torch.randn(qkv.shape, device=DEV))
        grads[0].mul_(3.0 if i % 2 else 0.01)
        if i == 2:
            grads[1][5] = float("inf")                   # this replay's status, and no other's
        for x in got.values():
            if x.dtype == torch.int32 and x.numel() == 1:
                x.fill_(-1)                              # words that only a replay clears
        graph.replay()
        torch.cuda.synchronize()
        have = {x: y.clone() for x, y in got.items()}
        table.copy_(first[0])
        want = step()
        torch.cuda.synchronize()
        for x in status:
            assert int(have[x].item()) == (pair.ST_NONFINITE if x == "clip" and i >= 2 else 0), (i, x)
        rows_of = int(have["plan_q_offsets"][-1].item())
        assert rows_of == rows - (new if i < n else 0)
        for x in have:
            if x in ("out", "lse"):
                assert torch.equal(have[x][:rows_of], want[x][:rows_of]), (i, x)
            elif x != "norm" or i < 2:
                assert torch.equal(have[x], want[x]), (i, x)
        busy = torch.randn(512, 512, device=DEV)         # the program's own work in between
        (busy @ busy).sum().item()
