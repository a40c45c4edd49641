"""Block tables, slot maps and the page pool against a plain walk over the
requests, and the store of keys and values against plain indexing: whole
numbers and copies, so equal to the last bit."""
import numpy as np
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


def walk(cached, fresh, mask, table, free, page, max_tokens, capacity):
    """The definition, request by request (the pool holds enough)."""
    table = table.copy()
    pool = list(free)
    for r, c in enumerate(cached):
        if mask is not None and not mask[r]:
            pool += table[r, :-(-int(c) // page)].tolist()
    taken, q, lens, slots, positions = 0, [0], [], [], []
    for r, (c, f) in enumerate(zip(cached.tolist(), fresh.tolist())):
        if mask is not None and not mask[r]:
            f, total = 0, 0
        else:
            total = c + f
            for k in range(-(-c // page), -(-total // page)):
                table[r, k] = pool[taken]
                taken += 1
            for x in range(c, total):
                slots.append(int(table[r, x // page]) * page + x % page)
                positions.append(x)
        q.append(q[-1] + f)
        lens.append(total)
    pad = [-1] * (max_tokens - len(slots))
    left = pool[taken:]
    return dict(q_offsets=q, lens=lens, slots=slots + pad, positions=positions + pad, table=table,
                free_pages=left + [-1] * (capacity - len(left)), free_count=[len(left)])


def make(n, page, most_cached, most_fresh, masked, seed):
    rng = np.random.default_rng(seed)
    cached = rng.integers(0, most_cached + 1, n)
    fresh = rng.integers(0, most_fresh + 1, n)
    mask = rng.integers(0, 2, n).astype(np.uint8) if masked else None
    held, all_ = -(-cached // page), -(-(cached + fresh) // page)
    pool = int(all_.sum()) + 5
    ids = rng.permutation(pool).astype(np.int32)
    width = max(1, int(all_.max()))
    table = np.full((n, width), -3, dtype=np.int32)
    at = np.arange(width)[None, :] < held[:, None]
    table[at] = ids[:int(held.sum())]
    return cached, fresh, mask, table, ids[int(held.sum()):], pool


def call(cached, fresh, mask, table, free, capacity, page, max_tokens, **kw):
    full = np.full(capacity, -9, dtype=np.int32)
    full[:len(free)] = free
    up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)  # noqa: E731
    r = pair.page_plan(up(cached.astype(np.int32)), up(fresh.astype(np.int32)), up(table),
                       up(full), up(np.array([len(free)], dtype=np.int64)), page, max_tokens,
                       mask=None if mask is None else up(mask), **kw)
    torch.cuda.synchronize()
    return r


def same(got, want):
    for k, w in want.items():
        g = got[k].cpu().numpy()
        assert np.array_equal(g, np.asarray(w).reshape(g.shape)), k


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("n,page,most_cached,most_fresh", [
    (1, 16, 0, 1), (1, 1, 5, 3), (3, 16, 40, 1), (64, 16, 500, 1), (63, 20, 100, 40),
    (255, 8, 30, 5), (256, 64, 300, 0), (257, 7, 10, 100), (2048, 16, 64, 3), (2049, 16, 64, 3),
    (5000, 32, 100, 9), (2, 128, 1000, 5000)])
def test_plan_against_a_walk(n, page, most_cached, most_fresh, masked):
    log(f"page plan: n={n} page={page} cached<={most_cached} fresh<={most_fresh} mask={masked}")
    for seed in (0, 1):
        cached, fresh, mask, table, free, pool = make(n, page, most_cached, most_fresh, masked, seed)
        room = int(fresh.sum()) + 3 * seed
        got = call(cached, fresh, mask, table, free, pool, page, room)
        assert int(got["status"].item()) == 0
        same(got, walk(cached, fresh, mask, table, free, page, room, pool))


@pytest.mark.parametrize("n", [16_384, 16_385, 70_001])
def test_plan_of_many_against_a_walk(n):
    log(f"page plan: n={n}")
    cached, fresh, mask, table, free, pool = make(n, 8, 20, 2, True, n)
    room = int(fresh.sum()) + 7
    got = call(cached, fresh, mask, table, free, pool, 8, room)
    assert int(got["status"].item()) == 0
    same(got, walk(cached, fresh, mask, table, free, 8, room, pool))


@pytest.mark.parametrize("n", [5, 2500])
def test_all_released_and_none(n):
    log(f"page plan: all released, none released, n={n}")
    cached, fresh, _, table, free, pool = make(n, 16, 90, 4, False, 3)
    for mask in (np.zeros(n, np.uint8), np.ones(n, np.uint8)):
        got = call(cached, fresh, mask, table, free, pool, 16, int(fresh.sum()))
        assert int(got["status"].item()) == 0
        same(got, walk(cached, fresh, mask, table, free, 16, int(fresh.sum()), pool))


@pytest.mark.parametrize("n", [6, 3000])
def test_released_pages_serve_the_same_step(n):
    """An empty free list: the kept requests grow into the released ones' pages."""
    log(f"page plan: pool from released pages, n={n}")
    cached, mask = np.full(n, 32), np.arange(n) % 2
    fresh = np.full(n, 16)
    table = np.full((n, 3), -1, dtype=np.int32)
    table[:, :2] = np.random.default_rng(0).permutation(2 * n).reshape(n, 2)
    free = np.zeros(0, dtype=np.int32)
    got = call(cached, fresh, mask.astype(np.uint8), table, free, 2 * n, 16, 16 * n)
    assert int(got["status"].item()) == 0
    same(got, walk(cached, fresh, mask, table, free, 16, 16 * n, 2 * n))


@pytest.mark.parametrize("n", [4, 2100])
def test_status(n):
    log(f"page plan: what does not fit, n={n}")
    cached, fresh = np.full(n, 8), np.full(n, 16)
    table = np.full((n, 2), -1, dtype=np.int32)
    table[:, 0] = np.arange(n)
    free = np.arange(n, 2 * n - 1).astype(np.int32)          # one page short
    got = call(cached, fresh, None, table, free, 2 * n, 16, 16 * n)
    assert int(got["status"].item()) == pair.ST_PAGES
    want = walk(cached[:-1], fresh[:-1], None, table[:-1], free, 16, 16 * (n - 1), 0)
    assert np.array_equal(got["slots"].cpu().numpy()[:16 * (n - 1)], want["slots"])
    last = got["slots"].cpu().numpy()[16 * (n - 1):]
    assert np.array_equal(last[:8], (n - 1) * 16 + np.arange(8, 16)) and np.all(last[8:] == -1)
    assert int(got["table"][n - 1, 1]) == -1 and int(got["free_count"].item()) == 0
    # too few token entries
    free = np.arange(n, 2 * n).astype(np.int32)
    got = call(cached, fresh, None, table, free, 2 * n, 16, 16 * n - 1)
    assert int(got["status"].item()) == pair.ST_LENGTH
    # a negative length, and a row that is too narrow: the request is left out
    for at, c, f, bit in ((1, -1, 16, pair.ST_LENGTH), (1, 8, -2, pair.ST_LENGTH),
                          (1, 8, 25, pair.ST_PAGES), (1, 2 ** 31 - 1, 2 ** 31 - 1, pair.ST_LENGTH)):
        cc, ff = cached.copy(), fresh.copy()
        cc[at], ff[at] = c, f
        got = call(cc, ff, None, table, free, 2 * n, 16, 16 * n)
        assert int(got["status"].item()) == bit, (c, f)
        lens = got["lens"].cpu().numpy()
        assert lens[at] == 0 and np.all(np.delete(lens, at) == 24)
        assert int(got["q_offsets"][-1]) == 16 * (n - 1)
        assert int(got["free_count"].item()) == 1
    # a list that is full cannot take the released pages
    got = call(cached, fresh, np.zeros(n, np.uint8), table, free, n + n - 1, 16, 16)
    assert int(got["status"].item()) == pair.ST_PAGES
    assert int(got["free_count"].item()) == 2 * n - 1


def test_plan_on_another_stream_and_in_a_graph():
    for n in (100, 2500):
        log(f"page plan: side stream and graph, n={n}")
        cached, fresh, mask, table, free, pool = make(n, 16, 90, 4, True, 4)
        room = int(fresh.sum())
        want = walk(cached, fresh, mask, table, free, 16, room, pool)
        side = torch.cuda.Stream()
        got = call(cached, fresh, mask, table, free, pool, 16, room, stream=side)
        side.synchronize()
        same(got, want)
        full = np.full(pool, -9, dtype=np.int32)
        full[:len(free)] = free
        up = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DEV)  # noqa: E731
        c, f, m = up(cached.astype(np.int32)), up(fresh.astype(np.int32)), up(mask)
        tb, fr, fc = up(table), up(full), up(np.array([len(free)], dtype=np.int64))
        out = dict(q_offsets=torch.empty(n + 1, dtype=torch.int64, device=DEV),
                   lens=torch.empty(n, dtype=torch.int32, device=DEV),
                   slots=torch.empty(room, dtype=torch.int64, device=DEV),
                   positions=torch.empty(room, dtype=torch.int32, device=DEV),
                   free_pages=torch.empty_like(fr),
                   free_count=torch.empty(1, dtype=torch.int64, device=DEV))
        ws = torch.empty(pair.pair_page_plan_workspace_bytes(n), dtype=torch.uint8, device=DEV)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)

        def step():
            pair.pair_page_plan(n, c, f, m, 16, tb, fr, fc, room, out["q_offsets"], out["lens"],
                                out["slots"], out["positions"], out["free_pages"],
                                out["free_count"], ws, st)

        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        rng = np.random.default_rng(1)
        for _ in range(3):
            mask = rng.permutation(mask)
            m.copy_(up(mask))
            tb.copy_(up(table))
            g.replay()
            torch.cuda.synchronize()
            assert int(st.item()) == 0
            same({**out, "table": tb}, walk(cached, fresh, mask, table, free, 16, room, pool))


def test_plan_refusals():
    cached, fresh, mask, table, free, pool = make(4, 16, 90, 4, True, 4)
    ok = dict(cached=cached, fresh=fresh, mask=mask, table=table, free=free, capacity=pool, page=16,
              max_tokens=20)
    call(**ok)
    for error, bad in ((pair.PairError, dict(page=0)), (ValueError, dict(fresh=fresh[:3])),
                       (ValueError, dict(mask=mask[:3])), (ValueError, dict(table=table[:3])),
                       (TypeError, dict(table=table.astype(np.int64))),
                       (TypeError, dict(mask=mask.astype(np.int32)))):
        with pytest.raises(error):
            call(**{**ok, **bad})


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("tokens,heads,dim,page,layout", [
    (1, 1, 8, 1, "token"), (5, 2, 64, 16, "token"), (333, 8, 128, 16, "head"),
    (70, 3, 128, 20, "padded"), (1000, 1, 256, 64, "token"), (64, 40, 128, 16, "token"),
    (37, 5, 24, 7, "padded")])
def test_store_equals_indexing(tokens, heads, dim, page, layout, dtype):
    log(f"cache store: tokens={tokens} heads={heads} dim={dim} page={page} {layout}")
    rng = np.random.default_rng(tokens)
    pages = -(-tokens // page) + 2
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    slots[::4] = np.where(rng.random(len(slots[::4])) < 0.3, -1, slots[::4])
    fused = torch.randn((tokens, 2 * heads + 1, dim), device=DEV).to(dtype)
    fused[0, 0, 0] = float("nan")
    k, v = fused[:, :heads], fused[:, heads + 1:]
    caches = []
    for _ in range(2):
        x = torch.randn((pages, page, heads, dim), device=DEV).to(dtype)
        if layout == "head":
            x = x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
        elif layout == "padded":
            x = torch.randn((pages, page + 2, heads, dim + 8), device=DEV).to(dtype)[:, 1:page + 1, :, :dim]
        caches.append(x)
    want = []
    keep = torch.from_numpy(slots >= 0).to(DEV)
    at = torch.from_numpy(slots).to(DEV)[keep]
    for x, new in zip(caches, (k, v)):
        y = x.clone()
        y[at // page, at % page] = new[keep]
        want.append(y)
    r = pair.cache_store(k, v, torch.from_numpy(slots).to(DEV), *caches)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == 0
    for x, y in zip(caches, want):
        assert torch.equal(x.contiguous().view(torch.int16), y.contiguous().view(torch.int16))


def test_store_status_stream_and_refusals():
    k = torch.randn((6, 2, 64), device=DEV).bfloat16()
    caches = [torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    slots = torch.tensor([0, 48, 2, -1, 2 ** 40, 47], device=DEV)
    side = torch.cuda.Stream()
    r = pair.cache_store(k, k, slots, *caches, stream=side)
    side.synchronize()
    assert int(r["status"].item()) == pair.ST_PAGES
    flat = caches[0].view(48, 2, 64)
    assert torch.equal(flat[[0, 2, 47]], k[[0, 2, 5]])
    assert int((flat != 0).any(2).any(1).sum()) == 3
    none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    pair.cache_store(none, none, slots[:0], *caches)
    ok = dict(k=k, v=k, slots=slots, k_cache=caches[0], v_cache=caches[1])
    for error, bad in ((TypeError, dict(k=k.half())), (ValueError, dict(k=k[:, :1])),
                       (ValueError, dict(v=k[:5])), (TypeError, dict(slots=slots.int())),
                       (ValueError, dict(slots=slots[:5])), (ValueError, dict(k=k[..., :32])),
                       (TypeError, dict(k_cache=caches[0].float(), v_cache=caches[1].float())),
                       (ValueError, dict(v=torch.cat([k, k], 1)[:, :2]))):
        with pytest.raises(error):
            pair.cache_store(**{**ok, **bad})
    odd = torch.randn(6 * 2 * 64 + 8, device=DEV).bfloat16()[4:4 + 768].view(6, 2, 64)
    with pytest.raises(pair.PairError):
        pair.cache_store(odd, odd, slots, *caches)
    torch.cuda.synchronize()
