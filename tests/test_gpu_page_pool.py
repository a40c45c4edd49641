"""The page pool over several steps: a pool that runs out, the recovery from it,
and lists that hold what is no page.  Whole numbers, equal to the last bit."""
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


def i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def count(x):
    return torch.tensor([x], dtype=torch.int64, device=DEV)


def listed(r):
    return r["free_pages"][:int(r["free_count"].item())].tolist()


@pytest.mark.parametrize("n", [4, 70, 2048, 2049, 5000])
@pytest.mark.parametrize("cached,fresh,short", [(8, 16, 1), (16, 1, 1), (0, 40, 5), (20, 13, 3)])
def test_what_ran_short_can_be_released(n, cached, fresh, short):
    """The pool lacks `short` pages: the requests at the end keep the lengths that
    their pages hold, and when they are released with those, each page returns to
    the list once and nothing else does."""
    log(f"page pool: {short} pages short, n={n}, {fresh} after {cached}")
    page = 16
    held, need = -(-cached // page), -(-(cached + fresh) // page)
    ids = np.random.default_rng(n).permutation(n * need).astype(np.int32)
    table = np.full((n, need), -1, dtype=np.int32)
    table[:, :held] = ids[:n * held].reshape(n, held)
    free = np.full(n * need, -1, dtype=np.int32)
    pool = n * (need - held) - short
    free[:pool] = ids[n * held:n * held + pool]
    tab = i32(table)
    a = pair.page_plan(i32([cached] * n), i32([fresh] * n), tab, i32(free), count(pool), page,
                       n * fresh)
    torch.cuda.synchronize()
    assert int(a["status"].item()) == pair.ST_PAGES and listed(a) == []
    got = np.full(n, need - held)              # new pages: in request order until the last
    for r in range(n - 1, -1, -1):
        lack = min(short, got[r])
        got[r] -= lack
        short -= lack
    want = np.minimum(cached + fresh, (held + got) * page)
    assert np.array_equal(a["lens"].cpu().numpy(), want)
    rows = tab.cpu().numpy()
    has = np.arange(need)[None, :] < (held + got)[:, None]
    assert np.all(rows[~has] == -1)
    assert sorted(rows[has].tolist()) == sorted(ids[:n * held + pool].tolist())
    # the tokens with a slot are those below the length
    slots = a["slots"].cpu().numpy().reshape(n, fresh)
    below = cached + np.arange(fresh)[None, :] < want[:, None]
    assert np.array_equal(slots >= 0, below)
    # release the ones that ran short, then everyone
    mask = (got == need - held).astype(np.uint8)
    b = pair.page_plan(a["lens"], i32([0] * n), tab, a["free_pages"], a["free_count"], page, 1,
                       mask=torch.from_numpy(mask).to(DEV))
    torch.cuda.synchronize()
    assert int(b["status"].item()) == 0
    assert listed(b) == [p for r in np.flatnonzero(mask == 0) for p in rows[r, :held + got[r]]]
    c = pair.page_plan(b["lens"], i32([0] * n), tab, b["free_pages"], b["free_count"], page, 1,
                       mask=torch.zeros(n, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    assert int(c["status"].item()) == 0
    assert sorted(listed(c)) == sorted(ids[:n * held + pool].tolist())


@pytest.mark.parametrize("n", [3, 2100])
def test_what_ran_short_can_go_on(n):
    """The last request gets its missing tokens a step later, from released pages."""
    log(f"page pool: short, then served, n={n}")
    page = 16
    table = np.full((n, 3), -1, dtype=np.int32)
    table[:, 0] = np.arange(n)
    tab, free = i32(table), np.full(2 * n, -1, dtype=np.int32)
    free[:n - 1] = np.arange(n, 2 * n - 1)
    a = pair.page_plan(i32([8] * n), i32([16] * n), tab, i32(free), count(n - 1), page, 16 * n)
    mask = torch.ones(n, dtype=torch.uint8, device=DEV)
    mask[0] = 0
    fresh = np.zeros(n, dtype=np.int32)
    fresh[-1] = 8
    b = pair.page_plan(a["lens"], i32(fresh), tab, a["free_pages"], a["free_count"], page, 8,
                       mask=mask)
    torch.cuda.synchronize()
    assert int(a["lens"][-1].item()) == 16 and int(b["status"].item()) == 0
    assert b["slots"].tolist() == [0 * page + x for x in range(8)]      # request 0's first page
    assert b["positions"].tolist() == list(range(16, 24))
    assert int(b["lens"][-1].item()) == 24 and listed(b) == [n]


@pytest.mark.parametrize("n", [2, 2100])
def test_an_entry_that_is_no_page(n):
    """A negative entry of the list or of a released row sets the status, whether
    a request gets it or it stays listed; the others keep what is theirs."""
    log(f"page pool: negative entries, n={n}")
    page, cap = 16, 2 * n + 4
    for taken in (True, False):
        for released in (True, False):
            table = np.full((n, 2), -1, dtype=np.int32)
            cached, fresh = np.zeros(n), np.zeros(n)
            mask = np.ones(n, dtype=np.uint8)
            free = np.full(cap, -1, dtype=np.int32)
            if released:
                cached[0], mask[0] = 20, 0
                table[0] = [5, -1]
                pool = [5, -1]
                left = 0
            else:
                free[:3], left = [7, -4, 9], 3
                pool = [7, -4, 9]
            fresh[-1] = 32 if taken else 0
            r = pair.page_plan(i32(cached), i32(fresh), i32(table), i32(free), count(left), page, 32,
                               mask=torch.from_numpy(mask).to(DEV))
            torch.cuda.synchronize()
            assert int(r["status"].item()) == pair.ST_PAGES, (taken, released)
            assert listed(r) == (pool[2:] if taken else pool)
            if taken:
                assert r["slots"].tolist() == [pool[0] * page + x for x in range(16)] + [-1] * 16


@pytest.mark.parametrize("n", [1, 2100])
def test_a_count_that_the_list_does_not_hold(n):
    """A free count below zero or beyond the list sets the status; the plan then
    takes the list as empty or full."""
    log(f"page pool: counts outside the list, n={n}")
    cap = n + 3
    for given, taken in ((-1, 0), (cap + 1, cap), (2 ** 40, cap)):
        table = torch.full((n, 2), -1, dtype=torch.int32, device=DEV)
        r = pair.page_plan(i32([0] * n), i32([1] * n), table, i32(np.arange(cap)), count(given), 16, n)
        torch.cuda.synchronize()
        assert int(r["status"].item()) == pair.ST_PAGES, given
        assert listed(r) == list(range(n, taken))
        assert r["slots"].tolist() == ([x * 16 for x in range(n)] if taken else [-1] * n)
    for fine in (n, cap):
        table = torch.full((n, 2), -1, dtype=torch.int32, device=DEV)
        r = pair.page_plan(i32([0] * n), i32([1] * n), table, i32(np.arange(cap)), count(fine), 16, n)
        torch.cuda.synchronize()
        assert int(r["status"].item()) == 0 and listed(r) == list(range(n, fine))


def walk(cached, fresh, mask, table, free, page, max_tokens, cap):
    """The definition, request by request: requests that do not fit are left out,
    a pool that runs out leaves -1 and shorter lengths, a list that is full drops
    what is beyond it."""
    table, width, status = table.copy(), table.shape[1], 0
    fits = []
    for c, f, live in zip(cached.tolist(), fresh.tolist(), mask.tolist()):
        good = c >= 0 and f >= 0 and c + f < 2 ** 31
        status |= 0 if good else pair.ST_LENGTH
        if good and -(-(c + f if live else c) // page) > width:
            good, status = False, status | pair.ST_PAGES
        fits.append(good)
    pool = list(free)
    for r, c in enumerate(cached.tolist()):
        if fits[r] and not mask[r]:
            pool += table[r, :-(-c // page)].tolist()
    if any(p < 0 for p in pool):
        status |= pair.ST_PAGES
    taken, q, lens, slots, positions = 0, [0], [], [], []
    for r, (c, f) in enumerate(zip(cached.tolist(), fresh.tolist())):
        if not fits[r] or not mask[r]:
            q.append(q[-1])
            lens.append(0)
            continue
        total, held = c + f, -(-c // page)
        for k in range(held, -(-total // page)):
            if taken >= len(pool) and total == c + f:
                total, status = k * page, status | pair.ST_PAGES
            table[r, k] = pool[taken] if taken < len(pool) else -1
            taken += 1
        for x in range(c, c + f):
            p = int(table[r, x // page])
            slots.append(p * page + x % page if p >= 0 else -1)
            positions.append(x)
        q.append(q[-1] + f)
        lens.append(total)
    left = pool[taken:]
    if len(left) > cap:
        status |= pair.ST_PAGES
    if len(slots) > max_tokens:
        status |= pair.ST_LENGTH
    pad = [-1] * (max_tokens - len(slots))
    return dict(q_offsets=q, lens=lens, slots=(slots + pad)[:max_tokens],
                positions=(positions + pad)[:max_tokens], table=table,
                free_pages=(left + [-1] * cap)[:cap], free_count=[min(len(left), cap)], status=[status])


@pytest.mark.parametrize("n", [1, 2, 5, 63, 64, 65, 256, 1000, 2047, 2048, 2049, 4000, 16_384, 17_000])
def test_random_plans_against_a_walk(n):
    """Pools that are short, exact or ample, lists that are too short for what
    comes back, requests that do not fit, masks of every density."""
    log(f"page pool: random plans of {n}")
    for seed in range(12 if n < 3000 else 4):
        rng = np.random.default_rng([n, seed])
        page = int(rng.choice([1, 3, 16, 20, 64]))
        cached = rng.integers(0, int(rng.choice([2, 30, 200])), n)
        fresh = rng.integers(0, int(rng.choice([2, 9, 60])), n)
        mask = (rng.random(n) < rng.choice([0.0, 0.2, 0.6, 1.0, 1.0])).astype(np.uint8)
        held, need = -(-cached // page), -(-(cached + fresh) // page)
        width = max(1, int(need.max()) - int(rng.integers(0, 2)), int(held.max()))
        ids = rng.permutation(int(need.sum()) + 9).astype(np.int32)
        table = np.full((n, width), -1, dtype=np.int32)
        at = np.arange(width)[None, :] < held[:, None]
        table[at] = ids[:int(held.sum())]
        wanted = int((need - held).sum())
        some = int(rng.choice([0, wanted // 3, max(0, wanted - 1), wanted, wanted + 9]))
        free = ids[int(held.sum()):][:some]
        cap = max(1, len(free) + int(rng.choice([0, 3, int(held.sum())])))
        if rng.random() < 0.3:
            cached[rng.integers(0, n)] = -1
        if rng.random() < 0.3:
            fresh[rng.integers(0, n)] = 2 ** 31 - 1
        live = mask != 0
        room = int(rng.choice([0, 1, 5])) + int(fresh[live & (fresh < 1000)].sum())
        room = max(0, room - int(rng.choice([0, 0, 3])))
        full = np.full(cap, -9, dtype=np.int32)
        full[:len(free)] = free
        r = pair.page_plan(i32(cached), i32(fresh), i32(table), i32(full), count(len(free)), page, room,
                           mask=torch.from_numpy(mask).to(DEV))
        torch.cuda.synchronize()
        want = walk(cached, fresh, mask, table, free, page, room, cap)
        for k, w in want.items():
            got = r[k].cpu().numpy()
            assert np.array_equal(got, np.asarray(w).reshape(got.shape)), (seed, k)


@pytest.mark.parametrize("n", [2, 600, 2500])
@pytest.mark.parametrize("cap", [0, 1, 5])
def test_a_short_list_and_many_released_pages(n, cap):
    """More pages change hands in one step than the list has entries: they go
    straight from the released requests to the others."""
    log(f"page pool: a list of {cap}, {n} requests")
    page, half = 16, n // 2
    table = np.full((n, 4), -1, dtype=np.int32)
    table[:half, :3] = np.random.default_rng(n).permutation(3 * half).reshape(half, 3)
    cached, fresh = np.where(np.arange(n) < half, 40, 0), np.where(np.arange(n) < half, 0, 48)
    mask = (np.arange(n) >= half).astype(np.uint8)
    fresh[half * 2:] = 0
    r = pair.page_plan(i32(cached), i32(fresh), i32(table),
                       torch.full((cap,), -9, dtype=torch.int32, device=DEV), count(0), page,
                       48 * half, mask=torch.from_numpy(mask).to(DEV))
    torch.cuda.synchronize()
    want = walk(cached, fresh, mask, table, [], page, 48 * half, cap)
    for k, w in want.items():
        got = r[k].cpu().numpy()
        assert np.array_equal(got, np.asarray(w).reshape(got.shape)), k
    assert want["status"] == [0] and want["free_count"] == [0]
