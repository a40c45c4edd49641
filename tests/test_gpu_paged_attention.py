"""Attention over a paged cache against a plain softmax in 64 bits, request by
request over the visible keys only.

The bar of an output element is derived, not tuned.  With u the unit roundoff
of the type (2^-8 for bf16, 2^-11 for fp16) and w = sum_j p_j |v_j| / l:
  - the result is rounded once:                       u |out|
  - each weight is rounded once before the product:   u w   (and 2^-24 sum |v_j| / l
    for fp16 weights below its normal range, where the largest weight is taken as 1)
  - scores are fp32 sums of `dim` products, so a weight is off by a relative
    2 * 2^-24 * dim * a with a = scale * max sum |q k|, and the sums over the
    keys by at most 2^-24 * keys; both act on w, and a few roundings more.
"""
import math

import numpy as np
import pytest
import torch

import paper_2608_11368_amd as pair
from tests.gpu_util import DEV, log

pytestmark = pytest.mark.gpu
TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8), "f16": (torch.float16, 2.0 ** -11)}


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pair.lib()
    yield
    torch.cuda.synchronize()


class Cache:
    """Requests over shuffled pages; every slot that no request owns holds NaN."""

    def __init__(self, lens, new, hq, hkv, dim, page, dtype, seed=0, std=1.0, layout="token"):
        self.lens, self.new = np.array(lens), np.array(new)
        self.hq, self.hkv, self.dim, self.page = hq, hkv, dim, page
        self.dtype, self.u = TYPES[dtype]
        rng = np.random.default_rng(seed)
        held = -(-self.lens // page)
        pages = int(held.sum()) + 2
        ids = rng.permutation(pages)
        width = max(1, int(held.max())) + 1
        self.table = np.full((len(lens), width), -7, dtype=np.int32)
        self.table[np.arange(width)[None, :] < held[:, None]] = ids[:int(held.sum())]
        self.off = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int64)
        t = int(self.off[-1])
        fused = torch.from_numpy(rng.normal(0, std, (t, hq + 3, dim)).astype(np.float32))
        self.q = fused.to(self.dtype).to(DEV)[:, 1:1 + hq]
        self.k, self.v = (np.full((pages * page, hkv, dim), np.nan, dtype=np.float32)
                          for _ in range(2))
        for r, n in enumerate(self.lens):
            at = self.slots(r)
            self.k[at] = rng.normal(0, std, (n, hkv, dim))
            self.v[at] = rng.normal(0, 1, (n, hkv, dim))
        self.pages, self.layout, self.scale = pages, layout, 0.9 / math.sqrt(dim)

    def slots(self, r):
        x = np.arange(self.lens[r])
        return self.table[r, x // self.page].astype(np.int64) * self.page + x % self.page

    def tensors(self):
        out = []
        for c in (self.k, self.v):
            x = torch.from_numpy(c).to(self.dtype).to(DEV)
            x = x.view(self.pages, self.page, self.hkv, self.dim)
            if self.layout == "head":       # heads outside the page's slots
                x = x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
            elif self.layout == "padded":
                full = torch.full((self.pages, self.page + 1, self.hkv, self.dim + 8), float("nan"),
                                  dtype=self.dtype, device=DEV)
                full[:, :self.page, :, :self.dim] = x
                x = full[:, :self.page, :, :self.dim]
            out.append(x)
        return out

    def call(self, **kw):
        k, v = self.tensors()
        r = pair.paged_attention(
            self.q, k, v, torch.from_numpy(self.table).to(DEV), torch.from_numpy(self.off).to(DEV),
            torch.from_numpy(self.lens.astype(np.int32)).to(DEV), int(self.new.max()),
            int(self.lens.max()), scale=self.scale, want_lse=True, **kw)
        torch.cuda.synchronize()
        return r

    def check(self, r, rows=None, only=None):
        """Every output against 64 bits (`rows`: tokens to look at per request;
        `only`: the requests to look at, where the call has a bad one)."""
        assert int(r["status"].item()) == 0 or only is not None
        out = r["out"].double().cpu().numpy()
        lse = r["lse"].double().cpu().numpy()
        q = self.q.double().cpu().numpy()
        k, v = (torch.from_numpy(c).to(self.dtype).double().numpy() for c in (self.k, self.v))
        worst, group = 0.0, self.hq // self.hkv
        for r_ in range(len(self.lens)) if only is None else only:
            at = self.slots(r_)
            tokens = range(self.new[r_]) if rows is None else [i for i in rows if i < self.new[r_]]
            for i in tokens:
                t = self.off[r_] + i
                seen = max(0, min(int(self.lens[r_]) - int(self.new[r_]) + i + 1, len(at)))
                if seen == 0:
                    assert np.all(out[t] == 0.0), (r_, i)
                    assert np.all(lse[t] == -np.inf), (r_, i)
                    continue
                kk, vv = k[at[:seen]], v[at[:seen]]
                for h in range(self.hq):
                    kh, vh = kk[:, h // group], vv[:, h // group]
                    s = kh @ q[t, h] * self.scale
                    m = s.max()
                    p = np.exp(s - m)
                    l = p.sum()
                    with np.errstate(invalid="ignore"):
                        want = p @ vh / l
                        w = p @ np.abs(vh) / l
                        small = np.abs(vh).sum(0) / l * 2.0 ** -24 * (self.dtype == torch.float16)
                    a = float((np.abs(kh) @ np.abs(q[t, h])).max()) * self.scale
                    rel = 2.0 ** -24 * (2 * self.dim * a + seen + 64)
                    tol = self.u * np.abs(want) + (1.01 * self.u + rel) * w + small
                    ok = np.isfinite(want)
                    assert np.array_equal(np.isnan(out[t, h]), np.isnan(want)), (r_, i, h)
                    assert np.array_equal(out[t, h][~ok & ~np.isnan(want)],
                                          want[~ok & ~np.isnan(want)]), (r_, i, h)
                    err = np.abs(out[t, h] - want)[ok]
                    assert np.all(err <= tol[ok]), (r_, i, h, float((err / tol[ok]).max()))
                    worst = max(worst, float((err / tol[ok]).max()) if err.size else 0.0)
                    elog = abs(lse[t, h] - (m + math.log(l)))
                    assert elog <= rel + 2.0 ** -22 * abs(m + math.log(l)), (r_, i, h, elog)
        log(f"  largest error {worst:.2f} of the bar")


DECODE = [
    # lens, new, q heads, kv heads, dim, page, type
    ([1], [1], 1, 1, 128, 16, "bf16"),
    ([1, 2, 15, 16, 17, 31, 32, 33], [1] * 8, 2, 1, 64, 16, "f16"),
    ([63, 64, 65, 127, 128, 129, 300], [1] * 7, 8, 2, 128, 32, "bf16"),
    ([700, 3, 1, 511, 513], [1] * 5, 16, 8, 128, 16, "bf16"),
    ([260, 77], [1, 1], 40, 8, 64, 20, "f16"),           # five queries a head, page 20
    ([100, 41], [1, 1], 64, 1, 128, 1, "bf16"),          # one key head, a token a page
    ([1025, 2049, 4100], [1, 1, 1], 4, 4, 128, 64, "f16"),
    ([5000, 9, 3001], [1, 1, 1], 8, 4, 64, 256, "bf16"),
]
CHUNKS = [
    ([5, 40, 8], [5, 3, 8], 8, 2, 128, 16, "bf16"),      # drafted tokens
    ([700, 800], [7, 4], 32, 4, 128, 16, "f16"),
    ([900, 64, 2000], [16, 1, 9], 8, 8, 64, 24, "bf16"),
    ([17], [17], 2, 2, 64, 8, "f16"),
    ([33, 65, 129], [33, 65, 129], 4, 2, 128, 16, "bf16"),
    ([400, 290], [130, 257], 6, 2, 64, 12, "bf16"),      # three queries a head, page 12
    ([515, 1, 260], [200, 1, 64], 16, 2, 128, 32, "f16"),   # a chunk beside a decoding request
    ([1100], [600], 5, 1, 128, 48, "bf16"),
    ([640], [640], 2, 1, 64, 1, "f16"),
]


@pytest.mark.parametrize("case", DECODE + CHUNKS, ids=lambda c: f"{c[0]}-{c[1]}-{c[2:]}")
def test_against_64_bits(case):
    log(f"paged attention: lens {case[0]} new {case[1]} {case[2:]}")
    c = Cache(*case, seed=len(case[0]))
    rows = None if sum(case[1]) <= 64 else [0, 1, 2, 30, 31, 32, 33, 63, 64, 127, 128, 129, 199,
                                            255, 256, 300, 599, 639]
    c.check(c.call(), rows)


@pytest.mark.parametrize("new", [[0, 3, 0, 1, 0], [200, 0, 1, 0, 150]])
def test_requests_without_tokens_or_keys(new):
    """No new token, no key at all, and more tokens than keys: rows that see
    nothing are zero with lse = -inf."""
    log(f"paged attention: empty rows, new {new}")
    c = Cache([0, 2, 50, 0, 100], new, 8, 2, 128, 16, "bf16", seed=2)
    c.check(c.call())


@pytest.mark.parametrize("layout", ["head", "padded"])
@pytest.mark.parametrize("new", [1, 90])
def test_cache_layouts(layout, new):
    log(f"paged attention: cache layout {layout}, {new} new tokens")
    c = Cache([300, 170], [new, new], 4, 2, 64, 16, "bf16", seed=3, layout=layout)
    c.check(c.call(), [0, 1, 45, 89])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("new,hq", [(6, 4), (40, 4), (150, 8)])
def test_what_a_token_does_not_see_has_no_effect(bad, new, hq):
    """Keys and values of later tokens of the chunk are not finite: the tokens
    before them keep their results, the others show what they see."""
    log(f"paged attention: {bad} in keys and values of later tokens, chunk {new}")
    c = Cache([new + 37, new], [new, new], hq, 2, 128, 16, "bf16", seed=4)
    for r in range(2):
        at = c.slots(r)
        c.v[at[-2], 1, 5] = bad          # the last token but one, one element
        c.v[at[-1], 0, :] = bad
    c.check(c.call())
    for r in range(2):                   # a key that is not finite, for the last token only
        at = c.slots(r)
        c.v[at] = np.nan_to_num(c.v[at], nan=1.0, posinf=1.0, neginf=1.0)
        c.k[at[-1]] = np.nan
    k, v = c.tensors()
    r = c.call()
    got = r["out"].double()
    assert bool(torch.isnan(got[c.off[1:] - 1]).all())
    keep = np.ones(int(c.off[-1]), dtype=bool)
    keep[c.off[1:] - 1] = False
    assert bool(torch.isfinite(got[torch.from_numpy(keep).to(DEV)]).all())


@pytest.mark.parametrize("new", [1, 80])
def test_large_scores(new):
    """Scores in the thousands: the running maximum keeps the sums in range."""
    log(f"paged attention: large scores, {new} new tokens")
    c = Cache([400, 90], [new, new], 4, 2, 64, 16, "bf16", seed=5, std=16.0)
    r = c.call()
    assert int(r["status"].item()) == 0
    q, (k, v) = c.q.double().cpu().numpy(), c.tensors()
    kd, vd = (x.reshape(-1, 2, 64).double().cpu().numpy() for x in (k, v))
    out = r["out"].double().cpu().numpy()
    for r_ in range(2):
        at = c.slots(r_)
        for i in (0, new - 1):
            t = c.off[r_] + i
            seen = c.lens[r_] - new + i + 1
            for h in range(4):
                s = kd[at[:seen], h // 2] @ q[t, h] * c.scale
                p = np.exp(s - s.max())
                want = p @ vd[at[:seen], h // 2] / p.sum()
                # a score of size s is off by up to 64 * 2^-24 * sum |q k| in fp32
                a = float((np.abs(kd[at[:seen], h // 2]) @ np.abs(q[t, h])).max()) * c.scale
                tol = 2 * c.u * np.abs(vd[at[:seen], h // 2]).max() + 2 * 64 * 2.0 ** -24 * a * 5
                assert np.abs(out[t, h] - want).max() <= tol


def test_offsets_beyond_32_bits():
    """A cache whose strides put its later pages past 2^32 bytes: the same
    results as the same pages in a dense cache."""
    log("paged attention: page offsets past 2^32")
    pages, page, hkv, dim = 5, 16, 2, 128
    c = Cache([70, 64], [3, 1], 4, hkv, dim, page, "bf16", seed=6)
    want = c.call()
    k, v = c.tensors()
    stride = (1 << 29) + 64                  # elements from page to page: 2^30 bytes and more
    wide = []
    for x in (k, v):
        base = torch.empty((c.pages - 1) * stride + page * hkv * dim, dtype=x.dtype, device=DEV)
        y = base.as_strided(x.shape, (stride, hkv * dim, dim, 1))
        y.copy_(x)
        wide.append(y)
    assert (c.pages - 1) * stride * 2 > 1 << 32
    got = pair.paged_attention(c.q, wide[0], wide[1], torch.from_numpy(c.table).to(DEV),
                               torch.from_numpy(c.off).to(DEV),
                               torch.from_numpy(c.lens.astype(np.int32)).to(DEV), 3, 70,
                               scale=c.scale, want_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])


@pytest.mark.parametrize("new", [[2, 1], [60, 45]])
def test_slots_far_apart(new):
    """Slots 2^27 bytes apart, the pages' rows beside each other: offsets past
    2^32 within a page, for few rows and for tiles."""
    log(f"paged attention: slots 2^27 bytes apart, new {new}")
    hkv, dim, page = 2, 64, 64
    c = Cache([60, 50], new, 4, hkv, dim, page, "bf16", seed=11)
    k, v = c.tensors()
    slot = 1 << 26
    wide = []
    for x in (k, v):
        base = torch.empty((page - 1) * slot + c.pages * hkv * dim, dtype=x.dtype, device=DEV)
        y = base.as_strided(x.shape, (hkv * dim, slot, dim, 1))
        y.copy_(x)
        wide.append(y)
    assert (page - 1) * slot * 2 > 1 << 32
    got = pair.paged_attention(c.q, wide[0], wide[1], torch.from_numpy(c.table).to(DEV),
                               torch.from_numpy(c.off).to(DEV),
                               torch.from_numpy(c.lens.astype(np.int32)).to(DEV), max(new), 60,
                               scale=c.scale, want_lse=True)
    torch.cuda.synchronize()
    c.check(got)


@pytest.mark.parametrize("n,case", [(2100, "few"), (300, "few"), (300, "chunks"), (70, "chunks"),
                                    (2100, "chunks")])
def test_many_requests(n, case):
    """Batches past what a workgroup scans or orders itself; requests of chunks
    beside ones of a token, without tokens and without keys."""
    log(f"paged attention: {n} requests, {case}")
    rng = np.random.default_rng(n)
    new = np.ones(n, dtype=np.int64)
    lens = rng.integers(1, 60, n)
    lens[5], lens[n - 2] = 1400, 1290
    if case == "chunks":
        new = rng.integers(0, 3, n)
        new[[3, n // 2, n - 1]] = [40, 70, 33]
    new[7], lens[9] = 0, 0
    lens = np.maximum(lens, np.where(np.arange(n) == 9, 0, new))
    c = Cache(lens, new, 4, 2, 64, 16, "bf16", seed=n)
    c.check(c.call(), only=[0, 3, 5, 7, 8, 9, 63, 64, 65, n // 2, n - 2, n - 1])


@pytest.mark.parametrize("page", [16, 20])
@pytest.mark.parametrize("dim,dtype", [(64, "bf16"), (128, "f16")])
@pytest.mark.parametrize("new,past,only", [
    ([320] * 6 + [1, 7], 30, [1, 6, 7]),           # many tiles: two launches
    ([1, 90, 0, 8, 1, 9, 1, 1], 400, None),        # few tiles: one, side by side
    ([1] * 40 + [130] + [2] * 20, 1300, [0, 39, 40, 41, 60]),
])
def test_chunks_beside_few(new, past, only, dim, dtype, page):
    log(f"paged attention: new {new[:8]} over {past}, width {dim}, pages of {page}")
    lens = np.array([past + x + 37 * (i % 5) for i, x in enumerate(new)])
    c = Cache(lens, new, 32 if len(new) == 8 else 16, 8 if len(new) == 8 else 4, dim, page, dtype,
              seed=dim + page)
    c.check(c.call(), only=only)


@pytest.mark.parametrize("n,most", [(3, 1024), (3, 1025), (140, 1024), (140, 1025)])
@pytest.mark.parametrize("page", [16, 20])
def test_short_requests_around_the_cut(n, most, page):
    """Lengths at which a call of single tokens changes its split: workgroups of
    eight waves (few requests) or four, whole or in runs, the longest last."""
    log(f"paged attention: {n} requests of at most {most} keys, pages of {page}")
    lens = np.random.default_rng(most).integers(1, 300, n)
    lens[:3], lens[n - 1] = [33, 257, 0], most
    c = Cache(lens, np.ones(n, dtype=np.int64), 4, 2, 128, page, "bf16", seed=n)
    c.check(c.call(), only=[0, 1, 2, n // 2, n - 1])


@pytest.mark.parametrize("new", [[1, 1, 0, 1], [70, 1, 0, 40]])
def test_rows_past_the_last_request(new):
    """More rows of q than the requests have: the others are not touched."""
    log(f"paged attention: rows past the last request, new {new}")
    c = Cache([90, 33, 20, 1100], new, 4, 2, 64, 16, "f16", seed=12)
    t = int(c.off[-1])
    q = torch.randn((t + 9, 4, 64), device=DEV).to(c.dtype)
    q[:t] = c.q
    out = torch.full_like(q, 3.0)
    k, v = c.tensors()
    r = pair.paged_attention(q, k, v, torch.from_numpy(c.table).to(DEV),
                             torch.from_numpy(c.off).to(DEV),
                             torch.from_numpy(c.lens.astype(np.int32)).to(DEV), max(new), 1100,
                             scale=c.scale, want_lse=True, out=out)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == 0 and bool((out[t:] == 3.0).all())
    c.check({**r, "out": out[:t], "lse": r["lse"][:t]})


def test_bounds_are_only_bounds():
    """max_q and max_len larger than the lengths: within the bar, and a call
    repeated gives the same bits."""
    log("paged attention: loose bounds")
    c = Cache([600, 1300, 20], [2, 1, 3], 8, 2, 128, 16, "bf16", seed=7)
    k, v = c.tensors()
    args = (c.q, k, v, torch.from_numpy(c.table).to(DEV), torch.from_numpy(c.off).to(DEV),
            torch.from_numpy(c.lens.astype(np.int32)).to(DEV))
    for max_q, max_len in ((3, 1300), (3, 1312), (8, 100_000), (500, 1300), (2000, 40_000)):
        a = pair.paged_attention(*args, max_q, max_len, scale=c.scale, want_lse=True)
        b = pair.paged_attention(*args, max_q, max_len, scale=c.scale, want_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])
        c.check(a)


def test_status_of_bad_requests():
    """Wrong lengths, pages and offsets set their status bits; the other
    requests of the call keep their results."""
    log("paged attention: bad requests")
    for what in ("len", "page", "offsets", "narrow"):
        for new in ([1, 1, 1], [70, 2, 90]):
            c = Cache([100, 120, 140], new, 4, 2, 64, 16, "bf16", seed=8)
            table, lens, off = c.table.copy(), c.lens.astype(np.int32), c.off.copy()
            if what == "len":
                lens[1] = -5
            elif what == "page":
                table[1, 2] = c.pages + 3
            elif what == "offsets":
                off[3] = off[2] - 1
            else:
                lens[1] = table.shape[1] * 16 + 1
            k, v = c.tensors()
            r = pair.paged_attention(c.q, k, v, torch.from_numpy(table).to(DEV),
                                     torch.from_numpy(off).to(DEV), torch.from_numpy(lens).to(DEV),
                                     int(c.new.max()), 1000, scale=c.scale, want_lse=True)
            torch.cuda.synchronize()
            bit = {"len": pair.ST_LENGTH, "page": pair.ST_PAGES, "offsets": pair.ST_BAD_GROUP,
                   "narrow": pair.ST_LENGTH}[what]
            assert int(r["status"].item()) & bit, what
            c.check(r, only=[0] if what == "offsets" else [0, 2])


def test_on_another_stream_and_in_a_graph():
    """A side stream gives the default stream's bits; a captured call replays
    on new lengths, tables and queries."""
    log("paged attention: side stream and graph")
    for new in ([1, 1, 1], [3, 1, 70]):
        c = Cache([900, 50, 2100], new, 8, 2, 128, 16, "bf16", seed=9)
        want = c.call()
        side = torch.cuda.Stream()
        busy = torch.randn(2048, 2048, device=DEV)
        for _ in range(8):
            busy = busy @ busy / 50
        got = c.call(stream=side)
        side.synchronize()
        assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
        k, v = c.tensors()
        table, off = torch.from_numpy(c.table).to(DEV), torch.from_numpy(c.off).to(DEV)
        lens = torch.from_numpy(c.lens.astype(np.int32)).to(DEV)
        q = c.q.contiguous()
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        args = (int(c.new.max()), 2100)
        ws = torch.empty(pair.pair_paged_attention_workspace_bytes(3, q.shape[0], 8, 2, 128, *args),
                         dtype=torch.uint8, device=DEV)

        def call():
            pair.pair_paged_attention(q, k, v, table, off, lens, *args, c.scale, out, lse, ws, st)

        with torch.cuda.stream(side):
            call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        for step in range(3):
            q.copy_(torch.randn(q.shape, device=DEV))
            lens.copy_(torch.tensor([900 - 7 * step, 50 - step, 2100 - 300 * step], device=DEV))
            ws.fill_(255)
            g.replay()
            torch.cuda.synchronize()
            ref = pair.paged_attention(q, k, v, table, off, lens, *args, scale=c.scale,
                                       want_lse=True)
            torch.cuda.synchronize()
            assert torch.equal(out, ref["out"]) and torch.equal(lse, ref["lse"])
            assert int(st.item()) == 0


def test_refusals():
    c = Cache([40, 9], [1, 1], 4, 2, 64, 16, "bf16", seed=10)
    k, v = c.tensors()
    table, off = torch.from_numpy(c.table).to(DEV), torch.from_numpy(c.off).to(DEV)
    lens = torch.from_numpy(c.lens.astype(np.int32)).to(DEV)
    ok = dict(q=c.q, k_cache=k, v_cache=v, table=table, q_offsets=off, lens=lens, max_q=1,
              max_len=40)
    pair.paged_attention(**ok)
    for error, bad in (
            (TypeError, dict(q=c.q.half())), (TypeError, dict(q=c.q.float())),
            (ValueError, dict(q=c.q.cpu())), (ValueError, dict(q=c.q[..., ::2])),
            (ValueError, dict(v_cache=v[:, :, :, :32])), (ValueError, dict(v_cache=v.half())),
            (ValueError, dict(v_cache=v.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3))),
            (TypeError, dict(table=table.long())), (ValueError, dict(table=table[:1])),
            (TypeError, dict(lens=lens.long())), (ValueError, dict(q_offsets=off[:2])),
            (pair.PairError, dict(scale=-1.0)), (pair.PairError, dict(scale=float("nan"))),
            (pair.PairError, dict(max_q=0)), (pair.PairError, dict(q=c.q[:, :3])),
            (pair.PairError, dict(max_len=-1))):
        with pytest.raises(error):
            pair.paged_attention(**{**ok, **bad})
    torch.cuda.synchronize()
