"""Attention over a paged cache in 8 and 4 bits, against a plain softmax in 64 bits
over what the codes stand for; the bar is that of the 16-bit cache's test
(test_gpu_paged_attention.py), for the values are exact in the type of q."""
import numpy as np
import pytest
import torch

import paper_2608_11368_amd as pair
from tests import mx_util as mx
from tests import test_gpu_paged_attention as wide
from tests.gpu_util import DEV, log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pair.lib()
    yield
    torch.cuda.synchronize()


class Cache(wide.Cache):
    """Requests over shuffled pages; what no request owns holds codes and scales that
    stand for NaN and for huge numbers."""

    def __init__(self, *args, bits=8, layout="heads", **kw):
        super().__init__(*args, **kw)
        self.bits, self.layout = bits, layout
        self.codes, self.scales = {}, {}
        rng = np.random.default_rng(7)
        for name, x in (("k", self.k), ("v", self.v)):
            x = x * np.exp(rng.normal(0, 0.5, (*x.shape[:2], 1))).astype(np.float32)
            own = np.isfinite(x).all((1, 2))
            at16 = torch.from_numpy(np.where(own[:, None, None], x, 0)).to(self.dtype)
            code, scale = mx.quantise(at16.double().numpy(), bits, self.dtype)
            code[~own] = rng.choice([(1 << bits) - 1, (1 << (bits - 1)) - 1, 1], code[~own].shape)
            scale[~own] = rng.choice([255, 254, 130], scale[~own].shape)
            self.codes[name], self.scales[name] = code, scale
            self.put(name)

    def put(self, name):
        """The values that codes and scales stand for."""
        v = mx.values(self.codes[name], self.scales[name], self.bits)
        setattr(self, name, v)
        return v

    def tensors(self):
        shape = (self.pages, self.page, self.hkv, -1)
        codes = [mx.to_device(mx.pack(self.codes[n], self.bits).reshape(shape), self.layout,
                              mx.CODES[self.bits]) for n in "kv"]
        return codes + [mx.to_device(self.scales[n].astype(np.uint8).reshape(shape), self.layout,
                                     torch.float8_e8m0fnu) for n in "kv"]

    def arguments(self):
        return (torch.from_numpy(self.table).to(DEV), torch.from_numpy(self.off).to(DEV),
                torch.from_numpy(self.lens.astype(np.int32)).to(DEV))

    def call(self, **kw):
        r = pair.paged_attention_mx(self.q, *self.tensors(), *self.arguments(), int(self.new.max()),
                                    int(self.lens.max()), scale=self.scale, want_lse=True, **kw)
        torch.cuda.synchronize()
        return r


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("case", wide.DECODE + wide.CHUNKS, ids=lambda c: f"{c[0]}-{c[1]}-{c[2:]}")
def test_against_64_bits(case, bits):
    log(f"mx attention: {bits} bits, lens {case[0]} new {case[1]} {case[2:]}")
    c = Cache(*case, seed=len(case[0]), bits=bits)
    rows = None if sum(case[1]) <= 64 else [0, 1, 2, 30, 31, 32, 33, 63, 64, 127, 128, 129, 199,
                                            255, 256, 300, 599, 639]
    c.check(c.call(), rows)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new", [[0, 3, 0, 1, 0], [200, 0, 1, 0, 150]])
def test_requests_without_tokens_or_keys(new, bits):
    log(f"mx attention: empty rows, {bits} bits, new {new}")
    c = Cache([0, 2, 50, 0, 100], new, 8, 2, 128, 16, "bf16", seed=2, bits=bits)
    c.check(c.call())


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("layout", ["slots", "padded"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 20)])
@pytest.mark.parametrize("new", [1, 90])
def test_cache_layouts(layout, new, dim, page, bits):
    log(f"mx attention: {bits} bits, layout {layout}, {new} new tokens, width {dim}")
    c = Cache([300, 170], [new, new], 4, 2, dim, page, "f16", seed=3, layout=layout, bits=bits)
    c.check(c.call(), [0, 1, 45, 89])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new,hq", [(1, 4), (6, 4), (40, 4), (150, 8)])
def test_what_a_token_does_not_see_has_no_effect(new, hq, bits):
    """Blocks of later tokens of the chunk stand for NaN or infinities: the tokens
    before them keep their results, the others show what they see."""
    log(f"mx attention: odd blocks of later tokens, {bits} bits, chunk {new}")
    c = Cache([new + 37, new + 1], [new, new], hq, 2, 128, 16, "f16", seed=4, bits=bits)
    for r in range(2):
        at = c.slots(r)
        c.scales["v"][at[-2], 1, 2] = 255        # the last token but one, one block
        if bits == 8:
            c.codes["v"][at[-1], 0, 5] = 127     # the last token, one element
        c.scales["v"][at[-1], 0, 3] = 200        # beyond fp16's range
        c.codes["v"][at[-1], 0, 96:] |= 1        # infinite there, and none a zero
    v = c.put("v")
    v[np.abs(v) > 65504] *= np.inf
    with np.errstate(invalid="ignore"):
        c.check(c.call())
    c = Cache([new + 37, new], [new, new], hq, 2, 128, 16, "bf16", seed=4, bits=bits)
    clean = c.call()["out"].double()
    for r in range(2):                           # a key that is NaN, for the last token only
        c.scales["k"][c.slots(r)[-1], :, 1] = 255
    got = c.call()["out"].double()
    last = torch.from_numpy(c.off[1:] - 1).to(DEV)
    assert bool(torch.isnan(got[last]).all())
    keep = torch.ones(got.shape[0], dtype=torch.bool, device=DEV)
    keep[last] = False
    assert torch.equal(got[keep], clean[keep])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new", [1, 5, 80])
def test_the_same_as_over_the_values(new, bits):
    """A 16-bit cache of the very values: as far from 64 bits, and near each other."""
    log(f"mx attention: {bits} bits beside 16 bits, {new} new tokens")
    c = Cache([900, 33, 2000], [new, min(new, 33), new], 8, 2, 128, 16, "bf16", seed=5, bits=bits)
    slots = torch.arange(c.pages * c.page, device=DEV)
    cache = c.tensors()
    rows = pair.cache_load_mx(slots, *cache, dtype=c.dtype)
    shape = (c.pages, c.page, c.hkv, c.dim)
    r = pair.paged_attention(c.q, rows["k"].view(shape), rows["v"].view(shape), *c.arguments(), new,
                             2000, scale=c.scale, want_lse=True)
    c.check(r)
    c.check(c.call())


def test_offsets_beyond_32_bits():
    """Codes and scales whose pages lie past 2^32 bytes; slots far apart."""
    log("mx attention: offsets past 2^32")
    for new, page_wide in (([3, 1], True), ([60, 45], True), ([3, 1], False), ([60, 45], False)):
        c = Cache([70, 64], new, 4, 2, 128, 16, "bf16", seed=6)
        want = c.call()
        cache = []
        for x in c.tensors():
            pages, page, heads, w = x.shape
            strides = ((1 << 30) + 16, heads * w, w, 1) if page_wide else (heads * w, (1 << 28) + 16, w, 1)
            n = (pages - 1) * strides[0] + (page - 1) * strides[1] + heads * w
            assert n > 1 << 32 or not page_wide or pages < 5
            y = torch.empty(n, dtype=torch.uint8, device=DEV).as_strided(x.shape, strides)
            y.copy_(x.view(torch.uint8))
            cache.append(y.view(x.dtype))
        got = pair.paged_attention_mx(c.q, *cache, *c.arguments(), max(new), 70, scale=c.scale,
                                      want_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
        c.check(got)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("n,case", [(2100, "few"), (300, "chunks"), (70, "chunks"), (2100, "chunks")])
def test_many_requests(n, case, bits):
    log(f"mx attention: {n} requests, {case}, {bits} bits")
    rng = np.random.default_rng(n)
    new = np.ones(n, dtype=np.int64)
    lens = rng.integers(1, 60, n)
    lens[5], lens[n - 2] = 1400, 1290
    if case == "chunks":
        new = rng.integers(0, 3, n)
        new[[3, n // 2, n - 1]] = [40, 70, 33]
    new[7], lens[9] = 0, 0
    lens = np.maximum(lens, np.where(np.arange(n) == 9, 0, new))
    c = Cache(lens, new, 4, 2, 64, 16, "bf16", seed=n, bits=bits)
    c.check(c.call(), only=[0, 3, 5, 7, 8, 9, 63, 64, 65, n // 2, n - 2, n - 1])


def test_16_million_requests():
    """A token each over one shared page, as many workgroups as a launch can have: all
    the same, and the same as of few."""
    n = (1 << 24) - 1
    log(f"mx attention: {n} requests")
    cache = pair.mx_cache(1, 16, 1, 64, torch.float4_e2m1fn_x2)
    rows = torch.randn((2, 16, 1, 64), device=DEV).bfloat16()
    pair.cache_store_mx(rows[0], rows[1], torch.arange(16, device=DEV), *cache)
    q = torch.randn((1, 1, 64), device=DEV).bfloat16()

    def call(n):
        return pair.paged_attention_mx(q.expand(n, 1, 64), *cache,
                                       torch.zeros((n, 1), dtype=torch.int32, device=DEV),
                                       torch.arange(n + 1, device=DEV),
                                       torch.full((n,), 7, dtype=torch.int32, device=DEV), 1, 7)

    r, few = call(n), call(5)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == 0 and int(few["status"].item()) == 0
    assert bool((r["out"] == few["out"][0]).all()) and bool(few["out"].any())
    with pytest.raises(pair.PairError, match="size out of the supported range"):
        call(n + 1)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("page", [16, 20])
@pytest.mark.parametrize("dim,dtype", [(64, "bf16"), (128, "f16")])
@pytest.mark.parametrize("new,past,only", [
    ([320] * 6 + [1, 7], 30, [1, 6, 7]),           # many tiles: two launches
    ([1, 90, 0, 8, 1, 9, 1, 1], 400, None),        # few tiles: one, side by side
    ([1] * 40 + [130] + [2] * 20, 1300, [0, 39, 40, 41, 60]),
])
def test_chunks_beside_few(new, past, only, dim, dtype, page, bits):
    log(f"mx attention: {bits} bits, new {new[:8]} over {past}, width {dim}, pages of {page}")
    lens = np.array([past + x + 37 * (i % 5) for i, x in enumerate(new)])
    c = Cache(lens, new, 32 if len(new) == 8 else 16, 8 if len(new) == 8 else 4, dim, page, dtype,
              seed=dim + page, bits=bits)
    c.check(c.call(), only=only)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("n,most", [(3, 1025), (3, 2048), (3, 2049), (140, 2048), (140, 2049)])
@pytest.mark.parametrize("page", [16, 20])
def test_short_requests_around_the_cut(n, most, page, bits):
    log(f"mx attention: {bits} bits, {n} requests of at most {most} keys, pages of {page}")
    lens = np.random.default_rng(most).integers(1, 300, n)
    lens[:3], lens[n - 1] = [33, 257, 0], most
    c = Cache(lens, np.ones(n, dtype=np.int64), 4, 2, 128, page, "bf16", seed=n, bits=bits)
    c.check(c.call(), only=[0, 1, 2, n // 2, n - 1])


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("page", [16, 20])
@pytest.mark.parametrize("new,dim", [([5, 3, 4], 128), ([8, 1, 2], 64), ([1, 90, 1, 7], 128),
                                     ([1, 1, 40, 0, 2], 64)])
def test_long_requests_are_cut(new, dim, page, bits):
    """Requests long enough for a call to be cut into runs and joined: one tile of rows
    and two, alone and beside chunks."""
    log(f"mx attention: {bits} bits, new {new} over 2600, width {dim}, pages of {page}")
    lens = [2600 + 300 * i for i in range(len(new))]
    lens[0] = 70
    c = Cache(lens, new, 32, 8, dim, page, "bf16", seed=dim + page, bits=bits)
    c.check(c.call(), [0, 1, 4, 7, 39, 89])


@pytest.mark.parametrize("new", [[1, 1, 0, 1], [70, 1, 0, 40]])
def test_rows_past_the_last_request(new):
    log(f"mx attention: rows past the last request, new {new}")
    c = Cache([90, 33, 20, 1100], new, 4, 2, 64, 16, "f16", seed=12)
    t = int(c.off[-1])
    q = torch.randn((t + 9, 4, 64), device=DEV).to(c.dtype)
    q[:t] = c.q
    out = torch.full_like(q, 3.0)
    r = pair.paged_attention_mx(q, *c.tensors(), *c.arguments(), max(new), 1100, scale=c.scale,
                                want_lse=True, out=out)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == 0 and bool((out[t:] == 3.0).all())
    c.check({**r, "out": out[:t], "lse": r["lse"][:t]})


def test_bounds_are_only_bounds():
    log("mx attention: loose bounds")
    c = Cache([600, 1300, 20], [2, 1, 3], 8, 2, 128, 16, "bf16", seed=7)
    args = (c.q, *c.tensors(), *c.arguments())
    for max_q, max_len in ((3, 1300), (3, 1312), (8, 100_000), (500, 1300), (2000, 40_000)):
        a, b = (pair.paged_attention_mx(*args, max_q, max_len, scale=c.scale, want_lse=True)
                for _ in range(2))
        torch.cuda.synchronize()
        assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])
        c.check(a)


def test_given_results_and_workspaces():
    """Results and workspaces of the caller's, too small ones among them: the same bits."""
    log("mx attention: given results and workspaces")
    c = Cache([1500, 3000], [1, 2], 8, 2, 128, 16, "f16", seed=13, bits=4)
    args = (c.q, *c.tensors(), *c.arguments(), 2, 3000)
    want = pair.paged_attention_mx(*args, want_lse=True)
    need = pair.pair_paged_attention_mx_workspace_bytes(2, 3, 8, 2, 128, pair.PAIR_MXFP4, 2, 3000)
    assert need > 256                    # cut
    for out in (None, torch.full_like(c.q, 7.0)):
        for size in (None, 256, need, need + 4096):
            ws = None if size is None else torch.full((size,), 255, dtype=torch.uint8, device=DEV)
            for lse in (False, True):
                r = pair.paged_attention_mx(*args, want_lse=lse, out=out, workspace=ws)
                torch.cuda.synchronize()
                assert torch.equal(r["out"], want["out"]) and (out is None or r["out"] is out)
                assert (r["lse"] is None) if not lse else torch.equal(r["lse"], want["lse"])


def test_status_of_bad_requests():
    log("mx attention: bad requests")
    for what in ("len", "page", "offsets", "narrow"):
        for new in ([1, 1, 1], [70, 2, 90]):
            c = Cache([100, 120, 140], new, 4, 2, 64, 16, "bf16", seed=8, bits=4)
            table, off, lens = c.arguments()
            if what == "len":
                lens[1] = -5
            elif what == "page":
                table[1, 2] = c.pages + 3
            elif what == "offsets":
                off[3] = off[2] - 1
            else:
                lens[1] = table.shape[1] * 16 + 1
            r = pair.paged_attention_mx(c.q, *c.tensors(), table, off, lens, int(c.new.max()), 1000,
                                        scale=c.scale, want_lse=True)
            torch.cuda.synchronize()
            bit = {"len": pair.ST_LENGTH, "page": pair.ST_PAGES, "offsets": pair.ST_BAD_GROUP,
                   "narrow": pair.ST_LENGTH}[what]
            assert int(r["status"].item()) & bit, what
            c.check(r, only=[0] if what == "offsets" else [0, 2])


@pytest.mark.parametrize("bits", [8, 4])
def test_a_step_on_another_stream_and_in_a_graph(bits):
    """Plan, store, attention and reading back, eager on a side stream and captured:
    each replay gives what eager calls give on the inputs that it finds."""
    log(f"mx attention: a step in a graph, {bits} bits")
    n, page, heads, kv, dim = 3, 16, 8, 2, 128
    for new in (1, 40):
        rows = n * new
        cached = torch.tensor([100, 7, 33], dtype=torch.int32, device=DEV)
        fresh = torch.full((n,), new, dtype=torch.int32, device=DEV)
        table = torch.full((n, 12), -1, dtype=torch.int32, device=DEV)
        held = [7, 1, 3]
        for r in range(n):
            table[r, :held[r]] = torch.arange(held[r], device=DEV) + sum(held[:r])
        first = table.clone()
        free = torch.arange(11, 40, dtype=torch.int32, device=DEV)
        count = torch.tensor([29], device=DEV)
        cache = pair.mx_cache(40, page, kv, dim, mx.CODES[bits])
        old = torch.arange(11 * page, device=DEV)
        past = torch.randn((2, old.numel(), kv, dim), device=DEV).bfloat16()
        pair.cache_store_mx(past[0], past[1], old, *cache)
        qkv = torch.randn((rows, heads + 2 * kv, dim), device=DEV).bfloat16()

        def step(stream=None):
            p = pair.page_plan(cached, fresh, table, free, count, page, rows, stream=stream)
            q, k, v = qkv.split([heads, kv, kv], dim=1)
            s = pair.cache_store_mx(k, v, p["slots"], *cache, stream=stream)
            a = pair.paged_attention_mx(q, *cache, table, p["q_offsets"], p["lens"], new, 200,
                                        want_lse=True, stream=stream)
            b = pair.cache_load_mx(p["slots"], *cache, stream=stream)
            return {"slots": p["slots"], "out": a["out"], "lse": a["lse"], "k": b["k"], "v": b["v"],
                    "s1": p["status"], "s2": s["status"], "s3": a["status"], "s4": b["status"]}

        want = step()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        table.copy_(first)
        torch.cuda.synchronize()
        got = step(side)
        side.synchronize()
        for x in want:
            assert torch.equal(got[x], want[x]), x
        table.copy_(first)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step()
        for i in range(3):
            table.copy_(first)
            qkv.copy_(torch.randn(qkv.shape, device=DEV))
            cached[1] = 7 + i
            for x in ("s1", "s2", "s3", "s4"):
                got[x].fill_(-1)
            graph.replay()
            torch.cuda.synchronize()
            have = {x: y.clone() for x, y in got.items()}
            table.copy_(first)
            want = step()
            torch.cuda.synchronize()
            for x in have:
                assert torch.equal(have[x], want[x]), (new, i, x)
                if x[0] == "s" and len(x) == 2:
                    assert int(have[x].item()) == 0
            busy = torch.randn(512, 512, device=DEV)
            (busy @ busy).sum().item()


def test_gradients_are_refused():
    """A backward pass that comes to the results fails; writes in place count."""
    log("mx attention: no gradient")
    c = Cache([40, 9], [1, 1], 4, 2, 64, 16, "bf16", seed=10)
    cache, args = c.tensors(), (*c.arguments(), 1, 40)
    want = pair.paged_attention_mx(c.q, *cache, *args, want_lse=True)
    q = c.q.detach().requires_grad_()
    r = pair.paged_attention_mx(q, *cache, *args, want_lse=True)
    assert torch.equal(r["out"], want["out"]) and torch.equal(r["lse"], want["lse"])
    for x in (r["out"], r["lse"]):
        with pytest.raises(NotImplementedError, match="no gradient"):
            x.float().sum().backward()
    with torch.no_grad():
        assert not pair.paged_attention_mx(q, *cache, *args)["out"].requires_grad
    out = torch.empty_like(want["out"])
    before = out._version
    r = pair.paged_attention_mx(q, *cache, *args, out=out)
    torch.cuda.synchronize()
    assert r["out"] is out and not out.requires_grad and torch.equal(out, want["out"])
    assert out._version == before + 1


@pytest.mark.parametrize("cache", ["fp8", "fp4"])
def test_update_example(cache):
    """The example's calls in a row over a cache in 8 and 4 bits: its status, its
    pool's pages, and attention over what the cache ends with."""
    log(f"update example: 6 prompts of 5, {cache}")
    from examples import continue_and_update as example

    prefix, steps = 48, 12
    r = example.run(prompts=6, group=5, steps=steps, prefix=prefix, max_norm=0.05, cache=cache)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == 0
    mask, policy = r["mask"].bool(), r["policy"]
    assert 0 < int(mask.sum()) < mask.numel()
    assert bool((r["lens"][mask] == prefix + steps).all()) and bool((r["lens"][~mask] == 0).all())
    per = policy.table.shape[1]
    assert int(r["free_count"]) == int((~mask).sum()) * per
    # the last kept candidate's keys are its tokens' projections, to the formats' half step
    c = int(torch.nonzero(mask)[-1])
    x = torch.arange(prefix + steps, device=DEV)
    slots = policy.table[c][x // policy.page].long() * policy.page + x % policy.page
    got = pair.cache_load_mx(slots, *policy.cache)
    q_heads, kv_heads, dim = policy.heads
    qkv = (policy.embed[r["text"][c]] @ policy.w_qkv).view(-1, q_heads + 2 * kv_heads, dim)
    for name, want in (("k", qkv[:, q_heads:q_heads + kv_heads]), ("v", qkv[:, q_heads + kv_heads:])):
        want = want.double().cpu().numpy()
        code, scale = mx.quantise(want, 8 if cache == "fp8" else 4, torch.bfloat16)
        # the projection of other rows of a batch may be off by a bf16 rounding: a
        # code's step beside it, the largest being a 8th (half) of the largest code
        step = np.repeat(2.0 ** (scale - 127.0), 32, -1) * (32 if cache == "fp8" else 2)
        have = got[name].double().cpu().numpy()
        assert np.all(np.abs(have - want) <= step / 2 + np.abs(want) * 2.0 ** -6), name


def test_tensors_of_another_device(monkeypatch):
    """Kernels run on the current device's stream; caches of another are refused."""
    c = Cache([40, 9], [1, 1], 4, 2, 64, 16, "bf16", seed=10)
    cache, args = c.tensors(), (*c.arguments(), 1, 40)
    slots = torch.arange(3, device=DEV)
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=DEV)
    monkeypatch.setattr(pair, "_device_index", lambda: 1)
    monkeypatch.setattr(pair, "_stream", lambda stream: 0)
    out, ws = torch.empty_like(c.q), torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    for call in (lambda: pair.pair_paged_attention_mx(c.q, *cache, *args, 0.1, out, None, ws),
                 lambda: pair.pair_cache_store_mx(k, k, slots, *cache),
                 lambda: pair.pair_cache_load_mx(slots, *cache, k, k.clone())):
        with pytest.raises(ValueError, match="current device"):
            call()


def test_nothing_to_do():
    """No token, no slot: nothing is launched or written."""
    c = Cache([40, 9], [1, 1], 4, 2, 64, 16, "bf16", seed=10)
    cache = c.tensors()
    before = [x.view(torch.uint8).clone() for x in cache]
    table, off, lens = c.arguments()
    none = torch.zeros(0, dtype=torch.int64, device=DEV)
    r = pair.paged_attention_mx(c.q[:0], *cache, table, torch.zeros_like(off), lens, 0, 40,
                                want_lse=True)
    s = pair.cache_store_mx(c.q[:0, :2], c.q[:0, :2], none, *cache)
    g = pair.cache_load_mx(none, *cache)
    torch.cuda.synchronize()
    assert r["out"].shape == (0, 4, 64) and r["lse"].shape == (0, 4) and g["k"].shape == (0, 2, 64)
    assert int(r["status"].item()) == int(s["status"].item()) == int(g["status"].item()) == 0
    for x, y in zip(cache, before):
        assert torch.equal(x.view(torch.uint8), y)


def test_refusals():
    c = Cache([40, 9], [1, 1], 4, 2, 64, 16, "bf16", seed=10)
    kc, vc, ks, vs = c.tensors()
    table, off, lens = c.arguments()
    ok = dict(q=c.q, k_cache=kc, v_cache=vc, k_scale=ks, v_scale=vs, table=table, q_offsets=off,
              lens=lens, max_q=1, max_len=40)
    pair.paged_attention_mx(**ok)
    for error, bad in (
            (TypeError, dict(q=c.q.float())), (ValueError, dict(q=c.q.cpu())),
            (ValueError, dict(q=c.q[..., ::2])), (TypeError, dict(k_cache=kc.view(torch.uint8))),
            (TypeError, dict(v_scale=vs.view(torch.uint8))), (ValueError, dict(v_scale=vs[:1])),
            (ValueError, dict(v_cache=vc[:, :, :, :32])), (ValueError, dict(v_cache=vc.contiguous())),
            (TypeError, dict(table=table.long())), (ValueError, dict(table=table[:1])),
            (TypeError, dict(lens=lens.long())), (ValueError, dict(q_offsets=off[:2])),
            (TypeError, dict(out=c.q.half())),
            (pair.PairError, dict(scale=-1.0)), (pair.PairError, dict(scale=float("nan"))),
            (pair.PairError, dict(max_q=0)), (pair.PairError, dict(q=c.q[:, :3])),
            (pair.PairError, dict(max_len=-1))):
        with pytest.raises(error):
            pair.paged_attention_mx(**{**ok, **bad})
    torch.cuda.synchronize()
