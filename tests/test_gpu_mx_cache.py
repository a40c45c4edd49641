"""Keys and values into a paged cache in 8 and 4 bits and out of it, against the
plain model: codes, scales and values are the same to the bit."""
import numpy as np
import pytest
import torch

import paper_2608_11368_amd as pair
from tests import mx_util as mx
from tests.gpu_util import DEV, log

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pair.lib()
    yield
    torch.cuda.synchronize()


def empty(rng, pages, page, heads, dim, bits, layout):
    """Host bytes of a cache's four arrays, and the tensors of them."""
    host = [rng.integers(0, 256, (pages, page, heads, w), dtype=np.uint8)
            for w in (dim * bits // 8, dim * bits // 8, dim // 32, dim // 32)]
    types = (mx.CODES[bits],) * 2 + (torch.float8_e8m0fnu,) * 2
    return host, [mx.to_device(h, layout, t) for h, t in zip(host, types)]


def rows(rng, shape, dtype):
    """Rows of every size, zeros, the type's ends and values next to a border."""
    x = rng.normal(0, 1, shape) * np.exp(rng.normal(0, 3, (*shape[:2], 1)))
    x[rng.random(shape) < 0.02] = 0.0
    flat = x.reshape(-1, shape[-1])
    fi = torch.finfo(dtype)
    for i, v in enumerate((0.0, -0.0, fi.max, -fi.max * 0.93, fi.smallest_normal, fi.tiny / 64, 448.0,
                           449.0, 6.0, 7.0, 2.0 ** -99)):
        if i < len(flat):
            flat[i, :32] = v
            flat[i, 3] = -v / 3
    if len(flat) > 12:
        flat[11, :32] = np.arange(32) / 4 - 4             # ties between codes
        flat[12, :32] = 448 - np.arange(32) * 8
    return torch.from_numpy(x).clamp(-fi.max, fi.max).to(dtype)


CASES = [
    # tokens, heads, dim, page, bits, type, layout
    (1, 1, 32, 1, 8, "bf16", "slots"),
    (1, 1, 32, 16, 4, "f16", "heads"),
    (7, 3, 64, 16, 8, "f16", "heads"),
    (33, 2, 96, 20, 4, "bf16", "padded"),
    (64, 8, 128, 16, 8, "bf16", "heads"),
    (301, 8, 128, 64, 4, "f16", "heads"),
    (257, 1, 160, 8, 8, "f16", "slots"),
    (1000, 4, 64, 32, 4, "bf16", "slots"),
    (2049, 2, 256, 24, 8, "bf16", "padded"),
    (129, 5, 224, 128, 4, "f16", "padded"),
    (40, 64, 256, 16, 8, "bf16", "heads"),               # more pieces a token than a workgroup has
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_store_and_load(case):
    tokens, heads, dim, page, bits, dtype, layout = case
    log(f"mx cache: {case}")
    t = TYPES[dtype]
    rng = np.random.default_rng(tokens + dim)
    pages = -(-tokens // page) + 3
    host, cache = empty(rng, pages, page, heads, dim, bits, layout)
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    slots[rng.random(tokens) < 0.1] = -rng.integers(1, 1 << 40)
    fused = torch.zeros((tokens, 3 * heads + 1, dim), dtype=t, device=DEV)
    k, v = fused[:, heads:2 * heads], fused[:, 2 * heads + 1:]
    k.copy_(rows(rng, (tokens, heads, dim), t))
    v.copy_(rows(rng, (tokens, heads, dim), t))
    r = pair.cache_store_mx(k, v, torch.from_numpy(slots).to(DEV), *cache)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == 0 and r["k_cache"] is cache[0]
    real = slots >= 0
    for i, new in ((0, k), (1, v)):
        code, scale = mx.quantise(new.double().cpu().numpy()[real], bits, t)
        host[i].reshape(-1, heads, host[i].shape[3])[slots[real]] = mx.pack(code, bits)
        host[2 + i].reshape(-1, heads, dim // 32)[slots[real]] = scale
    for h, c in zip(host, cache):            # what was not written is as it was
        np.testing.assert_array_equal(mx.to_host(c), h)

    # every row of the batch, some of them again, and none
    back = np.concatenate([slots, slots[:3], [-1]])
    got = pair.cache_load_mx(torch.from_numpy(back).to(DEV), *cache, dtype=t)
    torch.cuda.synchronize()
    assert int(got["status"].item()) == 0
    at = np.maximum(back, 0)
    for i, x in ((0, "k"), (1, "v")):
        code = mx.unpack(host[i].reshape(-1, heads, host[i].shape[3])[at], bits)
        want = mx.values(code, host[2 + i].reshape(-1, heads, dim // 32)[at], bits)
        want[back < 0] = 0.0
        assert got[x].dtype == t and got[x].shape == (len(back), heads, dim)
        np.testing.assert_array_equal(got[x].double().cpu().numpy(), want)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_every_number_of_the_type(bits, dtype):
    """Each 16-bit number as the largest of its block, beside smaller ones."""
    log(f"mx cache: all {dtype} numbers in {bits} bits")
    t = TYPES[dtype]
    bitsof = np.arange(1 << 16).astype(np.uint16).view(np.int16)
    x = torch.from_numpy(bitsof).view(t)
    x = x[torch.isfinite(x)]
    share = torch.rand((x.numel(), 32), generator=torch.Generator().manual_seed(bits)) * 2 - 1
    share[:, 5] = 1.0
    k = (x.double()[:, None] * share.double()).to(t)
    tokens = k.shape[0] // 4
    k = k[:tokens * 4].view(tokens, 4, 32)
    cache = pair.mx_cache(-(-tokens // 64), 64, 4, 32, mx.CODES[bits])
    kd = k.to(DEV)
    slots = torch.arange(tokens, device=DEV)
    r = pair.cache_store_mx(kd, kd, slots, *cache)
    code, scale = mx.quantise(k.double().numpy(), bits, t)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == 0
    for c, s in (cache[::2], cache[1::2]):
        np.testing.assert_array_equal(mx.to_host(c).reshape(-1, 4, 4 * bits)[:tokens],
                                      mx.pack(code, bits))
        np.testing.assert_array_equal(mx.to_host(s).reshape(-1, 4, 1)[:tokens], scale)
    got = pair.cache_load_mx(slots, *cache, dtype=t)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(got["v"].double().cpu().numpy(), mx.values(code, scale, bits))


@pytest.mark.parametrize("bits", [8, 4])
def test_blocks_that_are_not_finite(bits):
    """Their block is NaN, with a status bit; the row's others are as they would be."""
    log(f"mx cache: NaN and infinities, {bits} bits")
    rng = np.random.default_rng(bits)
    k = torch.from_numpy(rng.normal(0, 1, (6, 2, 128))).bfloat16()
    v = k.clone()
    k[0, 0, 40], k[1, 1, 127], k[2, 0, 0], v[5, 1, 64] = np.nan, np.inf, -np.inf, np.nan
    cache = pair.mx_cache(1, 16, 2, 128, mx.CODES[bits])
    slots = torch.tensor([3, 4, 5, 0, 9, 15], device=DEV)
    r = pair.cache_store_mx(k.to(DEV), v.to(DEV), slots, *cache)
    got = pair.cache_load_mx(slots, *cache)
    clean = pair.cache_store_mx(k[3:5].to(DEV), v[3:5].to(DEV), slots[3:5], *cache)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == pair.ST_NONFINITE and int(clean["status"].item()) == 0
    for x, new in (("k", k), ("v", v)):
        want = mx.values(*mx.quantise(new.double().numpy(), bits, torch.bfloat16), bits)
        assert np.isnan(want).sum() == (96 if x == "k" else 32)
        np.testing.assert_array_equal(got[x].double().cpu().numpy(), want)


@pytest.mark.parametrize("bits", [8, 4])
def test_all_codes_under_all_scales(bits):
    """What any bytes of a cache stand for, in both types."""
    log(f"mx cache: every code and scale, {bits} bits")
    rng = np.random.default_rng(1)
    host, cache = empty(rng, 16, 16, 1, 256, bits, "heads")
    codes = np.tile(np.arange(256), (256, 1)) % (1 << bits)
    host[0][:] = mx.pack(codes, bits).reshape(host[0].shape)
    host[2][:] = np.repeat(np.arange(256), 8).reshape(host[2].shape)
    cache[0].view(torch.uint8).copy_(torch.from_numpy(host[0]))
    cache[2].view(torch.uint8).copy_(torch.from_numpy(host[2]))
    slots = torch.arange(256, device=DEV)
    want = mx.values(codes, np.repeat(np.arange(256)[:, None], 8, 1), bits)
    for t in TYPES.values():
        got = pair.cache_load_mx(slots, *cache, dtype=t)["k"]
        torch.cuda.synchronize()
        rounded = torch.from_numpy(want).to(t)
        # below the type's normal numbers a value may be cleared or rounded once
        low = torch.from_numpy(np.abs(want) < torch.finfo(t).smallest_normal)
        same = (got[:, 0].cpu() == rounded) | (got[:, 0].cpu().isnan() & rounded.isnan())
        assert bool((same | (low & (got[:, 0].cpu().abs() <= torch.finfo(t).smallest_normal))).all())
        if t == torch.float16:                          # fp16 keeps its subnormal numbers
            assert bool(same.all())


def test_slots_beyond_the_cache():
    """Skipped when storing, zeros when loading, with a status bit."""
    log("mx cache: slots beyond the cache")
    rng = np.random.default_rng(0)
    host, cache = empty(rng, 2, 16, 2, 64, 8, "heads")
    k = torch.from_numpy(rng.normal(0, 1, (4, 2, 64))).half().to(DEV)
    slots = torch.tensor([5, 32, 1 << 40, 31], device=DEV)
    r = pair.cache_store_mx(k, k, slots, *cache)
    got = pair.cache_load_mx(slots, *cache, dtype=torch.float16)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == pair.ST_PAGES and int(got["status"].item()) == pair.ST_PAGES
    code, scale = mx.quantise(k.double().cpu().numpy(), 8, torch.float16)
    want = mx.values(code, scale, 8)
    want[1:3] = 0.0
    np.testing.assert_array_equal(got["v"].double().cpu().numpy(), want)
    host[0].reshape(32, 2, 64)[[5, 31]] = code[[0, 3]]
    np.testing.assert_array_equal(mx.to_host(cache[0]), host[0])


def test_pages_past_32_bits():
    """Pages and slots whose offsets pass 2^32 bytes."""
    log("mx cache: offsets past 2^32")
    rng = np.random.default_rng(3)
    pages, page, heads, dim = 4, 4, 2, 64
    k = torch.from_numpy(rng.normal(0, 1, (8, heads, dim))).bfloat16().to(DEV)
    slots = torch.tensor([15, 0, 7, 9, 14, 3, 12, -1], device=DEV)
    stride = (1 << 31) + 64
    wide = [torch.zeros((pages - 1) * stride + page * heads * w, dtype=torch.uint8, device=DEV)
            .as_strided((pages, page, heads, w), (stride, heads * w, w, 1)) for w in (dim, dim)]
    small = [torch.zeros((pages, page, heads, 2), dtype=torch.uint8, device=DEV) for _ in range(2)]
    cache = [x.view(torch.float8_e4m3fn) for x in wide] + [x.view(torch.float8_e8m0fnu) for x in small]
    pair.cache_store_mx(k, -k, slots, *cache)
    got = pair.cache_load_mx(slots, *cache)
    torch.cuda.synchronize()
    want = mx.values(*mx.quantise(k.double().cpu().numpy(), 8, torch.bfloat16), 8)
    want[7] = 0.0
    np.testing.assert_array_equal(got["k"].double().cpu().numpy(), want)
    np.testing.assert_array_equal(got["v"].double().cpu().numpy(), -want)


def test_many_tokens():
    """More tokens than a launch has workgroups, nearly all of them skipped."""
    n = (1 << 24) + 77
    log(f"mx cache: {n} tokens")
    row = torch.randn((1, 16, 128), device=DEV).bfloat16()
    cache = pair.mx_cache(2, 16, 16, 128)
    slots = torch.full((n,), -1, dtype=torch.int64, device=DEV)
    slots[5], slots[n // 2], slots[n - 1] = 3, 30, 17
    r = pair.cache_store_mx(row.expand(n, 16, 128), row.expand(n, 16, 128), slots, *cache)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == 0
    got = pair.cache_load_mx(torch.arange(32, device=DEV), *cache)
    want = mx.values(*mx.quantise(row.double().cpu().numpy(), 8, torch.bfloat16), 8)[0]
    v = got["v"].double().cpu().numpy()
    for y in range(32):
        np.testing.assert_array_equal(v[y], want if y in (3, 30, 17) else 0 * want)


@pytest.mark.parametrize("bits", [8, 4])
def test_streams_graphs_and_written_counts(bits):
    """A side stream gives the same bytes; a captured store and load follows its
    inputs on every replay; the writes in place are counted."""
    log(f"mx cache: side stream and graph, {bits} bits")
    tokens, heads, dim = 50, 2, 64
    k = torch.randn((tokens, heads, dim), device=DEV).half()
    slots = torch.randperm(64, device=DEV)[:tokens]
    a, b = (pair.mx_cache(4, 16, heads, dim, mx.CODES[bits]) for _ in range(2))
    before = [c._version for c in a]
    pair.cache_store_mx(k, -k, slots, *a)
    assert [c._version for c in a] == [x + 1 for x in before]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pair.cache_store_mx(k, -k, slots, *b, stream=side)
    got = pair.cache_load_mx(slots, *b, dtype=torch.float16, stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    for x, y in zip(a, b):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert torch.equal(got["k"], -got["v"]) and bool(got["k"].any())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = pair.cache_store_mx(k, -k, slots, *b)
        got = pair.cache_load_mx(slots, *b, dtype=torch.float16)
    for step in range(3):
        k.copy_(torch.randn(k.shape, device=DEV))
        if step == 1:
            k[3, 1, 5] = float("inf")                    # this replay's status, and no other's
        slots.copy_(torch.randperm(64, device=DEV)[:tokens])
        s["status"].fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        have = {x: got[x].clone() for x in ("k", "v")}
        assert int(s["status"].item()) == (pair.ST_NONFINITE if step == 1 else 0)
        assert int(got["status"].item()) == 0
        pair.cache_store_mx(k, -k, slots, *a)
        want = pair.cache_load_mx(slots, *a, dtype=torch.float16)
        torch.cuda.synchronize()
        for x in ("k", "v"):
            assert torch.equal(have[x].view(torch.int16), want[x].view(torch.int16)), step


def test_refusals():
    cache = pair.mx_cache(2, 16, 2, 64)
    four = pair.mx_cache(2, 16, 2, 64, torch.float4_e2m1fn_x2)
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=DEV)
    slots = torch.arange(3, device=DEV)
    kc, vc, ks, vs = cache
    for error, change in (
            (TypeError, dict(k=k.float())), (TypeError, dict(v=k.half())), (ValueError, dict(v=k[:2])),
            (ValueError, dict(k=k[..., :32])), (ValueError, dict(k=k[:, :1])),
            (ValueError, dict(k=k.cpu())), (TypeError, dict(slots=slots.int())),
            (ValueError, dict(slots=slots[:2])), (TypeError, dict(k_cache=kc.view(torch.uint8))),
            (TypeError, dict(v_cache=four[1])), (TypeError, dict(k_scale=ks.view(torch.uint8))),
            (ValueError, dict(v_scale=vs[:1])), (ValueError, dict(v_scale=vs.contiguous())),
            (ValueError, dict(k_scale=four[2][..., :1], v_scale=four[3][..., :1])),
            (ValueError, dict(v_cache=vc.contiguous())), (ValueError, dict(k_cache=kc[0])),
            (ValueError, dict(k_cache=kc.cpu())),
            (pair.PairError, dict(k_cache=kc[:, :1].expand(2, 16, 2, 64),
                                  v_cache=vc[:, :1].expand(2, 16, 2, 64)))):
        args = {**dict(k=k, v=k, slots=slots, k_cache=kc, v_cache=vc, k_scale=ks, v_scale=vs), **change}
        with pytest.raises(error):
            pair.cache_store_mx(**args)
    with pytest.raises(TypeError):
        pair.cache_load_mx(slots, *cache, dtype=torch.float32)
    with pytest.raises(TypeError):
        pair.cache_load_mx(slots.int(), *cache)
    with pytest.raises(pair.PairError):
        pair.pair_cache_load_mx(slots, *cache, k[:1].expand(3, 2, 64), k[1:2].expand(3, 2, 64))
    for bad in (dict(dtype=torch.float8_e5m2), dict(dim=48), dict(dim=288)):
        with pytest.raises((TypeError, ValueError)):
            pair.mx_cache(**{**dict(pages=2, page=16, kv_heads=2, dim=64), **bad})
    torch.cuda.synchronize()
