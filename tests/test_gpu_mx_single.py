"""Caches of one page, one slot a page or one head, and rows of one token or head: a
stride that no element is found by is not looked at."""
import pytest
import torch

import paper_2608_11368_amd as pair
from tests import mx_util as mx
from tests.gpu_util import DEV, log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pair.lib()
    yield
    torch.cuda.synchronize()


def odd(x, step):
    """x with `step` as the stride of each dimension of one element."""
    return x.as_strided(x.shape, [s if n > 1 else step for n, s in zip(x.shape, x.stride())])


def odd_bytes(x, step):
    return odd(x.view(torch.uint8), step).view(x.dtype)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("pages,page,heads,tokens", [(1, 16, 2, 1), (1, 32, 1, 1), (40, 1, 1, 3),
                                                     (3, 16, 1, 1), (1, 1, 1, 1), (1, 20, 1, 7)])
def test_unused_strides(pages, page, heads, tokens, bits):
    log(f"mx cache: {pages} pages of {page}, {heads} heads, {tokens} tokens, {bits} bits")
    dim = 64
    g = torch.Generator(device=DEV)
    g.manual_seed(pages)
    total = pages * page
    k, v = (torch.randn((total, heads, dim), device=DEV, generator=g).bfloat16() for _ in range(2))
    slots = torch.arange(total, device=DEV)
    plain = pair.mx_cache(pages, page, heads, dim, mx.CODES[bits])
    pair.cache_store_mx(k, v, slots, *plain)
    # keys' and values' slices of different tensors
    cache = [odd_bytes(x.clone(), 13 + 4 * i) for i, x in enumerate(plain)]
    for x in cache:
        x.view(torch.uint8).zero_()
    pair.cache_store_mx(k, v, slots, *cache)
    one_k, one_v = odd(k[:1].clone(), 9), odd(v[:1].clone(), 11)
    r = pair.cache_store_mx(one_k, one_v, slots[:1], *cache)
    for x, y in zip(cache, plain):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    got = pair.cache_load_mx(slots, *cache)
    want = pair.cache_load_mx(slots, *plain)
    out_k, out_v = odd(torch.empty_like(one_k), 5), odd(torch.empty_like(one_k), 21)
    pair.pair_cache_load_mx(slots[:1], *cache, out_k, out_v)
    assert torch.equal(got["k"], want["k"]) and torch.equal(got["v"], want["v"])
    assert torch.equal(out_k, want["k"][:1]) and torch.equal(out_v, want["v"][:1])
    q = torch.randn((tokens, 2 * heads, dim), device=DEV, generator=g).bfloat16()
    args = (torch.arange(pages, dtype=torch.int32, device=DEV)[None],
            torch.tensor([0, tokens], device=DEV),
            torch.tensor([max(tokens, total - 1)], dtype=torch.int32, device=DEV), tokens, total)
    a = pair.paged_attention_mx(odd(q, 3), *cache, *args, want_lse=True,
                                out=odd(torch.empty_like(q), 7))
    b = pair.paged_attention_mx(q, *plain, *args, want_lse=True)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == int(a["status"].item()) == 0
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


def test_strides_that_differ_are_refused():
    cache = pair.mx_cache(2, 16, 2, 64)
    kc, vc, ks, vs = cache
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=DEV)
    slots = torch.arange(3, device=DEV)
    apart = torch.zeros((2, 2, 17, 64), dtype=torch.uint8, device=DEV)[:, :, :16].transpose(1, 2)
    wide = torch.zeros((3, 2, 72), dtype=torch.bfloat16, device=DEV)[..., :64]
    one = torch.zeros((2, 16, 2, 1), dtype=torch.uint8, device=DEV).view(ks.dtype).expand(2, 16, 2, 2)
    for change in (dict(v_cache=apart.view(vc.dtype)), dict(v=wide), dict(k=wide),
                   dict(k_scale=one, v_scale=one)):
        with pytest.raises(ValueError, match="strides"):
            pair.cache_store_mx(**{**dict(k=k, v=k, slots=slots, k_cache=kc, v_cache=vc, k_scale=ks,
                                          v_scale=vs), **change})
