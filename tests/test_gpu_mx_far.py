"""Attention over a cache in 8 and 4 bits whose slots, or their scales, lie more than
2^32 bytes apart within a page: the same bits as over the cache packed."""
import pytest
import torch

import paper_2608_11368_amd as pair
from tests.gpu_util import DEV, log
from tests.test_gpu_mx_attention import Cache

pytestmark = pytest.mark.gpu
APART = (1 << 29) + 16                       # bytes between two slots, of which a page has 16


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pair.lib()
    yield
    torch.cuda.synchronize()


def far(x):
    pages, page, heads, width = x.shape
    n = (pages - 1) * heads * width + (page - 1) * APART + heads * width
    assert (page - 1) * APART > 1 << 32
    y = torch.empty(n, dtype=torch.uint8, device=DEV).as_strided(
        x.shape, (heads * width, APART, width, 1))
    y.copy_(x.view(torch.uint8))
    return y.view(x.dtype)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("which", ["codes", "scales", "all"])
@pytest.mark.parametrize("new", [[3, 1], [60, 45], [1, 70, 2]], ids=str)
def test_slots_past_32_bits(new, which, bits):
    log(f"mx attention: slots past 2^32 bytes, {which}, new {new}, {bits} bits")
    c = Cache([70, 64, 90][:len(new)], new, 4, 2, 128, 16, "bf16", seed=6, bits=bits)
    want = c.call()
    cache = [far(x) if which in ("all", "codes" if i < 2 else "scales") else x
             for i, x in enumerate(c.tensors())]
    got = pair.paged_attention_mx(c.q, *cache, *c.arguments(), max(new), 90, scale=c.scale,
                                  want_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    c.check(got)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("which", ["codes", "scales"])
def test_stores_and_loads_past_32_bits(which, bits):
    log(f"mx cache: slots past 2^32 bytes, {which}, {bits} bits")
    c = Cache([70, 64], [1, 1], 4, 2, 128, 16, "bf16", seed=6, bits=bits)
    plain = c.tensors()
    cache = [far(x) if (which == "codes") == (i < 2) else x for i, x in enumerate(plain)]
    slots = torch.randperm(c.pages * c.page, device=DEV)
    k, v = (torch.randn((slots.numel(), 2, 128), device=DEV).bfloat16() for _ in range(2))
    pair.cache_store_mx(k, v, slots, *cache)
    pair.cache_store_mx(k, v, slots, *plain)
    got, want = pair.cache_load_mx(slots, *cache), pair.cache_load_mx(slots, *plain)
    torch.cuda.synchronize()
    for x, y in zip(cache, plain):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert torch.equal(got["k"], want["k"]) and torch.equal(got["v"], want["v"])
