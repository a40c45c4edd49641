"""Requests of several rows that are cut, among so many others that a workgroup joins
more than one of their rows: every row of the cut ones against 64 bits, over caches of
16, 8 and 4 bits.  The bar is that of test_gpu_paged_attention.py."""
import numpy as np
import pytest
import torch

import paper_2608_11368_amd as pair
from tests import test_gpu_mx_attention as mx
from tests import test_gpu_paged_attention as wide
from tests.gpu_util import log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pair.lib()
    yield
    torch.cuda.synchronize()


def cache(bits, *args, **kw):
    return wide.Cache(*args, **kw) if bits == 16 else mx.Cache(*args, bits=bits, **kw)


CASES = [
    # requests, new tokens, q heads, key heads, width, page, type: the rows of a request
    # and how many workgroups each request and head has on 256 compute units
    (72, 8, 32, 8, 128, 16, "bf16"),         # 32 rows: 7
    (300, 8, 32, 8, 64, 20, "f16"),          # 32: 1
    (300, 5, 10, 2, 128, 16, "f16"),         # 25: 6
    (300, 7, 6, 2, 64, 16, "bf16"),          # 21: 6
    (1030, 1, 4, 2, 64, 16, "f16"),          # 2: 1
    (1030, 3, 10, 2, 128, 16, "bf16"),       # 15: 1
    (2048, 9, 3, 1, 64, 16, "bf16"),         # 27: 2
]


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_cut_requests_among_many(case, bits):
    n, new, hq, hkv, dim, page, dtype = case
    log(f"attention joins: {bits} bits, {case}")
    lens = np.full(n, new + 3)
    lens[[5, n // 2, n - 1]] = [2300, 6000, 2777]
    news = np.full(n, new)
    news[n // 2 + 1], news[n - 2] = 0, max(1, new - 1)
    c = cache(bits, lens, news, hq, hkv, dim, page, dtype, seed=n)
    r = c.call()
    c.check(r, only=[0, 4, 5, 6, n // 2, n // 2 + 1, n // 2 + 2, n - 2, n - 1])
    again = c.call()
    assert torch.equal(again["out"], r["out"]) and torch.equal(again["lse"], r["lse"])


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("dim,dtype,page", [(128, "bf16", 16), (64, "f16", 20)])
def test_many_cut_requests_beside_a_chunk(dim, dtype, page, bits):
    """300 requests of few rows, a part of them long, and two chunks in one call."""
    log(f"attention joins: {bits} bits, beside chunks, width {dim}, pages of {page}")
    n = 300
    rng = np.random.default_rng(dim)
    news = rng.integers(1, 5, n)
    lens = news + rng.integers(0, 40, n)
    lens[::37] += 2500
    news[[11, 200]] = [70, 130]
    lens[[11, 200]] = [2400, 130]
    news[38], lens[39] = 0, 0
    news[39] = 1
    c = cache(bits, lens, news, 16, 2, dim, page, dtype, seed=dim)
    c.check(c.call(), rows=[0, 1, 2, 3, 69, 127, 129], only=[0, 1, 11, 37, 38, 39, 74, 200, 259, 296, 299])


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_all_requests_long(bits):
    """72 of three tokens after 2100 to 2900 keys: most runs hold ends of two."""
    log(f"attention joins: {bits} bits, 72 long requests")
    lens = np.random.default_rng(3).integers(2100, 2900, 72)
    c = cache(bits, lens, np.full(72, 3), 8, 1, 64, 16, "bf16", seed=3)
    c.check(c.call(), only=[0, 1, 2, 35, 36, 70, 71])
