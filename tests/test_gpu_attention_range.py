"""Attention where one key outweighs a long row of others.  All scores are zero but
the first key's, 18, so each of the others weighs e^-18 = 2^-26 of it; their
values are 1 and the first key's is 0, so with N of them an output is
x / (1 + x), x = N e^-18, and lse = 18 + log(1 + x).

The bar: an output is rounded once (u of it); weights and sums in fp32 are off by a
relative 2^-24 (2 dim * 18 + keys + 64), which lse, a sum's logarithm, is off by itself;
and a weight that small is rounded, in
fp16, to a multiple of 2^-31 of the largest, by 2^-32 at most, N times.  (Without
room below the largest weight they would all vanish, an error of x.)"""
import math

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


@pytest.mark.parametrize("dtype,u,step", [(torch.float16, 2.0 ** -11, 2.0 ** -32),
                                          (torch.bfloat16, 2.0 ** -8, 0.0)])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [64, 24])
@pytest.mark.parametrize("new,others,q_heads,kv_heads", [
    (1, 0, 1, 1),            # cut into runs
    (8, 0, 4, 1),            # two tiles of rows
    (1, 2100, 2, 1),         # so many requests that none is cut
    (40, 0, 1, 1),           # a tile, its keys split
    (1100, 0, 64, 8),        # tiles that fill the card
    (40, 3, 1, 1),           # both kinds in one launch
])
def test_one_key_outweighs_a_long_row(new, others, q_heads, kv_heads, page, dim, dtype, u, step):
    log(f"attention: one large weight, {new} tokens, {others} other requests, {q_heads}/{kv_heads} "
        f"heads of {dim}, pages of {page}, {dtype}")
    keys = 131_072
    pages = -(-keys // page)
    k = torch.zeros((pages + 1, page, kv_heads, dim), dtype=dtype, device=DEV)
    v = torch.ones_like(k)
    k[0, 0, :, 0], v[0, 0] = 36.0, 0.0
    q = torch.zeros((new + others, q_heads, dim), dtype=dtype, device=DEV)
    q[:, :, 0] = 4.0
    table = torch.full((1 + others, pages), -1, dtype=torch.int32, device=DEV)
    table[0] = torch.arange(pages)
    table[1:, 0] = pages                                  # the others see one key, of score 0
    lens = torch.ones(1 + others, dtype=torch.int32, device=DEV)
    lens[0] = keys
    off = torch.arange(2 + others, device=DEV) + (new - 1)
    off[0] = 0
    r = pair.paged_attention(q, k, v, table, off, lens, new, keys, scale=0.125, want_lse=True)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == 0
    out, lse = r["out"].double().cpu(), r["lse"].double().cpu()
    n = keys - new + torch.arange(new, dtype=torch.float64)     # keys beside the first
    x = n * math.exp(-18.0)
    want = x / (1 + x)
    rel = 2.0 ** -24 * (2 * dim * 18 + keys + 64)
    err = (out[:new] - want[:, None, None]).abs().amax((1, 2))
    assert bool((err <= u * want + rel * want + n * step).all()), float((err / want).max())
    top = 18 + torch.log1p(x)
    assert bool(((lse[:new] - top[:, None]).abs().amax(1) <= rel + 2.0 ** -22 * top).all())
    assert bool((out[new:] == 1.0).all()) and bool((lse[new:].abs() <= 2.0 ** -22).all())
