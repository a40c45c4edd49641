"""Blocks that stand for NaN or infinities in calls of more than 16 rows a request, and
beside chunks: kernels built for two tiles of rows serve one and two of them."""
import numpy as np
import pytest
import torch

import paper_2608_11368_amd as pair
from tests.gpu_util import log
from tests.test_gpu_mx_attention import Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pair.lib()
    yield
    torch.cuda.synchronize()


CALLS = [
    # new tokens of each request; four query heads to a key head
    [6, 3, 8, 1],                  # 24, 12, 32 and 4 rows
    [6, 90, 3, 1],                 # the same kernel's rows beside a chunk
]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dim,dtype,page", [(128, "f16", 16), (128, "bf16", 20), (64, "bf16", 16),
                                            (64, "f16", 20)])
@pytest.mark.parametrize("new", CALLS, ids=str)
def test_values_that_are_not_finite(new, dim, dtype, page, bits):
    log(f"mx attention: odd blocks, {bits} bits, width {dim}, {dtype}, pages of {page}, new {new}")
    c = Cache([x + 37 for x in new], new, 8, 2, dim, page, dtype, seed=dim + page, bits=bits)
    last = dim // 32 - 1
    for r in range(len(new)):
        at = c.slots(r)
        c.scales["v"][at[-2], 1, 0] = 255            # the last token but one, one block
        if bits == 8:
            c.codes["v"][at[-1], 0, 5] = 127         # the last token, one element
        if dtype == "f16":
            c.scales["v"][at[-1], 0, last] = 200     # beyond fp16's range
            c.codes["v"][at[-1], 0, 32 * last:] |= 1  # infinite there, and none a zero
    v = c.put("v")
    if dtype == "f16":
        v[np.abs(v) > 65504] *= np.inf
    with np.errstate(invalid="ignore"):
        c.check(c.call())


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("new", CALLS, ids=str)
def test_keys_that_are_not_finite(new, bits):
    """A NaN key that only a request's last token sees: the others keep their bits."""
    log(f"mx attention: a NaN key, {bits} bits, new {new}")
    c = Cache([x + 37 for x in new], new, 8, 2, 128, 16, "bf16", seed=4, bits=bits)
    clean = c.call()["out"]
    for r in range(len(new)):
        c.scales["k"][c.slots(r)[-1], :, 1] = 255
    got = c.call()["out"]
    last = torch.from_numpy(c.off[1:] - 1).to(got.device)
    assert bool(torch.isnan(got[last]).all())
    keep = torch.ones(got.shape[0], dtype=torch.bool, device=got.device)
    keep[last] = False
    assert torch.equal(got[keep], clean[keep])
