"""Calls of few workgroups over a cache in 8 and 4 bits around the length from which they
are cut, one and two tiles of rows, alone and beside a chunk."""
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


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("page,dim,dtype", [(16, 128, "bf16"), (20, 64, "f16")])
@pytest.mark.parametrize("most", [1536, 1537, 2048])
@pytest.mark.parametrize("new", [[1], [8, 5], [1, 1, 0, 1], [1, 3, 70, 1]], ids=str)
def test_lengths_around_the_cut(new, most, page, dim, dtype, bits):
    log(f"mx attention: {bits} bits, new {new}, up to {most} keys, width {dim}, pages of {page}")
    lens = np.array([most, 33, 1290, 129][:len(new)])
    lens = np.maximum(lens, new)
    c = Cache(lens, new, 8, 2, dim, page, dtype, seed=most, bits=bits)
    c.check(c.call(), rows=[0, 1, 4, 7, 31, 69])


@pytest.mark.parametrize("n", [16, 17])
@pytest.mark.parametrize("new", [1, 8])
def test_as_many_workgroups_as_are_cut_early(n, new):
    log(f"mx attention: {n} requests of {new}")
    lens = np.full(n, 1200)
    lens[[0, n - 1]] = [1800, 2000]
    c = Cache(lens, np.full(n, new), 8, 2, 128, 16, "bf16", seed=n)
    c.check(c.call(), rows=[0, new - 1], only=[0, 1, n - 2, n - 1])
