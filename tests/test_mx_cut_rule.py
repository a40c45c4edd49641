"""Which calls over a cache in 8 and 4 bits are cut, by the workspace that they ask for
(no GPU: the card's 256 compute units are assumed without one)."""
import pytest
import torch

import paper_2608_11368_amd as pair

UNCUT = 256                                    # bytes


@pytest.fixture(autouse=True)
def _no_device():
    if torch.cuda.is_available():
        pytest.skip("runs of another card")


def cut(n, kv, new, group, dim, fmt, most):
    return pair.pair_paged_attention_mx_workspace_bytes(n, n * new, kv * group, kv, dim, fmt, new,
                                                        most) > UNCUT


@pytest.mark.parametrize("fmt,dim", [(8, 128), (8, 64), (4, 128), (4, 64)])
def test_calls_of_few_workgroups(fmt, dim):
    for n, kv in ((1, 1), (4, 8), (32, 1), (2, 2)):
        for new, group in ((8, 4), (17, 1)):             # more than 16 rows
            assert not cut(n, kv, new, group, dim, fmt, 1536)
            assert cut(n, kv, new, group, dim, fmt, 1537)
        for new, group in ((1, 2), (4, 4)):              # at most 16
            first = 1537 if (fmt, dim) == (8, 128) else 2049
            assert not cut(n, kv, new, group, dim, fmt, first - 1)
            assert cut(n, kv, new, group, dim, fmt, first)


@pytest.mark.parametrize("fmt,dim", [(8, 128), (8, 64), (4, 128), (4, 64)])
def test_calls_of_many(fmt, dim):
    for n, kv in ((33, 1), (5, 8), (17, 2), (256, 8)):
        for new, group in ((8, 4), (1, 2)):
            assert not cut(n, kv, new, group, dim, fmt, 2048)
            assert cut(n, kv, new, group, dim, fmt, 2049)
    assert not cut(2049, 1, 1, 1, dim, fmt, 100_000)     # too many to order
