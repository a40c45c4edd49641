"""The longest calls: as many workgroups as one launch can have."""
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
    torch.cuda.empty_cache()


def test_attention_of_16_million_requests():
    """A token each over one shared page: all the same, and the same as of few."""
    n = (1 << 24) - 1
    log(f"paged attention: {n} requests")
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    k, v = (torch.randn((1, 16, 1, 64), generator=g, device=DEV).bfloat16() for _ in range(2))
    q = torch.randn((1, 1, 64), generator=g, device=DEV).bfloat16()

    def call(n):
        return pair.paged_attention(q.expand(n, 1, 64), k, v,
                                    torch.zeros((n, 1), dtype=torch.int32, device=DEV),
                                    torch.arange(n + 1, device=DEV),
                                    torch.full((n,), 7, dtype=torch.int32, device=DEV), 1, 7)

    r, few = call(n), call(5)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == 0 and int(few["status"].item()) == 0
    assert bool((r["out"] == few["out"][0]).all())
    with pytest.raises(pair.PairError, match="size out of the supported range"):
        call(n + 1)


def test_store_of_16_million_wide_tokens():
    """Rows of 16 KB, more of them than a launch has workgroups; nearly all are
    skipped."""
    n = (1 << 24) + 77
    log(f"cache store: {n} tokens of 32 heads of 128")
    row = torch.randn((1, 32, 128), device=DEV).bfloat16()
    caches = [torch.zeros((2, 16, 32, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    slots = torch.full((n,), -1, dtype=torch.int64, device=DEV)
    slots[5], slots[n // 2], slots[n - 1] = 3, 30, 17
    r = pair.cache_store(row.expand(n, 32, 128), row.expand(n, 32, 128), slots, *caches)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == 0
    for c in caches:
        flat = c.view(32, 32, 128)
        assert bool((flat[[3, 30, 17]] == row).all())
        assert int((flat != 0).any(2).any(1).sum()) == 3
