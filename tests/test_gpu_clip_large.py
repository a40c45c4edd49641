"""Clipping lists as long and as large as a training step's: workgroups whose runs
of chunks cross tensors, partial sums of many launches, and lists that the
memory-side cache does not hold.  Every element is compared, and what lies
between the tensors stays as it was.  The bars are those of test_gpu_clip.py."""
import numpy as np
import pytest
import torch

import paper_2608_11368_amd as pair
from tests.gpu_util import DEV, log
from tests.test_gpu_clip import BF16, F16, F32, check

pytestmark = pytest.mark.gpu
MB = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pair.lib()
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


def sizes_of(count, total, seed):
    """Uneven sizes: over a factor of 1000, some of them 0 or 1."""
    rng = np.random.default_rng(seed)
    w = np.exp(rng.normal(0.0, 1.5, count))
    size = np.maximum(1, (total * w / w.sum()).astype(np.int64))
    size[rng.integers(0, count, max(1, count // 40))] = 0
    size[rng.integers(0, count, max(1, count // 40))] = 1
    return size.tolist()


class Apart:
    """Tensors of one buffer, a few elements apart, so that they start at any
    element; what lies between them holds 3."""

    def __init__(self, sizes, dtype, seed=None):
        gaps = np.random.default_rng(1).integers(1, 9, len(sizes) + 1).tolist()
        self.flat = torch.full((sum(sizes) + sum(gaps),), 3.0, dtype=dtype, device=DEV)
        self.between = torch.ones(self.flat.numel(), dtype=torch.bool, device=DEV)
        self.parts, at = [], 0
        for size, gap in zip(sizes, gaps):
            at += gap
            self.parts.append(self.flat[at:at + size])
            self.between[at:at + size] = False
            at += size
        if seed is not None:
            g = torch.Generator(device=DEV)
            g.manual_seed(seed)
            values = torch.empty(self.flat.numel(), device=DEV).normal_(generator=g).to(dtype)
            self.flat.copy_(torch.where(self.between, self.flat, values))

    def untouched(self):
        return bool((self.flat[self.between] == 3.0).all())


# Elements of 16-bit types; half as many of 32.  A chunk is 16 KB; a launch of the
# norm takes 160 tensors and at most 1024 workgroups, one of the product 120 and 2048.
LISTS = [
    (5, 30 * MB),        # a few tensors over more workgroups' runs than they are
    (119, 40 * MB),      # one launch each, runs of several chunks across tensors
    (301, 60 * MB),
    (900, 60 * MB),      # more than 4096 partial sums: a launch sums them
    (60, 112 * MB),      # past the memory-side cache
    (1000, 120 * MB),    # both
]


@pytest.mark.parametrize("count,total", LISTS)
@pytest.mark.parametrize("grad,out", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32), (F32, F32)],
                         ids=str)
def test_long_and_large_lists(count, total, grad, out):
    log(f"clip: {count} tensors, {total // MB}M 16-bit elements or half as many of 32, {grad} into {out}")
    sizes = sizes_of(count, total // 2 if grad == F32 else total, count)
    grads = Apart(sizes, grad, seed=count)
    outs = Apart(sizes, out)
    for max_norm in (3.0, 1e9):
        r = pair.clip_grads(grads.parts, max_norm, out=outs.parts)
        torch.cuda.synchronize()
        check(grads.parts, r, outs.parts, max_norm)
        assert outs.untouched() and grads.untouched()
    if grad != out:
        return
    r = pair.clip_grads(grads.parts, 3.0, out=outs.parts)
    r2 = pair.clip_grads(grads.parts, 3.0)
    torch.cuda.synchronize()
    assert torch.equal(r["norm"], r2["norm"]) and torch.equal(r["coef"], r2["coef"])
    assert torch.equal(grads.flat, outs.flat)


@pytest.mark.parametrize("count,total", [(119, 12 * MB), (1000, 120 * MB)])
def test_mixed_types_in_one_list(count, total):
    """Types change from tensor to tensor, the results are fp32 or the gradient's."""
    log(f"clip: {count} tensors of three types, {total // MB}M elements")
    sizes = sizes_of(count, total, count + 1)
    types = [(BF16, F32), (F32, F32), (F16, F16), (BF16, BF16), (F16, F32)]
    apart = [(Apart(sizes[i::5], a, seed=i), Apart(sizes[i::5], b)) for i, (a, b) in enumerate(types)]
    grads = [apart[i % 5][0].parts[i // 5] for i in range(count)]
    outs = [apart[i % 5][1].parts[i // 5] for i in range(count)]
    r = pair.clip_grads(grads, 2.0, out=outs)
    torch.cuda.synchronize()
    check(grads, r, outs, 2.0)
    assert all(g.untouched() and o.untouched() for g, o in apart)


def test_a_value_that_is_not_finite_far_in():
    """One NaN in the last elements of a large list: found, and all of it copied."""
    log("clip: a NaN at the end of 250 MB")
    sizes = sizes_of(200, 125 * MB, 5)
    grads, outs = Apart(sizes, BF16, seed=5), Apart(sizes, BF16)
    last = max(i for i, n in enumerate(sizes) if n > 100)
    grads.parts[last][-3] = float("nan")
    r = pair.clip_grads(grads.parts, 1.0, out=outs.parts)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == pair.ST_NONFINITE and float(r["coef"].item()) == 1.0
    assert torch.equal(grads.flat.view(torch.int16), outs.flat.view(torch.int16))
