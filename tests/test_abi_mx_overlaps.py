"""Arrays of a cache in 8 and 4 bits that share bytes with each other or with the rows
that a call moves: refused before anything is enqueued, and arrays that only lie
between each other's rows are not (no GPU)."""
import ctypes
import itertools
import random

import pytest
import torch

import paper_2608_11368_amd as pair
from tests.test_abi_mx import cache

EINVAL = -1
BASE = 1 << 32
FAR = [BASE + (i << 34) for i in range(1, 8)]


@pytest.fixture(autouse=True)
def _no_device():
    if torch.cuda.is_available():
        pytest.skip("made-up addresses: only where a call that passed could not run")


def ptr(x):
    return ctypes.c_void_p(x)


def at(**kw):
    """A cache of far apart arrays but for those that are given."""
    return cache(**{**dict(zip(("k", "v", "ks", "vs"), FAR)), **kw})


def store(c, tokens=10, k=FAR[4], v=FAR[5], ts=256, hs=128):
    return pair.lib().pair_cache_store_mx(ctypes.addressof(c), tokens, 1, ptr(k), ptr(v), ts, hs,
                                          ptr(FAR[6]), None, None)


def load(c, tokens=10, k=FAR[4], v=FAR[5], ts=256, hs=128):
    return pair.lib().pair_cache_load_mx(ctypes.addressof(c), tokens, ptr(FAR[6]), 1, ptr(k), ptr(v),
                                         ts, hs, None, None)


def test_apart():
    assert store(at()) not in (0, EINVAL) and load(at()) not in (0, EINVAL)   # no device


def test_halves_that_are_shifted():
    """10 pages of 16 slots of 2 heads of 128: 4096 bytes of codes a page, 128 of scales."""
    for step in (16, 128, 2048, 4096, 9 * 4096, 10 * 4096 - 128, 10 * 4096 - 16):
        for a, b in ((BASE, BASE + step), (BASE + step, BASE)):
            assert store(at(k=a, v=b)) == EINVAL, step
    for step in (4, 64, 128, 9 * 128, 10 * 128 - 4):
        for a, b in ((BASE, BASE + step), (BASE + step, BASE)):
            assert store(at(ks=a, vs=b)) == EINVAL, step
    assert store(at(k=BASE, v=BASE + 10 * 4096)) != EINVAL
    assert store(at(ks=BASE, vs=BASE + 10 * 128)) != EINVAL


def test_codes_and_scales():
    for ks in (BASE, BASE + 4, BASE + 9 * 4096 + 4000, BASE + 10 * 4096 - 4, BASE - 10 * 128 + 4):
        for name in ("ks", "vs"):
            assert store(at(k=BASE, **{name: ks})) == EINVAL, ks - BASE
    for ks in (BASE + 10 * 4096, BASE - 10 * 128):
        assert store(at(k=BASE, ks=ks)) != EINVAL


def test_arrays_between_each_others_rows():
    """A page's four parts, a head's, and a row's side by side."""
    page, codes, scales = 16, 16 * 2 * 128, 16 * 2 * 4
    whole = 2 * codes + 2 * scales
    at_page = dict(k=BASE, v=BASE + codes, ks=BASE + 2 * codes, vs=BASE + 2 * codes + scales, ps=whole,
                   sp=whole)
    assert store(at(**at_page)) != EINVAL
    for name in ("v", "ks", "vs"):
        assert store(at(**{**at_page, name: at_page[name] - 16})) == EINVAL, name
    assert store(at(**{**at_page, "vs": at_page["vs"] + 4})) == EINVAL       # the next page's keys
    half = page * 128 * 2 + page * 4 * 2                                     # of one head
    at_head = dict(k=BASE, v=BASE + page * 128, ks=BASE + page * 256, vs=BASE + page * 260, ps=2 * half,
                   sp=2 * half, hs=half, sh=half)
    assert store(at(**at_head)) != EINVAL
    for name in ("v", "ks", "vs"):
        assert store(at(**{**at_head, name: at_head[name] - 16})) == EINVAL, name
    row = 128 + 128 + 16                                                     # of one slot and head
    at_row = dict(k=BASE, v=BASE + 128, ks=BASE + 256, vs=BASE + 260, ss=row, sl=row, hs=16 * row,
                  sh=16 * row, ps=32 * row, sp=32 * row)
    assert store(at(**at_row)) != EINVAL
    for name in ("ks", "vs"):
        assert store(at(**{**at_row, name: BASE + 252})) == EINVAL, name
    assert store(at(**{**at_row, "vs": BASE + row})) == EINVAL               # the next row's keys


def test_rows():
    for step in (8, 64, 128, 256, 1024, 9 * 256 + 128, 10 * 256 - 8):        # elements
        for a, b in ((BASE, BASE + 2 * step), (BASE + 2 * step, BASE)):
            assert load(at(), k=a, v=b) == EINVAL, step
    assert load(at(), k=BASE, v=BASE + 2 * 2560) != EINVAL
    # keys and values that are columns of one tensor, and those that share a column
    assert load(at(), k=BASE, v=BASE + 2 * 256, ts=512) != EINVAL
    assert load(at(), k=BASE, v=BASE + 2 * 248, ts=512) == EINVAL
    assert load(at(), k=BASE, v=BASE + 2 * 264, ts=512) == EINVAL
    assert load(at(), k=BASE, v=BASE + 2 * 264, ts=512, tokens=1) != EINVAL
    # heads of keys and values in turn
    assert load(at(), k=BASE, v=BASE + 2 * 128, ts=512, hs=256) != EINVAL
    assert load(at(), k=BASE, v=BASE + 2 * 136, ts=512, hs=256) == EINVAL
    # stored rows may be the same, and any number of times
    assert store(at(), k=BASE, v=BASE) != EINVAL
    assert store(at(), k=BASE, v=BASE + 16, ts=0, hs=0) != EINVAL


@pytest.mark.parametrize("call", [store, load], ids=lambda f: f.__name__)
def test_rows_in_the_cache(call):
    for name, size in (("k", 10 * 4096), ("v", 10 * 4096), ("ks", 10 * 128), ("vs", 10 * 128)):
        c = at(**{name: BASE})
        for row in ("k", "v"):
            for x in (BASE, BASE + size - 16, BASE - 10 * 512 + 16):
                assert call(c, **{row: x}) == EINVAL, (name, row, x - BASE)
            for x in (BASE + size, BASE - 10 * 512):
                assert call(c, **{row: x}) != EINVAL, (name, row, x - BASE)


def test_small_layouts_against_every_byte():
    """Halves in every order of their dimensions, with and without room, at shifts of
    16 bytes: refused exactly where some byte belongs to two rows."""
    rng = random.Random(5)
    seen = {True: 0, False: 0}
    for _ in range(1500):
        pages, page, heads, dim = rng.randint(1, 3), rng.randint(1, 3), rng.randint(1, 3), 32
        count, stride, size = [pages, page, heads], [0, 0, 0], dim
        for i in rng.sample(range(3), 3):
            size += rng.choice([0, 0, 16, 32, 64])
            stride[i] = size
            size *= count[i]
        shift = 16 * rng.randint(-size // 16, size // 16)
        places = [sum(i * s for i, s in zip(x, stride)) for x in itertools.product(*map(range, count))]
        first = {p + b for p in places for b in range(dim)}
        shared = any(p + shift + b in first for p in places for b in range(dim))
        c = at(k=BASE, v=BASE + shift, pages=pages, page=page, heads=heads, dim=dim, ps=stride[0],
               ss=stride[1], hs=stride[2], sp=9, sl=3, sh=1)
        assert (store(c) == EINVAL) == shared, (count, stride, shift)
        seen[shared] += 1
    assert min(seen.values()) > 200


def test_the_largest_strides():
    top = 1 << 40
    c = at(pages=(1 << 31) // 16 - 1, ps=top, ss=128, hs=2048, sp=top, sl=4, sh=64)
    assert store(c, tokens=(1 << 31) - 1, ts=0) != EINVAL      # pages of a TiB, between the others'
    assert store(at(pages=(1 << 31) // 16 - 1, ps=top, sp=top, v=FAR[0] + top * 5 + 128)) == EINVAL
