"""Host-side refusals of the calls of a paged cache in 8 and 4 bits: malformed
arguments return their codes before anything is enqueued (no GPU)."""
import ctypes

import pytest

import paper_2608_11368_amd as pair

AT = [1 << 20, 1 << 22, 1 << 24, 1 << 26]
FAKE, OTHER = ctypes.c_void_p(1 << 28), ctypes.c_void_p(1 << 29)
ODD = ctypes.c_void_p((1 << 20) + 2)
NULL = None
EINVAL, EDTYPE, ERANGE, EALIGN, EWORKSPACE = -1, -2, -3, -4, -6


class Cache(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("k", "v", "ks", "vs")]
                + [(n, ctypes.c_int64) for n in ("ps", "ss", "hs", "sp", "sl", "sh", "pages")]
                + [(n, ctypes.c_int32) for n in ("page", "heads", "dim", "format")])


def cache(**kw):
    c = dict(k=AT[0], v=AT[1], ks=AT[2], vs=AT[3], ps=16 * 2 * 128, ss=128, hs=16 * 128, sp=16 * 2 * 4,
             sl=4, sh=16 * 4, pages=10, page=16, heads=2, dim=128, format=8)
    c.update(kw)
    return Cache(*(c[n] for n, _ in Cache._fields_))


def store(c, tokens=10, dt=1, k=FAKE, v=FAKE, ts=256, hs=128, slots=FAKE):
    return pair.lib().pair_cache_store_mx(ctypes.addressof(c) if c else None, tokens, dt, k, v, ts, hs,
                                          slots, NULL, NULL)


def load(c, tokens=10, dt=1, k=FAKE, v=OTHER, ts=256, hs=128, slots=FAKE):
    return pair.lib().pair_cache_load_mx(ctypes.addressof(c) if c else None, tokens, slots, dt, k, v,
                                         ts, hs, NULL, NULL)


def attention(c, n=4, tokens=4, hq=16, dt=1, q=FAKE, qt=2048, qh=128, table=FAKE, ldt=64, off=FAKE,
              lens=FAKE, mq=1, ml=1000, scale=0.1, out=OTHER, ot=2048, oh=128, ws=FAKE, wsb=1 << 30):
    return pair.lib().pair_paged_attention_mx(
        ctypes.addressof(c) if c else None, n, tokens, hq, dt, q, qt, qh, table, ldt, off, lens, mq, ml,
        scale, out, ot, oh, NULL, ws, wsb, NULL, NULL)


def test_the_struct_of_the_header():
    """The binding's bytes are the header's struct: no padding, these places."""
    assert ctypes.sizeof(Cache) == 104 and Cache.ps.offset == 32 and Cache.page.offset == 88


@pytest.mark.parametrize("call", [store, load, attention], ids=lambda f: f.__name__)
def test_caches(call):
    assert call(None) == EINVAL
    for name in ("k", "v", "ks", "vs"):
        assert call(cache(**{name: None})) == EINVAL, name
    for f in (0, 1, 2, 16):
        assert call(cache(format=f)) == EDTYPE, f
    for kw in (dict(heads=0), dict(heads=2000), dict(dim=0), dict(dim=48), dict(dim=288), dict(page=0),
               dict(pages=0), dict(pages=1 << 27), dict(ps=-16), dict(sl=-4), dict(sh=1 << 41)):
        assert call(cache(**kw)) == ERANGE, kw
    for kw in (dict(k=AT[0] + 8), dict(v=AT[1] + 4), dict(ks=AT[2] + 2), dict(vs=AT[3] + 1),
               dict(ps=4096 + 8), dict(ss=136), dict(hs=2056), dict(sp=130), dict(sl=6), dict(sh=65)):
        assert call(cache(**kw)) == EALIGN, kw
    for dt in (0, 3):
        assert call(cache(), dt=dt) == EDTYPE


@pytest.mark.parametrize("call", [store, load], ids=lambda f: f.__name__)
def test_rows(call):
    for name in ("k", "v", "slots"):
        assert call(cache(), **{name: NULL}) == EINVAL, name
    for kw in (dict(tokens=-1), dict(tokens=1 << 31), dict(ts=-8), dict(hs=1 << 41)):
        assert call(cache(), **kw) == ERANGE, kw
    for kw in (dict(k=ODD), dict(v=ODD), dict(ts=260), dict(hs=4)):
        assert call(cache(), **kw) == EALIGN, kw
    assert call(cache(), tokens=0, k=NULL, v=NULL, slots=NULL) == 0        # nothing to do


def test_rows_that_share_memory():
    for kw in (dict(ss=0), dict(hs=64), dict(ss=64), dict(ps=2048), dict(sl=0), dict(sp=64), dict(sh=0)):
        assert store(cache(**kw)) == EINVAL, kw
    for a, b in (("k", "v"), ("ks", "vs"), ("k", "ks")):
        assert store(cache(**{a: AT[0], b: AT[0]})) == EINVAL, (a, b)
    # fp4 rows are half as wide
    assert store(cache(format=4, ss=48, hs=16 * 64)) == EINVAL
    for kw in (dict(ts=0), dict(hs=64), dict(ts=128), dict(v=FAKE)):
        assert load(cache(), **kw) == EINVAL, kw


def test_attention():
    size = pair.lib().pair_paged_attention_mx_workspace_bytes
    assert size(4, 4, 16, 2, 128, 8, 1, 1000) > 0
    for i, bad in ((0, 0), (1, -1), (2, 13), (3, 0), (4, 96), (5, 16), (6, 0), (7, -1)):
        args = [4, 4, 16, 2, 128, 4, 1, 1000]
        args[i] = bad
        assert size(*args) == 0, (i, bad)
    for name in ("q", "table", "off", "lens", "out"):
        assert attention(cache(), **{name: NULL}) == EINVAL, name
    for kw in (dict(n=0), dict(tokens=-1), dict(hq=13), dict(hq=256), dict(mq=0), dict(ml=-1),
               dict(ldt=0), dict(ldt=1 << 30), dict(scale=0.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(qt=-8), dict(oh=1 << 41)):
        assert attention(cache(), **kw) == ERANGE, kw
    assert attention(cache(dim=96, ps=8192, hs=2048, sl=4, sh=64, sp=128)) == ERANGE    # 64 or 128 only
    for kw in (dict(q=ODD), dict(out=ODD), dict(qt=2052), dict(qh=4), dict(ot=2052), dict(oh=4)):
        assert attention(cache(), **kw) == EALIGN, kw
    for kw in (dict(oh=64), dict(ot=0)):
        assert attention(cache(), **kw) == EINVAL, kw
    need = size(4, 4, 16, 2, 128, 8, 1, 1000)
    assert attention(cache(), ws=NULL) == EWORKSPACE and attention(cache(), wsb=need - 1) == EWORKSPACE
    assert attention(cache(), tokens=0, q=NULL, out=NULL, wsb=0) == 0      # nothing to do
    for n, tokens, heads, mq in ((1 << 24, 1 << 24, 1, 1), (1 << 14, 1 << 14, 1024, 1)):
        c = cache(heads=heads, hs=2048, ps=2048 * heads, sh=64, sp=64 * heads)
        assert attention(c, n=n, tokens=tokens, hq=heads, qt=heads * 128, ot=heads * 128, mq=mq,
                         ldt=1) == ERANGE
