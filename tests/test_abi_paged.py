"""Host-side refusals of the page plan, the cache store, the attention over a
paged cache and the gradient clipping: malformed arguments return their codes
before anything is enqueued (no GPU)."""
import ctypes

import paper_2608_11368_amd as pair

FAKE = ctypes.c_void_p(1 << 20)
OTHER = ctypes.c_void_p(1 << 21)
ODD = ctypes.c_void_p((1 << 20) + 2)
NULL = None
EINVAL, EDTYPE, ERANGE, EALIGN, EWORKSPACE = -1, -2, -3, -4, -6


def test_page_plan():
    L = pair.lib()
    assert L.pair_page_plan_workspace_bytes(0) == 0
    assert L.pair_page_plan_workspace_bytes(5000) >= 5000 * 12
    need = L.pair_page_plan_workspace_bytes(100)

    def call(n=100, cached=FAKE, fresh=FAKE, page=16, table=FAKE, ldt=64, cap=1000, free=FAKE,
             count=FAKE, room=1000, qo=FAKE, lens=FAKE, slots=FAKE, fo=OTHER, fco=FAKE, ws=FAKE,
             wsb=need):
        return L.pair_page_plan(n, cached, fresh, NULL, page, table, ldt, cap, free, count, room,
                                qo, lens, slots, NULL, fo, fco, ws, wsb, NULL, NULL)

    for name in ("cached", "fresh", "table", "count", "qo", "lens", "fco", "free", "fo", "slots"):
        assert call(**{name: NULL}) == EINVAL, name
    assert call(fo=FAKE) == EINVAL                       # the new list over the old one
    for kw in (dict(n=0), dict(n=1 << 25), dict(page=0), dict(ldt=0), dict(ldt=1 << 30),
               dict(cap=-1), dict(cap=1 << 30), dict(room=-1), dict(room=1 << 31)):
        assert call(**kw) == ERANGE, kw
    assert call(ws=NULL) == EWORKSPACE
    assert call(wsb=need - 1) == EWORKSPACE
    assert call(ws=ctypes.c_void_p((1 << 20) + 16)) == EWORKSPACE


def test_cache_store():
    f = pair.lib().pair_cache_store

    def call(tokens=10, heads=2, dim=64, dt=1, k=FAKE, v=FAKE, ts=128, hs=64, kc=FAKE, vc=FAKE,
             ps=2048, ss=128, ch=64, page=16, pages=10, slots=FAKE):
        return f(tokens, heads, dim, dt, k, v, ts, hs, kc, vc, ps, ss, ch, page, pages, slots, NULL,
                 NULL)

    for name in ("k", "v", "kc", "vc", "slots"):
        assert call(**{name: NULL}) == EINVAL, name
    assert call(dt=0) == EDTYPE and call(dt=3) == EDTYPE
    for kw in (dict(tokens=-1), dict(tokens=1 << 31), dict(heads=0), dict(heads=2000), dict(dim=0),
               dict(dim=12), dict(dim=264), dict(ts=-8), dict(ps=-8), dict(page=0), dict(pages=0),
               dict(pages=1 << 27), dict(hs=1 << 41)):
        assert call(**kw) == ERANGE, kw
    for kw in (dict(k=ODD), dict(v=ODD), dict(kc=ODD), dict(vc=ODD), dict(ts=132), dict(hs=4),
               dict(ps=2052), dict(ss=4), dict(ch=4)):
        assert call(**kw) == EALIGN, kw
    assert call(tokens=0, k=NULL, v=NULL, slots=NULL) == 0    # nothing to do


def test_paged_attention():
    L = pair.lib()
    size = L.pair_paged_attention_workspace_bytes
    ok = (4, 4, 16, 8, 128, 1, 1000)
    need = size(*ok)
    assert need > 0
    for i, bad in ((0, 0), (1, -1), (2, 12), (2, 0), (3, 0), (4, 96), (5, 0), (6, -1)):
        args = list(ok)
        args[i] = bad
        assert size(*args) == 0, (i, bad)
    assert size(4, 4, 65, 1, 128, 1, 1000) == 0          # over 64 query heads a key head

    def call(n=4, tokens=4, hq=16, hkv=8, dim=128, dt=1, q=FAKE, qt=2048, qh=128, kc=FAKE, vc=FAKE,
             ps=16384, ss=1024, ch=128, page=16, pages=100, table=FAKE, ldt=64, off=FAKE, lens=FAKE,
             mq=1, ml=1000, scale=0.1, out=FAKE, ot=2048, oh=128, ws=FAKE, wsb=need):
        return L.pair_paged_attention(n, tokens, hq, hkv, dim, dt, q, qt, qh, kc, vc, ps, ss, ch,
                                      page, pages, table, ldt, off, lens, mq, ml, scale, out, ot,
                                      oh, NULL, ws, wsb, NULL, NULL)

    for name in ("q", "kc", "vc", "table", "off", "lens", "out"):
        assert call(**{name: NULL}) == EINVAL, name
    assert call(dt=0) == EDTYPE
    for kw in (dict(n=0), dict(tokens=-1), dict(hq=12), dict(hkv=0), dict(dim=80), dict(mq=0),
               dict(ml=-1), dict(page=0), dict(pages=0), dict(ldt=0), dict(ldt=1 << 30),
               dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
               dict(scale=float("nan")), dict(qt=-8), dict(oh=1 << 41)):
        assert call(**kw) == ERANGE, kw
    for kw in (dict(q=ODD), dict(out=ODD), dict(kc=ODD), dict(qt=2052), dict(qh=4), dict(ot=2052),
               dict(oh=4), dict(ss=4)):
        assert call(**kw) == EALIGN, kw
    assert call(ws=NULL) == EWORKSPACE and call(wsb=need - 1) == EWORKSPACE
    assert call(tokens=0, q=NULL, out=NULL, wsb=0) == 0       # nothing to do


def test_clip_grads():
    L = pair.lib()
    need = L.pair_clip_grads_workspace_bytes(2)
    assert need > 0 and L.pair_clip_grads_workspace_bytes(-1) == 0

    def call(count=2, g=(1 << 20, 1 << 21), o=None, sizes=(10, 10), types=(0, 1), otypes=None,
             max_norm=1.0, norm=FAKE, coef=FAKE, ws=FAKE, wsb=need):
        arr = lambda t, x: None if x is None else (t * len(x))(*x)  # noqa: E731
        return L.pair_clip_grads(count, arr(ctypes.c_void_p, g), arr(ctypes.c_void_p, o),
                                 arr(ctypes.c_int64, sizes), arr(ctypes.c_int32, types),
                                 arr(ctypes.c_int32, otypes), max_norm, norm, coef, ws, wsb, NULL,
                                 NULL)

    outs = (1 << 22, 1 << 23)
    for kw in (dict(g=None), dict(sizes=None), dict(types=None), dict(norm=NULL), dict(coef=NULL),
               dict(g=(None, 1 << 21)), dict(o=outs), dict(o=(1 << 22, None), otypes=(0, 0))):
        assert call(**kw) == EINVAL, kw
    for kw in (dict(types=(0, 3)), dict(o=outs, otypes=(1, 1)), dict(o=outs, otypes=(0, 2))):
        assert call(**kw) == EDTYPE, kw
    for kw in (dict(count=-1), dict(sizes=(10, -1)), dict(sizes=(1 << 41, 1)), dict(max_norm=0.0),
               dict(max_norm=-1.0), dict(max_norm=float("nan"))):
        assert call(**kw) == ERANGE, kw
    for kw in (dict(g=((1 << 20) + 2, 1 << 21)), dict(g=(1 << 20, (1 << 21) + 1)),
               dict(o=((1 << 22) + 2, 1 << 23), otypes=(0, 1))):
        assert call(**kw) == EALIGN, kw
    assert call(ws=NULL) == EWORKSPACE and call(wsb=need - 1) == EWORKSPACE
