"""Arrays that may not overlap: refused before anything is enqueued (no GPU)."""
import ctypes

import pytest
import torch

import paper_2608_11368_amd as pair

OK, EINVAL = 0, -1


@pytest.fixture(autouse=True)
def _no_device():
    if torch.cuda.is_available():
        pytest.skip("made-up addresses: only where a call that passed could not run")


def ptr(x):
    return None if x is None else ctypes.c_void_p(x)


PLAN_IN = dict(cached=400, fresh=400, mask=100, free_pages=4000, free_count=8)
PLAN_OUT = dict(table=100 * 64 * 4, q_offsets=101 * 8, lens=400, slots=8000, positions=4000,
                free_out=4000, free_count_out=8, workspace=0, d_status=4)


def plan(**moved):
    L, n = pair.lib(), 100
    at = {k: (i + 1) << 20 for i, k in enumerate([*PLAN_IN, *PLAN_OUT])}
    at.update(moved)
    p = {k: ptr(x) for k, x in at.items()}
    return L.pair_page_plan(n, p["cached"], p["fresh"], p["mask"], 16, p["table"], 64, 1000,
                            p["free_pages"], p["free_count"], 1000, p["q_offsets"], p["lens"],
                            p["slots"], p["positions"], p["free_out"], p["free_count_out"],
                            p["workspace"], L.pair_page_plan_workspace_bytes(n), p["d_status"],
                            None), at


def test_page_plan():
    rc, at = plan()
    assert rc not in (OK, EINVAL)                        # no device to run it on
    size = {**PLAN_IN, **PLAN_OUT}
    size["workspace"] = pair.lib().pair_page_plan_workspace_bytes(100)
    for out in PLAN_OUT:
        for other in size:
            if other == out:
                continue
            step = 256 if out == "workspace" else 8
            last = at[other] + (size[other] - 1) // step * step      # the last bytes of the other
            before = at[other] - (size[out] - 1) // step * step      # its first ones, from below
            for where in {at[other], last, before}:
                assert plan(**{out: where})[0] == EINVAL, (out, other, where - at[other])
            beside = at[other] + (size[other] + 255) // 256 * 256
            assert plan(**{out: beside})[0] != EINVAL, (out, other)
    assert plan(cached=at["fresh"])[0] != EINVAL         # inputs may
    assert plan(mask=None, positions=None, d_status=None)[0] != EINVAL


BASE = 1 << 20


def store(ps, ss, ch, pages=10, page=16, heads=2):
    return pair.lib().pair_cache_store(
        10, heads, 64, 1, ptr(BASE), ptr(BASE), heads * 64, 64, ptr(BASE), ptr(BASE), ps, ss, ch,
        page, pages, ptr(BASE), None, None)


def attention(ot, oh, tokens=5, heads=4, qt=256, qh=64):
    L = pair.lib()
    need = L.pair_paged_attention_workspace_bytes(2, tokens, heads, 2, 64, 5, 100)
    return L.pair_paged_attention(
        2, tokens, heads, 2, 64, 1, ptr(BASE), qt, qh, ptr(BASE), ptr(BASE), 0, 0, 0, 16, 10,
        ptr(BASE), 7, ptr(BASE), ptr(BASE), 5, 100, 0.1, ptr(BASE), ot, oh, None, ptr(BASE), need,
        None, None)


def test_slots_that_share_elements():
    for fine in ((2048, 128, 64), (2048, 64, 1024), (64, 1280, 640), (4096, 136, 64), (128, 1 << 40, 64)):
        assert store(*fine) != EINVAL, fine
    for bad in ((0, 128, 64), (2048, 0, 64), (2048, 128, 0), (1920, 128, 64), (2048, 64, 64),
                (2048, 128, 56), (2048, 64, 960), (64, 1280, 632)):
        assert store(*bad) == EINVAL, bad
    # of one page, slot or head the stride does not count
    assert store(0, 128, 64, pages=1) != EINVAL
    assert store(128, 0, 64, page=1) != EINVAL
    assert store(1024, 64, 0, heads=1) != EINVAL


def test_results_that_share_elements():
    for fine in ((256, 64), (64, 320), (264, 64), (1 << 40, 64)):
        assert attention(*fine) != EINVAL, fine
    for bad in ((0, 64), (256, 0), (192, 64), (64, 256), (256, 56)):
        assert attention(*bad) == EINVAL, bad
    assert attention(0, 64, tokens=1) != EINVAL and attention(256, 64, qt=0, qh=0) != EINVAL
