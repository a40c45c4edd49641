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
