"""Calls of more workgroups than one launch can have: refused before anything is
enqueued (no GPU)."""
import ctypes

import paper_2608_11368_amd as pair

FAKE = ctypes.c_void_p(1 << 20)
ERANGE = -3


def attention(n, tokens, hq, hkv, mq):
    return pair.lib().pair_paged_attention(
        n, tokens, hq, hkv, 64, 1, FAKE, hq * 64, 64, FAKE, FAKE, 16 * hkv * 64, hkv * 64, 64, 16, 1,
        FAKE, 1, FAKE, FAKE, mq, 16, 0.1, FAKE, hq * 64, 64, None, None, 0, None, None)


def test_paged_attention():
    size = pair.lib().pair_paged_attention_workspace_bytes
    for n, tokens, hq, hkv, mq in (
            (1 << 24, 1 << 24, 1, 1, 1),          # a token each, one workgroup a request and head
            (1 << 21, 1 << 21, 8, 8, 1),
            (1 << 14, 1 << 14, 1024, 1024, 1),
            (1 << 24, 5, 1, 1, 40),               # few tokens, all of them perhaps of few rows
            (1 << 20, 1 << 24, 16, 8, 40),        # both kinds
            (1 << 23, (1 << 31) - 1, 1, 1, 256),  # chunks alone
    ):
        assert size(n, tokens, hq, hkv, 64, mq, 16) == 0, (n, tokens, hq, hkv, mq)
        assert attention(n, tokens, hq, hkv, mq) == ERANGE, (n, tokens, hq, hkv, mq)
    for n, tokens, hq, hkv, mq in (((1 << 24) - 1, 1 << 20, 1, 1, 1), ((1 << 21) - 1, 1 << 21, 8, 8, 1),
                                   (1 << 19, 1 << 24, 16, 8, 40)):
        assert size(n, tokens, hq, hkv, 64, mq, 16) > 0, (n, tokens, hq, hkv, mq)
        assert attention(n, tokens, hq, hkv, mq) == -6        # in range, no workspace


def test_paged_attention_past_the_limit():
    """HIP counts a launch's threads in 32 bits, so a little more than the limit
    is a launch of a few workgroups and no error."""
    size = pair.lib().pair_paged_attention_workspace_bytes
    for n, heads in (((1 << 23) + 77, 2), ((1 << 20) + 5, 16), ((1 << 22) + (1 << 21), 4)):
        assert attention(n, n, heads, heads, 1) == ERANGE
        assert size(n, n, heads, heads, 64, 1, 16) == 0


def test_calls_of_many_prompts():
    """64 threads a prompt: 2^26 prompts are one too many; 256: 2^24."""
    L, ws = pair.lib(), 1 << 62

    def calls(B):
        nv = 2 * B
        yield L.pair_edge_coeffs(B, nv, 2, FAKE, FAKE, FAKE, FAKE, FAKE, None, None, None)
        yield L.pair_design_coeffs(B, nv, 2, FAKE, FAKE, FAKE, 1, 0, None, None, FAKE, None, None,
                                   None, None)
        yield L.pair_design_alloc(B, nv, 2, FAKE, FAKE, FAKE, None, FAKE, 0.1, 0, FAKE, None, None,
                                  None, None)
        yield L.pair_cps_fit(B, nv, 2, FAKE, FAKE, FAKE, FAKE, None, None, None, None)
        yield L.pair_cps_draw(B, nv, 2, FAKE, FAKE, FAKE, 1, 0, 1, FAKE, None, None, None)
        yield L.pair_weighted_grad(B, nv, FAKE, 64, FAKE, 1, 64, FAKE, FAKE, 0, None, None)
        yield L.pair_audit_exact(B, nv, 2, FAKE, 64, FAKE, 1, 64, FAKE, FAKE, None, 0, 0.0, FAKE,
                                 FAKE, None, FAKE, ws, None, None)
        yield L.pair_audit(B, nv, 2, FAKE, 64, FAKE, 1, 64, FAKE, FAKE, None, 1, 0, 1, FAKE, FAKE,
                           None, None, FAKE, ws, None, None)
        yield L.pair_audit_direction(B, nv, 2, FAKE, 64, FAKE, 1, 64, FAKE, FAKE, None, 0, 0.0, 1, 0,
                                     1, FAKE, FAKE, FAKE, ws, None, None)

    for B in (1 << 26, (1 << 26) + 5, (1 << 31) - 1):
        assert list(calls(B)) == [ERANGE] * 9
