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
