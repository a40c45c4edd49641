"""The update example: its calls in a row against plain torch on the same
weights -- the continued text token by token from full attention without a cache,
the pool's pages, and the clipped gradients."""
import math

import pytest
import torch

from examples import continue_and_update as example
from tests.gpu_util import log

pytestmark = pytest.mark.gpu


def plain_logits(policy, tokens):
    """Full causal attention in float32 over one candidate's tokens."""
    q_heads, kv_heads, dim = policy.heads
    t = tokens.numel()
    qkv = (policy.embed[tokens] @ policy.w_qkv).view(t, q_heads + 2 * kv_heads, dim).float()
    q, k, v = qkv.split([q_heads, kv_heads, kv_heads], dim=1)
    k, v = (x.repeat_interleave(q_heads // kv_heads, dim=1) for x in (k, v))
    out = torch.empty_like(q)
    for h in range(q_heads):
        s = q[:, h] @ k[:, h].t().contiguous() / math.sqrt(dim)
        s.masked_fill_(torch.ones(t, t, device=s.device).triu(1).bool(), -math.inf)
        out[:, h] = torch.softmax(s, 1) @ v[:, h]
    return out.bfloat16().flatten(1) @ policy.w_out


def test_update_example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    prefix, steps = 48, 12
    log("update example: 6 prompts of 5")
    r = example.run(prompts=6, group=5, steps=steps, prefix=prefix, max_norm=0.05)
    torch.cuda.synchronize()
    assert int(r["status"].item()) == 0
    mask, text, policy = r["mask"].bool(), r["text"], r["policy"]
    assert 0 < int(mask.sum()) < mask.numel()
    lens = r["lens"]
    assert bool((lens[mask] == prefix + steps).all()) and bool((lens[~mask] == 0).all())
    per = policy.table.shape[1]
    assert int(r["free_count"]) == int((~mask).sum()) * per
    owned = torch.cat([policy.table[mask].flatten(), policy.free[:int(r["free_count"])]])
    assert torch.equal(owned.sort().values.cpu(), torch.arange(mask.numel() * per).int())
    # Each token was the best one under plain attention, up to what two bf16
    # roundings (of the attention's output and of a logit) can reorder: outputs
    # are below 8 here and a logit sums 512 of them with weights of deviation
    # 4 / sqrt(512), so it is off by a few times 4 * 8 * 2^-8 / sqrt(3), and is
    # itself rounded to 2^-8 of its size (below 64).
    bar = 4 * 4 * 8 * 2.0 ** -8 + 2 * 64 * 2.0 ** -8
    for c in torch.nonzero(mask)[:, 0].tolist():
        logits = plain_logits(policy, text[c, :-1]).float()
        for x in range(prefix, prefix + steps):
            row = logits[x - 1]
            assert float(row.max() - row[text[c, x]]) <= bar, (c, x)
    total = math.sqrt(sum(float(g.double().square().sum()) for g in r["grads"]))
    assert float(r["coef"].item()) < 1.0 and total <= 0.05 * (1 + 1e-6)
    assert total >= 0.05 * (1 - 1e-6)
