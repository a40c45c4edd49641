"""One update around the estimator, on the GPU: draw which rollouts continue,
continue those over a paged key/value cache, and clip the estimated gradient.

  1. every candidate of every prompt has a prefix in the cache;
  2. the design draw gives the completion mask and the logged rho;
  3. a page plan with that mask gives the kept candidates their next tokens'
     slots and returns the released candidates' pages to the pool;
  4. per token: keys and values into their slots, attention, the next token;
  5. rewards, sequence advantages, and the batch-mean gradient over each
     parameter's score block, clipped to a norm.

The policy is one attention layer with random weights, and rewards and scores are
synthetic: the point is the order of the calls, none of which waits for the GPU.

    python examples/continue_and_update.py [--prompts 16] [--group 8] [--steps 12]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_11368_amd as pair  # noqa: E402


class Policy:
    """One attention layer over a paged cache; tied to `n` candidates."""

    def __init__(self, n, longest, gen, width=512, q_heads=8, kv_heads=2, dim=64, vocab=512,
                 page=16, device="cuda:0"):
        def rand(*shape, scale=1.0):
            return (torch.randn(*shape, generator=gen, device=device) * scale).bfloat16()

        self.heads, self.page, self.longest, self.device = (q_heads, kv_heads, dim), page, longest, device
        self.embed = rand(vocab, width)
        self.w_qkv = rand(width, (q_heads + 2 * kv_heads) * dim, scale=width ** -0.5)
        self.w_out = rand(q_heads * dim, vocab, scale=4 * (q_heads * dim) ** -0.5)
        per = -(-longest // page)
        shape = (n * per, page, kv_heads, dim)
        self.k_cache = torch.zeros(shape, dtype=torch.bfloat16, device=device)
        self.v_cache = torch.zeros_like(self.k_cache)
        self.table = torch.full((n, per), -1, dtype=torch.int32, device=device)
        self.free = torch.arange(n * per, dtype=torch.int32, device=device)
        self.free_count = torch.full((1,), n * per, dtype=torch.int64, device=device)
        self.cached = torch.zeros(n, dtype=torch.int32, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def forward(self, fresh, most, rows, tokens_of, mask=None):
        """`fresh` new tokens (at most `most`) of each kept candidate, `rows` in all
        at most; `tokens_of` gives the packed rows' tokens.  Logits of the rows
        and the plan; rows past the plan's last belong to no candidate."""
        q_heads, kv_heads, dim = self.heads
        plan = pair.page_plan(self.cached, fresh, self.table, self.free, self.free_count, self.page,
                              rows, mask=mask)
        self.free, self.free_count, self.cached = (plan["free_pages"], plan["free_count"],
                                                   plan["lens"])
        qkv = (self.embed[tokens_of(plan)] @ self.w_qkv).view(rows, q_heads + 2 * kv_heads, dim)
        q, k, v = qkv.split([q_heads, kv_heads, kv_heads], dim=1)
        store = pair.cache_store(k, v, plan["slots"], self.k_cache, self.v_cache)
        a = pair.paged_attention(q, self.k_cache, self.v_cache, plan["table"], plan["q_offsets"],
                                 plan["lens"], most, self.longest)
        self.status |= plan["status"] | store["status"] | a["status"]
        return a["out"].flatten(1) @ self.w_out, plan


def run(prompts=16, group=8, steps=12, prefix=48, blocks=(4096, 777, 20_000), max_norm=0.5, seed=0,
        device="cuda:0"):
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    n = prompts * group
    policy = Policy(n, prefix + steps, gen, device=device)
    vocab = policy.embed.shape[0]
    owner = torch.arange(n, device=device)
    one = torch.ones(n, dtype=torch.int32, device=device)
    text = torch.zeros((n, prefix + steps), dtype=torch.int64, device=device)
    text[:, :prefix] = torch.randint(vocab, (n, prefix), generator=gen, device=device)

    # 1. the prefixes, a chunk of each candidate
    logits, plan = policy.forward(one * prefix, prefix, n * prefix,
                                  lambda plan: text[:, :prefix].reshape(-1))
    # 2. which candidates continue
    offsets = torch.arange(0, n + 1, group, device=device)
    p = 0.2 + 0.8 * torch.rand(n, generator=gen, device=device)
    design = pair.design_inclusion(offsets, p, seed, 0, 1, group, nv=n)
    mask = design["mask"][0]
    # 3, 4. the kept ones' tokens, one step at a time
    nxt = logits[plan["q_offsets"][1:] - 1].argmax(1)
    for x in range(prefix, prefix + steps):
        text[:, x] = torch.where(mask != 0, nxt, text[:, x])
        logits, plan = policy.forward(
            one, 1, n,
            lambda plan: nxt[torch.searchsorted(plan["q_offsets"][1:], owner, right=True)
                             .clamp_(max=n - 1)], mask)
        last = (plan["q_offsets"][1:] - 1).clamp_(min=0)
        nxt = torch.where(mask != 0, logits[last].argmax(1), nxt)
    # 5. the estimator's gradient over each parameter's scores, clipped
    rewards = (text[:, prefix:].float().mean(1) / vocab).float()
    fold = pair.edge_coeffs(offsets, rewards, mask, design["pi"], group, nv=n)
    grads = []
    for width in blocks:
        scores = torch.randn(n, -(-width // 4) * 4, generator=gen, device=device)[:, :width]
        grads.append(pair.weighted_grad(offsets, scores, fold["coeff"], nv=n, reduce=True)["out"])
    clipped = pair.clip_grads(grads, max_norm)
    status = policy.status | design["status"] | fold["status"] | clipped["status"]
    return dict(text=text, mask=mask, grads=grads, norm=clipped["norm"], coef=clipped["coef"],
                free_count=policy.free_count, lens=policy.cached, policy=policy, status=status)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--prompts", type=int, default=16)
    ap.add_argument("--group", type=int, default=8)
    ap.add_argument("--steps", type=int, default=12)
    args = ap.parse_args()
    r = run(args.prompts, args.group, args.steps)
    kept = int(r["mask"].sum())
    print(f"{kept} of {r['mask'].numel()} candidates continued for {args.steps} tokens, "
          f"{int(r['free_count'])} pages free; gradient norm {float(r['norm']):.4g}, "
          f"clipped by {float(r['coef']):.4g}; status {int(r['status'])}")


if __name__ == "__main__":
    main()
