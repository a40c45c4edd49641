"""The work whose speed is measured for the operators around the estimator: the
ones that continue the drawn rollouts over a paged key/value cache, and the one
that clips the gradients that a step ends with.

A case is a dict of plain values.  Its "kind" names the operator:

  clip    the 2-norm over a list of gradient tensors, and the clipped copies
  plan    block tables, slot maps and the page pool from request lengths and
          the completion mask
  store   new keys and values into the pages of the cache, by slot
  attn    attention of each request's new tokens over its pages of the cache

Sizes and lengths follow from the case alone (every seed of a case has the same
work); the seed decides their order and the values.
"""
import math
import statistics

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # The gradients of a small adapter: two dozen fp32 matrices of a few
        # thousand elements.  Launches and host calls count.
        dict(name="clip_adapter", kind="clip", count=24, numel=100_000, round=1, grad="f32",
             vectors=False, out="f32", clips=True),
        # A model of many small and odd parameters, bf16 matrices and fp32
        # vectors, into the optimiser's flat fp32 gradient.
        dict(name="clip_mixed", kind="clip", count=301, numel=40_000_000, round=1, grad="bf16",
             vectors=True, out="f32", clips=True),
        # Twelve layers of width 2048 in bf16: a step's whole gradient, more
        # than any cache holds.
        dict(name="clip_layers", kind="clip", count=132, numel=600_000_000, round=1024,
             grad="bf16", vectors=False, out="f32", clips=True),
        # One decoding step of 64 requests: a token each, a page now and then.
        dict(name="plan_decode", kind="plan", n=64, page=16, fresh=1, cached=2000, masked=False),
        # The continuation of a whole drawn population: prompts of 2..64
        # candidates, about half of them released, the others get a chunk of
        # up to 128 tokens each.
        dict(name="plan_population", kind="plan", n=16_896, page=16, fresh=128, cached=256,
             masked=True),
        # The keys and values of one decoding step.
        dict(name="store_decode", kind="store", tokens=64, pad=0, q_heads=16, kv_heads=8, dim=128,
             page=16, dtype="bf16"),
        # Those of a packed chunk of prompts with a padded tail.
        dict(name="store_prompts", kind="store", tokens=32_768, pad=301, q_heads=32, kv_heads=8,
             dim=128, page=64, dtype="f16"),
        # A token for each of four short requests: latency.
        dict(name="attn_few", kind="attn", n=4, ctx=400, spread=0.2, new_lo=1, new_hi=1, q_heads=16,
             kv_heads=8, dim=128, page=16, dtype="bf16"),
        # A decoding step of 256 rollouts of uneven length, 4000 tokens on
        # average: the cache is read once.
        dict(name="attn_decode", kind="attn", n=256, ctx=4000, spread=0.5, new_lo=1, new_hi=1,
             q_heads=16, kv_heads=8, dim=128, page=16, dtype="bf16"),
        # Five drafted tokens of two very long rollouts: few rows, a long axis.
        dict(name="attn_drafts_long", kind="attn", n=2, ctx=131_000, spread=0.05, new_lo=5,
             new_hi=5, q_heads=32, kv_heads=8, dim=128, page=64, dtype="f16"),
        # A chunk of about 2000 new tokens of three requests with a long past.
        dict(name="attn_chunk", kind="attn", n=3, ctx=6000, spread=0.4, new_lo=1501, new_hi=2048,
             q_heads=32, kv_heads=8, dim=128, page=16, dtype="bf16"),
        # Whole prompts of uneven length, nothing cached before them.
        dict(name="attn_prompts", kind="attn", n=8, ctx=0, spread=0.0, new_lo=301, new_hi=4096,
             q_heads=16, kv_heads=4, dim=64, page=32, dtype="f16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["clip", "plan", "store", "attn", "attn", "attn"])
    if kind == "clip":
        numel = _log_int(rng, 50_000, 500_000_000)
        grad = rng.choice(["f32", "bf16", "bf16", "f16"])
        if grad == "f32":
            numel = max(50_000, numel // 2)
        vectors = grad != "f32" and rng.random() < 0.5
        return dict(kind=kind, count=_log_int(rng, 1, 400), numel=numel,
                    round=rng.choice([1, 8, 1024]), grad=grad, vectors=vectors,
                    out="f32" if vectors else rng.choice(["f32", grad]),
                    clips=rng.random() < 0.75)
    if kind == "plan":
        n = _log_int(rng, 1, 16_000)
        fresh = rng.choice([1, rng.randint(2, 8), _log_int(rng, 16, 2048)])
        return dict(kind=kind, n=n, page=rng.choice([8, 16, 20, 32, 64, 128]),
                    fresh=max(1, min(fresh, 1_000_000 // n)),
                    cached=max(1, min(_log_int(rng, 16, 16_000), 32_000_000 // n)),
                    masked=rng.random() < 0.5)
    heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 4, 5, 8])
    dim = rng.choice([64, 128, 128])
    page = rng.choice([8, 16, 16, 20, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    layout = dict(q_heads=heads * group, kv_heads=heads, dim=dim, page=page, dtype=dtype)
    if kind == "store":
        tokens = _log_int(rng, 1, 30_000)
        return dict(kind=kind, tokens=tokens, pad=rng.choice([0, rng.randint(0, tokens // 4)]),
                    **layout)
    form = rng.choice(["decode", "decode", "drafts", "chunk", "prompts"])
    if form in ("decode", "drafts"):
        new = 1 if form == "decode" else rng.randint(2, 8)
        n = _log_int(rng, 1, 256)
        ctx = _log_int(rng, 100, max(101, min(130_000, 900_000 // n)))
        return dict(kind=kind, n=n, ctx=ctx, spread=rng.choice([0.1, 0.5]), new_lo=1 if new > 1
                    and rng.random() < 0.5 else new, new_hi=new, **layout)
    new = _log_int(rng, 32, 2048 if form == "chunk" else 4096)
    ctx = _log_int(rng, 64, 8000) if form == "chunk" else 0
    n = rng.randint(1, 8)
    # what the plain form holds: a padded score for every head, token and key
    while n > 1 and n * layout["q_heads"] * new * (2 * ctx + new) > 2_000_000_000:
        n -= 1
    while layout["q_heads"] * new * (2 * ctx + new) > 2_000_000_000:
        new //= 2
    return dict(kind=kind, n=n, ctx=ctx, spread=0.3 if ctx else 0.0,
                new_lo=max(1, new // rng.choice([1, 2, 8])), new_hi=new, **layout)


# ------------------------------------------------------------------ inputs --
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2 + 1)
    return g


def _up(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _sizes(case):
    """Elements of each gradient tensor: spread over about a factor of 100,
    every eighth one a short vector where the case has them."""
    rng = np.random.default_rng([case["count"], case["numel"]])
    w = np.exp(rng.normal(0.0, 1.2, case["count"]))
    size = np.maximum(1, (case["numel"] * w / w.sum()).astype(np.int64))
    size = (size + case["round"] - 1) // case["round"] * case["round"]
    if case["vectors"]:
        size[::8] = np.minimum(size[::8], 2048 + np.arange(len(size[::8])))
    return size


def _quantiles(n, mean, spread):
    """n lengths whose logarithms are spread normally, with the given mean."""
    if mean == 0:
        return np.zeros(n, dtype=np.int64)
    z = [statistics.NormalDist().inv_cdf((i + 0.5) / n) for i in range(n)]
    return np.maximum(1, (mean * np.exp(spread * np.array(z) - spread * spread / 2)).astype(np.int64))


def _plan_lengths(case):
    """Cached and new tokens of each request: a spread of cached lengths with
    a few empty ones, and where chunks are longer than a token every length
    from 0 (a finished rollout) to `fresh`."""
    n = case["n"]
    cached = _quantiles(n, case["cached"], 0.5)
    cached[::17] = 0
    fresh = np.full(n, 1, dtype=np.int64) if case["fresh"] == 1 else np.arange(n) * 7919 % (case["fresh"] + 1)
    live = np.arange(n) * 5 % 11 < 6 if case["masked"] else np.ones(n, dtype=bool)
    return cached, fresh, live


def _attn_lengths(case):
    n = case["n"]
    new = case["new_lo"] + (np.arange(n) * 7919 % n) * (case["new_hi"] - case["new_lo"]) // max(1, n - 1)
    return _quantiles(n, case["ctx"], case["spread"]) + new, new


def _pages(length, page):
    return (length + page - 1) // page


def prepare(case, seed):
    rng = np.random.default_rng([int(seed), 11])
    s = dict(case=case, kind=case["kind"])
    if case["kind"] == "clip":
        size = rng.permutation(_sizes(case))
        g, dtype = _gen(seed), TYPES[case["grad"]]
        total = int(size.sum())
        scale = (3.0 if case["clips"] else 0.3) / math.sqrt(total)
        s["grads"] = []
        for i, k in enumerate(size.tolist()):
            t = torch.empty(k, device=DEV).normal_(generator=g).mul_(scale * (1 + i % 3) / 2)
            s["grads"].append(t if case["vectors"] and k <= 4096 else t.to(dtype))
        # the optimiser's gradient buffer, one flat array, and its views
        s["flat"] = torch.zeros(total, dtype=TYPES[case["out"]], device=DEV)
        s["views"] = list(torch.split(s["flat"], size.tolist()))
        s["max_norm"] = 1.0
        return s
    if case["kind"] == "plan":
        n, page = case["n"], case["page"]
        cached, fresh, live = _plan_lengths(case)
        order = rng.permutation(n)
        cached, fresh, live = cached[order], fresh[order], rng.permutation(live)
        held = _pages(cached, page)
        need = _pages(cached + fresh, page) - held
        pool = int(held.sum() + need.sum()) + 64
        ids = rng.permutation(pool).astype(np.int32)
        # one column more than any request needs
        width = int((held + need).max()) + 1
        table = np.full((n, width), -1, dtype=np.int32)
        at = np.arange(width)[None, :] < held[:, None]
        table[at] = ids[:int(held.sum())]
        free = np.full(pool, -1, dtype=np.int32)
        left = pool - int(held.sum())
        free[:left] = ids[pool - left:]
        s.update(page=page, cached=_up(cached.astype(np.int32)), fresh=_up(fresh.astype(np.int32)),
                 mask=_up(live.astype(np.uint8)) if case["masked"] else None, table=_up(table),
                 free=_up(free), free_count=_up(np.array([left], dtype=np.int64)),
                 max_tokens=int(fresh.sum()))
        return s
    dim, hq, hkv, page = case["dim"], case["q_heads"], case["kv_heads"], case["page"]
    dtype, g = TYPES[case["dtype"]], _gen(seed)
    if case["kind"] == "store":
        tokens = case["tokens"]
        pages = _pages(tokens, page) + 9
        # a batch's tokens land in page-sized runs; the last page is never handed out
        ids = rng.permutation(pages - 1)[:_pages(tokens, page)]
        slots = (ids[:, None] * page + np.arange(page)[None, :]).reshape(-1)[:tokens].astype(np.int64)
        if case["pad"]:
            slots[tokens - case["pad"]:] = -1
        s["slots"] = _up(slots)
        total = tokens
    else:
        length, new = _attn_lengths(case)
        order = rng.permutation(case["n"])
        length, new = length[order], new[order]
        held = _pages(length, page)
        pages = int(held.sum()) + 3
        width = int(held.max()) + 2
        table = np.full((case["n"], width), -1, dtype=np.int32)
        table[np.arange(width)[None, :] < held[:, None]] = rng.permutation(pages)[:int(held.sum())]
        off = np.zeros(case["n"] + 1, dtype=np.int64)
        off[1:] = np.cumsum(new)
        total = int(off[-1])
        s.update(table=_up(table), q_offsets=_up(off), lens=_up(length.astype(np.int32)),
                 max_q=int(new.max()), max_len=int(length.max()), scale=1.0 / math.sqrt(dim))
    # queries, keys and values are columns of one projection's output
    fused = torch.empty((total, hq + 2 * hkv, dim), dtype=dtype, device=DEV).normal_(generator=g)
    s["q"], s["k"], s["v"] = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    s["k_cache"] = torch.empty((pages, page, hkv, dim), dtype=dtype, device=DEV).normal_(generator=g)
    s["v_cache"] = torch.empty((pages, page, hkv, dim), dtype=dtype, device=DEV).normal_(generator=g)
    return s


# ------------------------------------------------------------------- a pass --
def run(s):
    if own:
        return _run_own(s)
    return {"clip": _clip, "plan": _plan, "store": _store, "attn": _attn}[s["kind"]](s)


def _run_own(s):
    import paper_2608_11368_amd as pair

    if s["kind"] == "clip":
        r = pair.clip_grads(s["grads"], s["max_norm"], out=s["views"])
        return {"norm": r["norm"], "coef": r["coef"], "flat": s["flat"]}
    if s["kind"] == "plan":
        r = pair.page_plan(s["cached"], s["fresh"], s["table"], s["free"], s["free_count"],
                           s["page"], s["max_tokens"], mask=s["mask"])
        return {k: r[k] for k in ("q_offsets", "lens", "slots", "positions", "table",
                                  "free_pages", "free_count")}
    if s["kind"] == "store":
        pair.cache_store(s["k"], s["v"], s["slots"], s["k_cache"], s["v_cache"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    r = pair.paged_attention(s["q"], s["k_cache"], s["v_cache"], s["table"], s["q_offsets"],
                             s["lens"], s["max_q"], s["max_len"], scale=s["scale"], want_lse=True)
    return {"out": r["out"], "lse": r["lse"]}


def _clip(s):
    flat = torch.cat([g.float() for g in s["grads"]])
    norm = flat.square().sum().sqrt()
    coef = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm))
    s["flat"].copy_(flat * coef)
    return {"norm": norm.reshape(1), "coef": coef.reshape(1), "flat": s["flat"]}


def _plan(s):
    page, table, n = s["page"], s["table"], s["cached"].numel()
    cap = s["free"].numel()
    cached = s["cached"].long()
    live = torch.ones_like(cached) if s["mask"] is None else (s["mask"] != 0).long()
    fresh = s["fresh"].long() * live
    held = (cached + page - 1) // page
    more = ((cached + fresh + page - 1) // page - held) * live
    given = held * (1 - live)
    ends = torch.cumsum(torch.stack([fresh, more, given]), 1)
    starts = ends - torch.stack([fresh, more, given])
    free = s["free_count"][0]
    left = free + ends[2, -1] - ends[1, -1]

    def pool(i):     # the free pages, then the released ones in request order
        j = i - free
        r = torch.searchsorted(ends[2], j, right=True).clamp_(max=n - 1)
        back = table[r, (j - starts[2, r]).clamp_(0, table.shape[1] - 1)]
        return torch.where(i < free, s["free"][i.clamp(max=cap - 1)], back)

    k = torch.arange(cap, device=DEV)
    r = torch.searchsorted(ends[1], k, right=True).clamp_(max=n - 1)
    taken = k < ends[1, -1]
    # entries that are not taken go to the spare last column of row 0
    table.index_put_((torch.where(taken, r, 0),
                      torch.where(taken, held[r] + k - starts[1, r], table.shape[1] - 1)),
                     torch.where(taken, pool(k), -1))
    t = torch.arange(s["max_tokens"], device=DEV)
    r = torch.searchsorted(ends[0], t, right=True).clamp_(max=n - 1)
    pos = cached[r] + t - starts[0, r]
    inside = t < ends[0, -1]
    slot = table[r, (pos // page).clamp_(max=table.shape[1] - 1)].long() * page + pos % page
    return {
        "q_offsets": torch.cat([torch.zeros_like(ends[0, :1]), ends[0]]),
        "lens": ((cached + fresh) * live).int(),
        "slots": torch.where(inside, slot, -1),
        "positions": torch.where(inside, pos, -1).int(),
        "table": table,
        "free_pages": torch.where(k < left, pool(k + ends[1, -1]), -1),
        "free_count": left.reshape(1),
    }


def _store(s):
    at = s["slots"]
    spare = s["k_cache"].shape[0] * s["k_cache"].shape[1] - 1
    keep = (at >= 0)[:, None, None]
    at = torch.where(at >= 0, at, spare)
    for new, cache in ((s["k"], s["k_cache"]), (s["v"], s["v_cache"])):
        rows = cache.view(-1, *cache.shape[2:])
        rows.index_put_((at,), torch.where(keep, new, rows[spare]))
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attn(s):
    case, n, lens = s["case"], s["lens"].numel(), s["lens"].long()
    hq, hkv, dim, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    new, top = s["max_q"], s["max_len"]
    off = s["q_offsets"]
    total = s["q"].shape[0]
    t = torch.arange(total, device=DEV)
    r = torch.searchsorted(off[1:], t, right=True)
    i = t - off[r]
    q = torch.zeros((n, new, hq, dim), device=DEV)
    q[r, i] = s["q"].float()
    q = q.view(n, new, hkv, hq // hkv, dim).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, dim)
    key = torch.arange(top, device=DEV)
    there = key[None, :] < lens[:, None]
    at = s["table"].long()[:, :-(-top // page)].clamp(min=0)
    k, v = (c[at].flatten(1, 2)[:, :top].permute(0, 2, 1, 3).float()
            for c in (s["k_cache"], s["v_cache"]))
    score = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).view(n, hq, new, top)
    last = lens[:, None] - (off[1:] - off[:-1])[:, None] + torch.arange(new, device=DEV)[None, :]
    seen = there[:, None, None, :] & (key[None, None, None, :] <= last[:, None, :, None])
    score.masked_fill_(~seen, -math.inf)
    high = score.amax(3, keepdim=True).clamp_(min=-3e38)
    score.sub_(high).exp_()
    part = score.sum(3, keepdim=True)
    v = torch.where(there[:, None, :, None], v, 0.0)
    out = torch.matmul(score.view(n, hkv, -1, top), v).view(n, hq, new, dim)
    out = torch.where(part > 0, out / part, 0.0).permute(0, 2, 1, 3)
    lse = torch.where(part > 0, part.log() + high, -math.inf)[..., 0].permute(0, 2, 1)
    return {"out": out[r, i].to(s["q"].dtype), "lse": lse[r, i]}


# ----------------------------------------------------------------- the work --
def work(case):
    if case["kind"] == "clip":
        size = _sizes(case)
        wide = sum(int(k) for k in size if k <= 4096) if case["vectors"] else 0
        total = int(size.sum())
        unit = {"f32": 4, "bf16": 2, "f16": 2}
        # a square and a sum, then a product, for each element
        return {"bytes": (total - wide) * unit[case["grad"]] + wide * 4 + total * unit[case["out"]],
                "flops": 3 * total}
    if case["kind"] == "plan":
        n, page = case["n"], case["page"]
        cached, fresh, live = _plan_lengths(case)
        held = _pages(cached, page)
        need = _pages(cached + fresh, page) - held
        pool = int(held.sum() + need.sum()) + 64
        tokens = int(fresh.sum())
        share = float(live.mean())
        # lengths, mask and offsets; slots and positions; new, held and released
        # table entries; the pool's list in and out
        return {"bytes": int(n * (8 + case["masked"] + 12) + 12 * tokens
                             + 4 * (need.sum() * share + held.sum() * (1 - share) + n)
                             + 4 * (pool - held.sum()) + 4 * pool), "flops": 0}
    unit = 2 * case["dim"]
    if case["kind"] == "store":
        real = case["tokens"] - case["pad"]
        return {"bytes": 4 * real * case["kv_heads"] * unit + 8 * case["tokens"], "flops": 0}
    length, new = _attn_lengths(case)
    pairs = int((new * (length - new) + new * (new + 1) // 2).sum())
    tokens = int(new.sum())
    return {"bytes": int(2 * length.sum() * case["kv_heads"] * unit
                         + tokens * case["q_heads"] * (2 * unit + 4)
                         + 4 * _pages(length, case["page"]).sum()),
            "flops": 4 * case["dim"] * case["q_heads"] * pairs}


# ------------------------------------------------------ the results, exactly --
def exact(case, seed):
    s = prepare(case, seed)
    return {"clip": _exact_clip, "plan": _exact_plan, "store": _exact_store,
            "attn": _exact_attn}[case["kind"]](s)


def _exact_clip(s):
    square = sum(float(torch.dot(g.double(), g.double())) for g in s["grads"])
    norm = math.sqrt(square)
    coef = min(1.0, s["max_norm"] / norm) if norm else 1.0
    flat = torch.empty(s["flat"].numel(), dtype=torch.float64, device=DEV)
    at = 0
    for g in s["grads"]:
        flat[at:at + g.numel()] = g.double() * coef
        at += g.numel()
    return {"norm": np.array([norm]), "coef": np.array([coef]), "flat": flat}


def _exact_plan(s):
    page = s["page"]
    cached, fresh = s["cached"].tolist(), s["fresh"].tolist()
    live = [1] * len(cached) if s["mask"] is None else s["mask"].tolist()
    table = s["table"].cpu().numpy().copy()
    cap = s["free"].numel()
    pages = s["free"].tolist()[:int(s["free_count"][0])]
    for r, c in enumerate(cached):
        if not live[r]:
            pages += table[r, :-(-c // page)].tolist()
    taken, q_offsets, lens, slots, positions = 0, [0], [], [], []
    for r, (c, f) in enumerate(zip(cached, fresh)):
        if live[r]:
            for k in range(-(-c // page), -(-(c + f) // page)):
                table[r, k] = pages[taken]
                taken += 1
            at = np.arange(c, c + f)
            positions.append(at)
            slots.append(table[r, at // page].astype(np.int64) * page + at % page)
        lens.append((c + f) if live[r] else 0)
        q_offsets.append(q_offsets[-1] + (f if live[r] else 0))
    tail = np.full(s["max_tokens"] - q_offsets[-1], -1)
    left = pages[taken:]
    return {"q_offsets": np.array(q_offsets, dtype=np.int64), "lens": np.array(lens, dtype=np.int32),
            "slots": np.concatenate(slots + [tail]).astype(np.int64),
            "positions": np.concatenate(positions + [tail]).astype(np.int32), "table": table,
            "free_pages": np.array(left + [-1] * (cap - len(left)), dtype=np.int32),
            "free_count": np.array([len(left)], dtype=np.int64)}


def _exact_store(s):
    out = {}
    slots = s["slots"].cpu()
    real = torch.nonzero(slots >= 0)[:, 0]
    for name in ("k", "v"):
        cache = s[name + "_cache"].double()
        rows = cache.view(-1, *cache.shape[2:])
        rows[slots[real].to(DEV)] = s[name][real.to(DEV)].double()
        out[name + "_cache"] = cache
    return out


def _exact_attn(s):
    case = s["case"]
    hq, hkv = case["q_heads"], case["kv_heads"]
    off, lens = s["q_offsets"].tolist(), s["lens"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    for r, length in enumerate(lens):
        a, b = off[r], off[r + 1]
        ids = s["table"][r, :-(-length // case["page"])].long()
        keys, values = (c[ids].flatten(0, 1)[:length].double() for c in (s["k_cache"], s["v_cache"]))
        for h in range(hkv):
            heads = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
            kt = keys[:, h].t().contiguous()
            vh = values[:, h].contiguous()
            for x in range(a, b, 512):      # rows of tokens, to bound the scores held
                y = min(b, x + 512)
                rows = s["q"][x:y, heads].double()
                score = torch.matmul(rows.reshape(-1, case["dim"]), kt) * s["scale"]
                where = length - (b - x) + torch.arange(y - x, device=DEV)
                where = where.repeat_interleave(rows.shape[1])
                score.masked_fill_(torch.arange(length, device=DEV)[None, :] > where[:, None], -math.inf)
                total = torch.logsumexp(score, 1)
                result = torch.matmul(torch.exp(score - total[:, None]), vh)
                out[x:y, heads] = result.view(rows.shape)
                lse[x:y, heads] = total.view(rows.shape[:2])
    return {"out": out, "lse": lse}
