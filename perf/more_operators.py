"""The work whose speed is measured for the paged key/value cache in 8 and 4 bits:
quantising new keys and values as they are written, reading cached rows back, and
attention over the cache as it is.

Blocks of 32 elements of a row share a scale, a power of two held in a byte
(float8_e8m0fnu); the elements are float8_e4m3fn or float4_e2m1fn, two of the
latter to a byte, the first in its low half.  The scale 2^e of a block is the
smallest for which no element passes the largest code, 448 or 6, and at least
2^-100; the elements are rounded to the nearest code, ties to the even one.
Magnitudes that no code near them stands for within the range of the 16-bit type
that they came in count as the largest that one does.

A case is a dict of plain values.  Its "kind" names the operator:

  store    new keys and values into the pages of the cache, by slot
  rewrite  the same, and what the cache then holds of them
  load     cached keys and values by slot, as 16-bit rows
  attn     attention of each request's new tokens over its pages of the cache

Sizes and lengths follow from the case alone (every seed of a case has the same
work); the seed decides their order and the values.
"""
import math
import statistics

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
CODES = {"fp8": torch.float8_e4m3fn, "fp4": torch.float4_e2m1fn_x2}
BLOCK = 32
LEAST = -100                     # least exponent of a scale
FP4 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def listed():
    return [
        # The keys and values of one decoding step: latency.
        dict(name="store_decode", kind="store", code="fp8", tokens=64, pad=0, q_heads=16,
             kv_heads=8, dim=128, page=16, layout="heads", dtype="bf16"),
        # Those of a packed chunk of prompts with a padded tail.
        dict(name="store_prompts", kind="store", code="fp8", tokens=32_768, pad=301, q_heads=32,
             kv_heads=8, dim=128, page=64, layout="heads", dtype="f16"),
        # A chunk in 4 bits, and its rows as the cache holds them, for layers
        # that go on with the very values that later steps will see.
        dict(name="rewrite_prompts", kind="rewrite", code="fp4", tokens=20_001, pad=0, q_heads=16,
             kv_heads=8, dim=128, page=16, layout="heads", dtype="bf16"),
        # One request's shared prefix, out of the cache.
        dict(name="load_prefix", kind="load", code="fp8", tokens=1500, pad=36, q_heads=16,
             kv_heads=8, dim=128, page=16, layout="heads", dtype="bf16"),
        # All rows of a drawn population of rollouts, in narrow heads.
        dict(name="load_population", kind="load", code="fp4", tokens=65_001, pad=0, q_heads=16,
             kv_heads=4, dim=64, page=32, layout="heads", dtype="f16"),
        # A token for each of four short requests: latency.
        dict(name="attn_few", kind="attn", code="fp8", n=4, ctx=400, spread=0.2, new_lo=1, new_hi=1,
             single=False, q_heads=16, kv_heads=8, dim=128, page=16, layout="heads", dtype="bf16"),
        # A decoding step of 256 rollouts of uneven length, 4000 tokens on
        # average: the cache is read once; the same in 4 bits.
        dict(name="attn_decode", kind="attn", code="fp8", n=256, ctx=4000, spread=0.5, new_lo=1,
             new_hi=1, single=False, q_heads=16, kv_heads=8, dim=128, page=16, layout="heads",
             dtype="bf16"),
        dict(name="attn_decode_fp4", kind="attn", code="fp4", n=256, ctx=4000, spread=0.5, new_lo=1,
             new_hi=1, single=False, q_heads=16, kv_heads=8, dim=128, page=16, layout="heads",
             dtype="bf16"),
        # Five drafted tokens of two very long rollouts: few rows, a long axis.
        dict(name="attn_drafts_long", kind="attn", code="fp8", n=2, ctx=131_000, spread=0.05,
             new_lo=5, new_hi=5, single=False, q_heads=32, kv_heads=8, dim=128, page=64,
             layout="heads", dtype="f16"),
        # Chunks of new prompts beside decoding requests in one step.
        dict(name="attn_mixed", kind="attn", code="fp8", n=72, ctx=2500, spread=0.4, new_lo=201,
             new_hi=640, single=True, q_heads=16, kv_heads=8, dim=128, page=16, layout="heads",
             dtype="bf16"),
        # A chunk of about 2000 new tokens of three requests with a long past.
        dict(name="attn_chunk", kind="attn", code="fp8", n=3, ctx=6000, spread=0.4, new_lo=1501,
             new_hi=2048, single=False, q_heads=32, kv_heads=8, dim=128, page=16, layout="heads",
             dtype="bf16"),
        # Whole prompts of uneven length, nothing cached before them.
        dict(name="attn_prompts", kind="attn", code="fp4", n=8, ctx=0, spread=0.0, new_lo=301,
             new_hi=4096, single=False, q_heads=16, kv_heads=4, dim=64, page=32, layout="slots",
             dtype="f16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["store", "rewrite", "load", "attn", "attn", "attn", "attn"])
    heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 2, 4, 5, 8])
    common = dict(code=rng.choice(["fp8", "fp8", "fp4"]), q_heads=heads * group, kv_heads=heads,
                  dim=rng.choice([64, 128, 128]), page=rng.choice([8, 16, 16, 20, 32, 64, 128]),
                  layout=rng.choice(["heads", "heads", "slots"]),
                  dtype=rng.choice(["bf16", "bf16", "f16"]))
    if kind == "store":
        common["code"] = "fp8"
    if kind != "attn":
        if rng.random() < 0.25:
            common["dim"] = rng.choice([32, 96, 160, 256])
        tokens = _log_int(rng, 1, 30_000)
        return dict(kind=kind, tokens=tokens, pad=rng.choice([0, rng.randint(0, tokens // 4)]),
                    **common)
    form = rng.choice(["decode", "decode", "drafts", "mixed", "chunk", "prompts"])
    if form in ("decode", "drafts"):
        new = 1 if form == "decode" else rng.randint(2, 8)
        n = _log_int(rng, 1, 256)
        ctx = _log_int(rng, 100, max(101, min(130_000, 900_000 // n)))
        return dict(kind=kind, n=n, ctx=ctx, spread=rng.choice([0.1, 0.5]), new_lo=1 if new > 1
                    and rng.random() < 0.5 else new, new_hi=new, single=False, **common)
    if form == "mixed":
        n = _log_int(rng, 9, 72)
        new = _log_int(rng, 16, 512)
        ctx = _log_int(rng, 64, 2000)
    else:
        new = _log_int(rng, 32, 2048 if form == "chunk" else 4096)
        ctx = _log_int(rng, 64, 8000) if form == "chunk" else 0
        n = rng.randint(1, 8)
    # what the plain form holds: a padded score for every head, token and key
    while n > 1 and n * common["q_heads"] * new * (2 * ctx + new) > 2_000_000_000:
        n -= 1
    while common["q_heads"] * new * (2 * ctx + new) > 2_000_000_000:
        new //= 2
    return dict(kind=kind, n=n, ctx=ctx, spread=0.3 if ctx else 0.0,
                new_lo=max(1, new // rng.choice([1, 2, 8])), new_hi=new, single=form == "mixed",
                **common)


# ------------------------------------------------------------------ inputs --
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2 + 1)
    return g


def _up(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _quantiles(n, mean, spread):
    """n lengths whose logarithms are spread normally, with the given mean."""
    if mean == 0:
        return np.zeros(n, dtype=np.int64)
    z = [statistics.NormalDist().inv_cdf((i + 0.5) / n) for i in range(n)]
    return np.maximum(1, (mean * np.exp(spread * np.array(z) - spread * spread / 2)).astype(np.int64))


def _attn_lengths(case):
    n = case["n"]
    new = case["new_lo"] + (np.arange(n) * 7919 % n) * (case["new_hi"] - case["new_lo"]) // max(1, n - 1)
    if case["single"]:                       # one in nine has a chunk
        new[np.arange(n) % 9 != 0] = 1
    return _quantiles(n, case["ctx"], case["spread"]) + new, new


def _pages(length, page):
    return (length + page - 1) // page


def _width(case):
    """Bytes of a row's codes."""
    return case["dim"] if case["code"] == "fp8" else case["dim"] // 2


def _cache(case, pages, g):
    """Codes [pages][page][kv_heads][..] and scales of one of the cache's halves,
    the slots of a head side by side ("heads") or the heads of a slot."""
    heads, page, dim = case["kv_heads"], case["page"], case["dim"]
    order = (heads, page) if case["layout"] == "heads" else (page, heads)
    codes = torch.empty((pages, *order, _width(case)), dtype=torch.uint8, device=DEV)
    scales = torch.empty((pages, *order, dim // BLOCK), dtype=torch.uint8, device=DEV)
    each = max(1, (1 << 26) // (page * heads * dim))
    for p in range(0, pages, each):
        there = codes[p:p + each].shape[:3]
        x = torch.empty((*there, dim), device=DEV).normal_(generator=g)
        x *= torch.empty((*there, 1), device=DEV).normal_(0, 0.3, generator=g).exp_()
        codes[p:p + each], scales[p:p + each] = _quantise(x, case)
    if case["layout"] == "heads":
        codes, scales = codes.transpose(1, 2), scales.transpose(1, 2)
    return codes.view(CODES[case["code"]]), scales.view(torch.float8_e8m0fnu)


def prepare(case, seed):
    rng = np.random.default_rng([int(seed), 11])
    s = dict(case=case, kind=case["kind"])
    dim, hq, hkv, page = case["dim"], case["q_heads"], case["kv_heads"], case["page"]
    dtype, g = TYPES[case["dtype"]], _gen(seed)
    if case["kind"] != "attn":
        tokens = total = case["tokens"]
        pages = _pages(tokens, page) + 9
        # a batch's tokens land in page-sized runs; the last page is never handed out
        ids = rng.permutation(pages - 1)[:_pages(tokens, page)]
        slots = (ids[:, None] * page + np.arange(page)[None, :]).reshape(-1)[:tokens].astype(np.int64)
        if case["pad"]:
            slots[tokens - case["pad"]:] = -1
        s["slots"] = _up(slots)
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
    if case["kind"] != "load":
        # queries, keys and values are columns of one projection's output
        fused = torch.empty((total, hq + 2 * hkv, dim), dtype=dtype, device=DEV).normal_(generator=g)
        s["q"], s["k"], s["v"] = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    s["k_cache"], s["k_scale"] = _cache(case, pages, g)
    s["v_cache"], s["v_scale"] = _cache(case, pages, g)
    return s


# ------------------------------------------------------------------- a pass --
def run(s):
    if own:
        return _run_own(s)
    return {"store": _store, "rewrite": _rewrite, "load": _load, "attn": _attn}[s["kind"]](s)


def _run_own(s):
    import paper_2608_11368_amd as pair

    cache = s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]
    if s["kind"] == "attn":
        r = pair.paged_attention_mx(s["q"], *cache, s["table"], s["q_offsets"], s["lens"],
                                    s["max_q"], s["max_len"], scale=s["scale"], want_lse=True)
        return {"out": r["out"], "lse": r["lse"]}
    if s["kind"] in ("store", "rewrite"):
        pair.cache_store_mx(s["k"], s["v"], s["slots"], *cache)
        if s["kind"] == "store":
            return _held(s)
    r = pair.cache_load_mx(s["slots"], *cache, dtype=TYPES[s["case"]["dtype"]])
    return {"k": r["k"], "v": r["v"]}


def _held(s):
    return {x: s[x] for x in ("k_cache", "v_cache", "k_scale", "v_scale")}


def _quantise(x, case):
    """Codes and scales, as bytes, of fp32 rows [..., dim]."""
    top = 448.0 if case["code"] == "fp8" else 6.0
    most = 1.875 if case["code"] == "fp8" else 1.5
    most *= 2.0 ** (15 if case["dtype"] == "f16" else 127)
    b = x.reshape(*x.shape[:-1], -1, BLOCK).clamp(-most, most)
    part, exponent = torch.frexp(b.abs().amax(-1, keepdim=True))     # part in [0.5, 1)
    top_part, top_exponent = math.frexp(top)
    exponent = exponent - top_exponent + (part > top_part).int()
    exponent = torch.where(part == 0, LEAST, exponent).clamp(min=LEAST)
    y = torch.ldexp(b, -exponent.float())
    if case["code"] == "fp8":
        code = y.to(torch.float8_e4m3fn).view(torch.uint8).view(x.shape)
    else:
        a = y.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        # at 2 and 4 steps the codes before are four and two further
        index = (a / step).round() + torch.where(a < 2, 0.0, torch.where(a < 4, 2.0, 4.0))
        code = (index.to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)).view(x.shape)
        code = code[..., ::2] | (code[..., 1::2] << 4)
    return code, (exponent[..., 0] + 127).to(torch.uint8)


def _values(code, scale):
    """fp32 rows of codes and scales given as bytes."""
    if code.shape[-1] == scale.shape[-1] * BLOCK:
        v = code.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor(FP4 + [-x for x in FP4], device=code.device)
        v = table[torch.stack([code & 15, code >> 4], -1).long()].flatten(-2)
    b = v.view(*v.shape[:-1], -1, BLOCK) * scale.view(torch.float8_e8m0fnu).float()[..., None]
    return b.view(v.shape)


def _bytes(s, half):
    return s[half + "_cache"].view(torch.uint8), s[half + "_scale"].view(torch.uint8)


def _store_half(s, half):
    page = s["case"]["page"]
    spare = s["k_cache"].shape[0] * page - 1
    keep = (s["slots"] >= 0)[:, None, None]
    at = torch.where(s["slots"] >= 0, s["slots"], spare)
    at = (at // page, at % page)
    new_codes, new_scales = _quantise(s[half].float(), s["case"])
    codes, scales = _bytes(s, half)
    codes.index_put_(at, torch.where(keep, new_codes, codes[-1, -1]))
    scales.index_put_(at, torch.where(keep, new_scales, scales[-1, -1]))


def _store(s):
    _store_half(s, "k")
    _store_half(s, "v")
    return _held(s)


def _load_half(s, half):
    page = s["case"]["page"]
    at = s["slots"].clamp(min=0)
    at = (at // page, at % page)
    codes, scales = _bytes(s, half)
    rows = torch.where((s["slots"] >= 0)[:, None, None], _values(codes[at], scales[at]), 0.0)
    return rows.to(TYPES[s["case"]["dtype"]])


def _load(s):
    return {"k": _load_half(s, "k"), "v": _load_half(s, "v")}


def _rewrite(s):
    _store(s)
    return _load(s)


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
    k, v = (_values(*(x[at].flatten(1, 2)[:, :top].permute(0, 2, 1, 3).contiguous()
                      for x in _bytes(s, half))) for half in ("k", "v"))
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
    row = _width(case) + case["dim"] // BLOCK          # bytes of a row in the cache
    if case["kind"] != "attn":
        real = case["tokens"] - case["pad"]
        rows = 2 * real * case["kv_heads"]
        wide = rows * 2 * case["dim"]                  # the 16-bit rows
        if case["kind"] == "rewrite":
            return {"bytes": 2 * wide + rows * row + 8 * case["tokens"], "flops": 0}
        if case["kind"] == "load":                     # a row of zeros for a slot that is none
            wide += 2 * case["pad"] * case["kv_heads"] * 2 * case["dim"]
        return {"bytes": wide + rows * row + 8 * case["tokens"], "flops": 0}
    length, new = _attn_lengths(case)
    pairs = int((new * (length - new) + new * (new + 1) // 2).sum())
    tokens = int(new.sum())
    return {"bytes": int(2 * length.sum() * case["kv_heads"] * row
                         + tokens * case["q_heads"] * (4 * case["dim"] + 4)
                         + 4 * _pages(length, case["page"]).sum()),
            "flops": 4 * case["dim"] * case["q_heads"] * pairs}


# ------------------------------------------------------ the results, exactly --
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attn":
        return _exact_attn(s)
    if case["kind"] == "load":
        real = (s["slots"] >= 0)[:, None, None]
        pg, y = s["slots"].clamp(min=0) // case["page"], s["slots"].clamp(min=0) % case["page"]
        return {h: torch.where(real, _exact_values(*(x[pg, y] for x in _bytes(s, h))), 0.0)
                for h in ("k", "v")}
    out = {}
    if case["kind"] == "rewrite":
        for h in ("k", "v"):
            code, scale = _exact_codes(s[h].double(), case)
            out[h] = torch.where((s["slots"] >= 0)[:, None, None],
                                 code * scale.repeat_interleave(BLOCK, -1), 0.0)
        return out
    slots = s["slots"].cpu()
    real = torch.nonzero(slots >= 0)[:, 0].to(DEV)
    pg, y = s["slots"][real] // case["page"], s["slots"][real] % case["page"]
    for h in ("k", "v"):
        code, scale = _exact_codes(s[h][real].double(), case)
        out[h + "_cache"], out[h + "_scale"] = s[h + "_cache"].double(), s[h + "_scale"].double()
        out[h + "_cache"][pg, y], out[h + "_scale"][pg, y] = code, scale
    return out


def _positive(code):
    """The code values that are not negative, in order, from their bits."""
    if code == "fp4":
        bits, mantissa, bias = np.arange(8), 1, 1
    else:
        bits, mantissa, bias = np.arange(127), 3, 7
    e, m = bits >> mantissa, (bits & ((1 << mantissa) - 1)) / (1 << mantissa)
    v = np.where(e > 0, (1 + m) * 2.0 ** (e - bias), m * 2.0 ** (1 - bias))
    return torch.from_numpy(v).to(DEV)


def _exact_codes(x, case):
    """Values of the codes and of the scales of rows in 64 bits."""
    known = _positive(case["code"])
    # the largest number of the 16-bit type that is a code's times a power of two
    most = float((known[known > 0] / 2.0 ** torch.floor(torch.log2(known[known > 0]))).max())
    most *= 2.0 ** math.floor(math.log2(torch.finfo(TYPES[case["dtype"]]).max))
    blocks = x.reshape(*x.shape[:-1], -1, BLOCK).clamp(-most, most)
    high = blocks.abs().amax(-1)
    scale = 2.0 ** torch.ceil(torch.log2(high / float(known[-1])))
    scale = torch.where(high == 0, 2.0 ** LEAST, scale).clamp(min=2.0 ** LEAST)
    a = blocks.abs() / scale[..., None]
    below = torch.searchsorted(known, a, right=True) - 1
    above = (below + 1).clamp(max=len(known) - 1)
    to_below, to_above = a - known[below], known[above] - a
    up = (to_above < to_below) | ((to_above == to_below) & (below % 2 == 1))
    code = torch.where(up, known[above], known[below])
    return torch.copysign(code, blocks).view(x.shape), scale


def _exact_values(code, scale):
    wide = code.shape[-1] == scale.shape[-1] * BLOCK
    known = _positive("fp8" if wide else "fp4")
    if wide:                                           # 127 is no number's code
        known = torch.cat([known, torch.full((1,), math.nan, device=DEV, dtype=torch.float64)])
        bits = code.long()
    else:
        bits = torch.stack([code.long() % 16, code.long() // 16], -1).flatten(-2)
    half = len(known)
    v = torch.where(bits < half, known[bits % half], -known[bits % half])
    return v * torch.pow(2.0, scale.double() - 127).repeat_interleave(BLOCK, -1)


def _exact_attn(s):
    case = s["case"]
    hq, hkv = case["q_heads"], case["kv_heads"]
    off, lens = s["q_offsets"].tolist(), s["lens"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    for r, length in enumerate(lens):
        a, b = off[r], off[r + 1]
        ids = s["table"][r, :-(-length // case["page"])].long()
        keys, values = (_exact_values(*(x[ids].flatten(0, 1)[:length] for x in _bytes(s, half)))
                        for half in ("k", "v"))
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
