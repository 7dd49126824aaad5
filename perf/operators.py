"""Performance cases of the cache operators that stand around a tree step: what the target model's attention layers ask of the library.

A tree step hands the target model T = n + 1 tokens per sequence: the root, then the packed nodes of the tree.  Each layer appends
their keys and values to a paged cache that holds 8-bit floats (e4m3) with one scale per page and head, attends with the tree's
bitmask, and after verification the entries of the accepted path move together.  The forms (`op`):

  append   norm and rotation of queries and keys, keys and values into the cache
  attend   attention of the step's tokens over the cached prefix and over their ancestors in the step
  compact  the accepted path's entries of every layer to the end of the prefix

`kind` says what a step is: `token` (one token, plain decoding), `tree` (root and nodes, bitmask), `chain` (a prompt's chunk).
Sizes are those of the decoding configurations (node budgets 10 ... 256, depths 6 ... 20, batches 1 ... 64); heads and contexts are
generic ones.
"""
import math
import random
from functools import lru_cache

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
F8 = torch.float8_e4m3fn
LARGEST = 448.0            # largest e4m3 value
LEAST_EXP = -64            # smallest scale: 2 to this
BASE = 10000.0             # rotation base
EPS = 1e-6


def listed():
    def case(name, op, kind, B, n, depth, ctx, hq, hkv, d, page, dtype="bf16", norm=False, style="halves", layers=1):
        return dict(name=name, op=op, kind=kind, B=B, n=n, depth=depth, ctx=ctx, hq=hq, hkv=hkv, d=d, page=page, dtype=dtype,
                    norm=norm, style=style, layers=layers)
    return [
        case("append-token", "append", "token", 1, 0, 0, 700, 32, 8, 128, 16),                              # one user, one token: latency
        case("append-tree-b32", "append", "tree", 32, 64, 10, 1000, 32, 8, 128, 32, norm=True),             # a serving batch's trees, normed heads
        case("append-chunk", "append", "chain", 4, 4095, 0, 0, 32, 8, 128, 64, "fp16", True, "pairs"),      # prompts, rotated in pairs
        case("attend-token-b1", "attend", "token", 1, 0, 0, 1500, 32, 8, 128, 16),                          # one user, one token: latency
        case("attend-token-b32", "attend", "token", 32, 0, 0, 16384, 32, 8, 128, 64),                       # plain decoding of a batch, long contexts
        case("attend-token-long", "attend", "token", 1, 0, 0, 131071, 28, 4, 128, 32),                      # one very long context, seven query heads a head
        case("attend-tree-n10", "attend", "tree", 1, 10, 6, 900, 32, 8, 128, 16),                           # the smallest tree
        case("attend-tree-n50", "attend", "tree", 1, 50, 10, 4000, 32, 8, 128, 32, "fp16"),                 # the usual tree of one user
        case("attend-tree-b32", "attend", "tree", 32, 64, 10, 4096, 32, 8, 128, 32),                        # the benchmark's batch
        case("attend-tree-b64-n256", "attend", "tree", 64, 256, 20, 2048, 16, 4, 64, 16),                   # the largest budget and batch, small heads
        case("compact-b1", "compact", "tree", 1, 50, 10, 300, 32, 8, 128, 16, layers=32),                   # one user, all layers
        case("compact-b32", "compact", "tree", 32, 64, 10, 150, 32, 8, 128, 32, layers=32),                 # a serving batch, all layers
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "attend", "compact"])
    kind = "tree" if op == "compact" else rng.choice(["token", "tree", "tree", "chain"])
    hkv = rng.choice([1, 2, 4, 8])
    c = dict(op=op, kind=kind, B=_log_int(rng, 1, 64), n=0, depth=0, ctx=_log_int(rng, 1, 40000), hq=hkv * rng.choice([1, 2, 3, 4, 6, 7, 8]),
             hkv=hkv, d=rng.choice([64, 128]), page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["bf16", "fp16"]),
             norm=rng.random() < 0.5, style=rng.choice(["halves", "pairs"]), layers=1)
    if kind == "tree":
        c["depth"] = rng.randint(4, 20)
        c["n"] = max(c["depth"], _log_int(rng, 4, 256))
    elif kind == "chain":
        c["n"] = _log_int(rng, 2, 1500) - 1
    if op == "compact":
        c["layers"] = rng.randint(1, 32)
    pairs = 32 * 65 * 32 * 4096                          # (query, key) pairs and cached tokens of the listed cases
    tokens = 16384 * 32 * 8
    while (c["n"] + 1) * c["B"] * c["hq"] * (c["ctx"] + c["n"] + 1) > pairs or (c["ctx"] + c["n"] + 1) * c["B"] * c["hkv"] * c["layers"] > tokens:
        c["B"], c["ctx"] = max(1, c["B"] // 2), max(1, c["ctx"] * 3 // 4)
    return c


# ---- sizes of a case: the same for every seed ----------------------------------------------------------------------

def lengths(case):
    """Cached tokens of each sequence: the first has all of `ctx`, the others between a half and all of it."""
    r = random.Random(case["B"] * 1000003 + case["ctx"])
    return [case["ctx"] - (r.randint(0, case["ctx"] // 2) if b else 0) for b in range(case["B"])]


def node_counts(case):
    """Nodes of each sequence's step: trees and chunks of a batch are not all of one size."""
    r = random.Random(case["B"] * 7919 + case["n"])
    return [case["n"] - (r.randint(0, case["n"] // 4) if b else 0) for b in range(case["B"])]


def _pages(case):
    return -(-(case["ctx"] + case["n"] + 1) // case["page"])


def work(case):
    lens, nodes, d, page = lengths(case), node_counts(case), case["d"], case["page"]
    hq, hkv = case["hq"], case["hkv"]
    new = sum(x + 1 for x in nodes)
    if case["op"] == "append":
        touched = sum((l + x) // page - l // page + 1 for l, x in zip(lens, nodes))
        table = sum(l + x + 1 - l for l, x in zip(lens, nodes)) if case["kind"] == "chain" else new
        return {"bytes": new * (hq + 2 * hkv) * d * 2 + new * hq * d * 2 + new * 2 * hkv * d + touched * hkv * 8 + min(table, case["ctx"] + case["n"] + 1) * d * 4,
                "flops": new * (hq + hkv) * d * (7 if case["norm"] else 3) + new * hkv * d * 4}
    if case["op"] == "attend":
        keys = sum(l + x + 1 for l, x in zip(lens, nodes))
        scales = sum((l + x) // page + 1 for l, x in zip(lens, nodes))
        inside = {"token": lambda x: 1, "chain": lambda x: (x + 1) * (x + 2) // 2, "tree": lambda x: (x + 1) * (2 + case["depth"] // 2)}[case["kind"]]
        seen = sum((x + 1) * l + inside(x) for l, x in zip(lens, nodes))
        return {"bytes": keys * 2 * hkv * d + scales * 8 * hkv + new * hq * d * 4, "flops": 4 * d * hq * seen}
    kept = sum(max(1, case["depth"] // 2 - b % 3) for b in range(case["B"]))
    return {"bytes": kept * 2 * hkv * d * case["layers"] * 2, "flops": kept * hkv * d * case["layers"]}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _tree(rs, n, nodes, depth):
    """(parent [n], depth [n]) of a random tree of `nodes` nodes in packed order; tail slots -1 and 0."""
    parent, level = np.full(n, -1, np.int32), np.zeros(n, np.int32)
    levels = min(depth, nodes)
    at = np.sort(np.concatenate([np.arange(1, levels + 1), 1 + (rs.random_sample(nodes - levels) ** 1.5 * levels).astype(np.int64)]))
    level[:nodes] = at
    for x in range(2, levels + 1):
        before, here = np.flatnonzero(at == x - 1), np.flatnonzero(at == x)
        parent[here] = np.sort(rs.choice(before, len(here)))
    return parent, level


def _bits(parent, nodes, n):
    """The ancestor-or-self bitmask [n][ceil(n/64)] as int64 words."""
    see = np.zeros((n, (n + 63) // 64 * 64), bool)
    for i in range(nodes):
        if parent[i] >= 0:
            see[i] = see[parent[i]]
        see[i, i] = True
    return np.packbits(see, axis=1, bitorder="little").view(np.int64)


def prepare(case, seed):
    c, dev = case, "cuda"
    B, n, d, page, hq, hkv, L = c["B"], c["n"], c["d"], c["page"], c["hq"], c["hkv"], c["layers"]
    T, per = n + 1, _pages(case)
    dt = DTYPES[c["dtype"]]
    rs = np.random.RandomState(seed % (1 << 31))
    g = torch.Generator(device=dev).manual_seed(seed)
    total = B * per
    table = torch.from_numpy(rs.permutation(total).astype(np.int32).reshape(B, per)).to(dev)

    def codes():        # one draw per layer keeps the temporary small
        x = torch.empty((L, total, hkv, page, d), dtype=F8, device=dev)
        for layer in x:
            layer.copy_((torch.randn(layer.shape, generator=g, device=dev) * 100).clamp_(-LARGEST, LARGEST))
        return x

    def scales():       # pages differ by a few powers of two
        return torch.exp2(torch.randint(-8, -5, (L, total, hkv), generator=g, device=dev).float())

    s = dict(case=dict(c), lens=torch.tensor(lengths(c), dtype=torch.int32, device=dev),
             nodes=torch.tensor(node_counts(c), dtype=torch.int32, device=dev), table=table,
             k=codes(), v=codes(), ks=scales(), vs=scales(), positions=None, mask=None)
    s["base"] = s["lens"]
    if c["kind"] == "tree":
        trees = [_tree(rs, n, x, c["depth"]) for x in node_counts(c)]
        s["mask"] = torch.from_numpy(np.stack([_bits(p, x, n) for (p, _), x in zip(trees, node_counts(c))])).to(dev)
        level = torch.from_numpy(np.stack([v for _, v in trees])).to(dev)
        s["positions"] = torch.where(level > 0, s["base"][:, None] + level, 0).to(torch.int32)
    if c["op"] == "compact":
        # the accepted path: the root, then nodes further on than the entries they replace, as deep nodes of a tree are
        keep = [max(1, c["depth"] // 2 - b % 3) for b in range(B)]
        gather = np.full((B, c["depth"] + 1), -1, np.int32)
        for b, (x, m) in enumerate(zip(node_counts(c), keep)):
            m = keep[b] = min(m, 1 + max(0, (x + 1 - m)))
            gather[b, 0] = 0
            gather[b, 1:m] = np.sort(rs.choice(np.arange(m, x + 1), m - 1, replace=False)) if m > 1 else []
        s["gather"], s["keep"] = torch.from_numpy(gather).to(dev), torch.tensor(keep, dtype=torch.int32, device=dev)
        return s
    if c["op"] == "append":
        # a fused projection's output; channels of keys differ in size, as they do in trained models
        qkv = torch.randn((B, T, hq + 2 * hkv, d), generator=g, device=dev) * torch.exp(0.7 * torch.randn(d, generator=g, device=dev))
        qkv = qkv.to(dt)
        s["q"], s["kn"], s["vn"] = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
        s["qw"] = s["kw"] = None
        if c["norm"]:
            s["qw"], s["kw"] = ((1 + 0.3 * torch.randn(d, generator=g, device=dev)).to(dt) for _ in range(2))
        angle = torch.arange(c["ctx"] + T, device=dev, dtype=torch.float64)[:, None] * BASE ** (-torch.arange(0, d, 2, device=dev, dtype=torch.float64) / d)
        s["rot"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        s["q_out"] = torch.zeros((B, T, hq, d), dtype=dt, device=dev)
    else:
        s["q"] = (2 * torch.randn((B, T, hq, d), generator=g, device=dev)).to(dt)
        s["out"] = torch.zeros((B, T, hq, d), dtype=dt, device=dev)
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------------

def _round_e4m3(x):
    """Nearest e4m3 value (ties to even, saturating) of fp64 x."""
    _, e = torch.frexp(x)
    ulp = torch.ldexp(torch.ones_like(x), e.clamp(min=-5) - 4)
    return (torch.round(x / ulp) * ulp).clamp(-LARGEST, LARGEST)


def _scale_of(amax):
    """Smallest power of two that brings amax to 448 or below."""
    m, e = torch.frexp(amax / LARGEST)
    e = torch.where(m == 0.5, e - 1, e)
    e = torch.where(amax > 0, e, torch.full_like(e, LEAST_EXP)).clamp(min=LEAST_EXP)
    return torch.ldexp(torch.ones_like(amax), e)


def _positions(s, T):
    j = torch.arange(T, device="cuda")
    if s["positions"] is None:
        return (s["base"][:, None] + j).long()
    return torch.cat([s["base"][:, None], s["positions"]], 1).long()


def _rotate(x, cs, style):
    h = x.shape[-1] // 2
    cos, sin = cs[..., :h], cs[..., h:]
    if style == "halves":
        a, b = x[..., :h], x[..., h:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)


def _norm(x, w):
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.double()


def _plain_append(s):
    c = s["case"]
    B, T, page = c["B"], c["n"] + 1, c["page"]
    valid = torch.arange(T, device="cuda") <= s["nodes"][:, None]
    pos = _positions(s, T).clamp(max=s["rot"].shape[0] - 1)
    cs = s["rot"].double()[pos][:, :, None]
    q = _rotate(_norm(s["q"].double(), s["qw"]), cs, c["style"])
    s["q_out"].copy_(torch.where(valid[..., None, None], q.to(s["q_out"].dtype), s["q_out"]))
    # the pages that the step touches, laid out over their slots
    first = s["lens"] // page
    most = (T - 1) // page + 2
    at = (first[:, None] + torch.arange(most, device="cuda")).long()
    slot = at[..., None] * page + torch.arange(page, device="cuda")
    j = slot - s["lens"][:, None, None]
    new = (j >= 0) & (j <= s["nodes"][:, None, None])
    used = new.any(-1)
    ids = torch.gather(s["table"], 1, at.clamp(max=s["table"].shape[1] - 1)).long()[used]
    j, new, old = j.clamp(0, T - 1)[used], new[used], (slot < s["lens"][:, None, None])[used]
    seq = torch.arange(B, device="cuda")[:, None].expand(B, most)[used]
    for name, scale, x in (("k", "ks", _rotate(_norm(s["kn"].double(), s["kw"]), cs, c["style"])), ("v", "vs", s["vn"].double())):
        x = x[seq[:, None], j].transpose(1, 2)                                          # [pages][head][slot][d]
        x = torch.where(new[:, None, :, None], x, 0)
        was, sc = s[name][0][ids].double(), s[scale][0][ids].double()
        now = _scale_of(x.abs().amax((-1, -2)))
        now = torch.maximum(now, torch.where(old.any(-1)[:, None], sc, 0))
        kept = torch.where(old[:, None, :, None], _round_e4m3(was * (sc / now)[..., None, None]), was)
        s[name][0][ids] = torch.where(new[:, None, :, None], _round_e4m3(x / now[..., None, None]), kept).float().to(F8)
        s[scale][0][ids] = now.float()
    return {"q": s["q_out"], "k": s["k"], "v": s["v"], "k_scale": s["ks"], "v_scale": s["vs"]}


def _visible(s, S):
    """[B][T][S] truth values: which slots each token of the step sees."""
    c = s["case"]
    B, T = c["B"], c["n"] + 1
    slot, i = torch.arange(S, device="cuda"), torch.arange(T, device="cuda")
    j = slot - s["lens"][:, None]                                                       # [B][S]: index inside the step
    inside = (j >= 0) & (j <= s["nodes"][:, None])
    if s["mask"] is None:
        step = j[:, None] <= i[:, None]
    else:
        bit = (j - 1).clamp(0, T - 2).long()[:, None].expand(B, T - 1, S)
        word = torch.gather(s["mask"], 2, bit >> 6)
        step = torch.cat([torch.zeros((B, 1, S), dtype=torch.bool, device="cuda"), ((word >> (bit & 63)) & 1).bool() & (j >= 1)[:, None]], 1) | (j == 0)[:, None]
    return (j < 0)[:, None] | (inside[:, None] & step)


def _plain_attend(s):
    c = s["case"]
    B, T, d, hq, hkv, page = c["B"], c["n"] + 1, c["d"], c["hq"], c["hkv"], c["page"]
    g, S = hq // hkv, s["table"].shape[1] * page
    ids = s["table"].long()

    def whole(x, scale):        # [B][head][S][d]
        x = x[0][ids].float() * scale[0][ids][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(B, hkv, S, d)

    see = _visible(s, S)
    q = s["q"].float().view(B, T, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(B, hkv, g * T, d)
    x = (q @ whole(s["k"], s["ks"]).transpose(2, 3)).view(B, hkv, g, T, S) * (d ** -0.5)
    x = torch.where(see[:, None, None], x, -math.inf)
    x = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-3e38))
    total = x.sum(-1, keepdim=True)
    v = torch.where((torch.arange(S, device="cuda") <= (s["lens"] + s["nodes"])[:, None])[:, None, :, None], whole(s["v"], s["vs"]), 0)
    o = (x.view(B, hkv, g * T, S) @ v).view(B, hkv, g, T, d) / total
    valid = torch.arange(T, device="cuda") <= s["nodes"][:, None]
    s["out"].copy_(torch.where(valid[..., None, None], o.permute(0, 3, 1, 2, 4).reshape(B, T, hq, d), s["out"].float()))
    return {"out": s["out"]}


def _plain_compact(s):
    c = s["case"]
    B, page, G = c["B"], c["page"], s["gather"].shape[1]
    first = s["lens"] // page
    most = (G - 1) // page + 2
    at = (first[:, None] + torch.arange(most, device="cuda")).long()
    slot = at[..., None] * page + torch.arange(page, device="cuda")
    j = slot - s["lens"][:, None, None]
    moved = (j >= 0) & (j < s["keep"][:, None, None])
    used = moved.any(-1)
    j, seq = j.clamp(0, G - 1)[used].long(), torch.arange(B, device="cuda")[:, None].expand(B, most)[used]
    ids = torch.gather(s["table"], 1, at.clamp(max=s["table"].shape[1] - 1)).long()[used]
    src = (s["lens"][seq][:, None] + s["gather"][seq[:, None], j].clamp(min=0)).long()
    moved = moved[used]
    sid = s["table"][seq[:, None], src // page].long()                                  # [pages][slot]
    for name, scale in (("k", "ks"), ("v", "vs")):
        own_s = s[scale][:, ids]                                                        # [L][pages][head]
        src_s = s[scale][:, sid].transpose(2, 3)                                        # [L][pages][head][slot]
        now = torch.maximum(own_s, torch.where(moved[:, None], src_s, 0).amax(-1))
        x = s[name][:, sid, :, src % page].float()                                      # [pages][slot][L][head][d]
        x = x.permute(2, 0, 3, 1, 4) * (src_s / now[..., None])[..., None]
        was = s[name][:, ids].float() * (own_s / now)[..., None, None]
        s[name][:, ids] = _round_e4m3(torch.where(moved[:, None, :, None], x, was).double()).float().to(F8)
        s[scale][:, ids] = now
    return {"k": s["k"], "v": s["v"], "k_scale": s["ks"], "v_scale": s["vs"], "len": s["lens"] + s["keep"]}


# ---- the framework's calls -----------------------------------------------------------------------------------------

@lru_cache(maxsize=64)
def _handle(hq, hkv, d, page, pages, per, B, T, layers, dtype):
    from paper_2406_17276_b200 import binding
    return binding.TreeKV(q_heads=hq, kv_heads=hkv, head_dim=d, page=page, num_pages=pages, max_pages=per, max_batch=B, max_step=T,
                          layers=layers, dtype=DTYPES[dtype])


def _own(s):
    from paper_2406_17276_b200 import binding
    c = s["case"]
    per = s["table"].shape[1]
    kv = _handle(c["hq"], c["hkv"], c["d"], c["page"], s["k"].shape[1], per, c["B"], c["n"] + 1, c["layers"], c["dtype"])
    cache = binding.KVCache(s["k"], s["v"], s["ks"], s["vs"], s["table"])
    if c["op"] == "compact":
        length = kv.compact(cache, s["lens"], s["gather"], s["keep"])
        return {"k": s["k"], "v": s["v"], "k_scale": s["ks"], "v_scale": s["vs"], "len": length}
    step = binding.KVStep(kv_len=s["lens"], nodes=s["nodes"], base_pos=s["base"], position_ids=s["positions"], mask=s["mask"])
    if c["op"] == "append":
        q = kv.append(cache, 0, s["q"], s["kn"], s["vn"], step, cos_sin=s["rot"], q_norm=s["qw"], k_norm=s["kw"], eps=EPS,
                      interleaved=c["style"] == "pairs", q_out=s["q_out"])
        return {"q": q, "k": s["k"], "v": s["v"], "k_scale": s["ks"], "v_scale": s["vs"]}
    return {"out": kv.attend(cache, 0, s["q"], step, out=s["out"])}


def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "attend": _plain_attend, "compact": _plain_compact}[s["case"]["op"]](s)


# ---- the definition in 64 bits, sequence by sequence ---------------------------------------------------------------

def _codes64():
    """All finite e4m3 values, ascending, from the format: 4 bits of exponent with bias 7, 3 of fraction."""
    pos = [m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127]
    return torch.tensor([-x for x in pos[:0:-1]] + pos, dtype=torch.float64, device="cuda")


def _nearest64(x):
    """Nearest code by comparison with both neighbours; ties to the even fraction."""
    all_ = _codes64()
    x = x.clamp(-LARGEST, LARGEST)
    hi = torch.searchsorted(all_, x).clamp(max=len(all_) - 1)
    lo = (hi - 1).clamp(min=0)
    below, above = x - all_[lo], all_[hi] - x
    odd_lo = (lo - 126).abs() % 2 == 1
    return torch.where((below < above) | ((below == above) & ~odd_lo), all_[lo], all_[hi])


def _turned64(x, w, cs, style):
    x = x.double()
    if w is not None:
        x = x / ((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w.double()
    h = x.shape[-1] // 2
    z = torch.complex(x[..., :h], x[..., h:]) if style == "halves" else torch.complex(x[..., 0::2].contiguous(), x[..., 1::2].contiguous())
    z = z * torch.complex(cs[..., :h], cs[..., h:])
    return torch.cat([z.real, z.imag], -1) if style == "halves" else torch.stack([z.real, z.imag], -1).reshape(x.shape)


def _exact_append(s):
    c = s["case"]
    page = c["page"]
    q, k, v = s["q_out"].double(), s["k"].double(), s["v"].double()
    ks, vs = s["ks"].double(), s["vs"].double()
    for b, (n0, x) in enumerate(zip(lengths(c), node_counts(c))):
        m = x + 1
        where = torch.arange(n0, n0 + m, device="cuda")
        at = where if s["positions"] is None else torch.cat([where[:1], s["positions"][b, :x].long()])
        cs = s["rot"].double()[at][:, None]
        q[b, :m] = _turned64(s["q"][b, :m], s["qw"], cs, c["style"])
        for codes, scale, new in ((k[0], ks[0], _turned64(s["kn"][b, :m], s["kw"], cs, c["style"])), (v[0], vs[0], s["vn"][b, :m].double())):
            for p in range(n0 // page, (n0 + x) // page + 1):
                lo, hi = max(n0, p * page), min(n0 + m, (p + 1) * page)
                part, i = new[lo - n0:hi - n0], int(s["table"][b, p])
                need = (part.abs().amax((0, 2)) / LARGEST).clamp(min=2.0 ** LEAST_EXP).log2()
                need = torch.where((need - need.round()).abs() < 1e-12, need.round(), need.ceil())
                now = torch.exp2(need)
                if lo > p * page:
                    now = torch.maximum(now, scale[i])
                    codes[i][:, :lo - p * page] = _nearest64(codes[i][:, :lo - p * page] * (scale[i] / now)[:, None, None])
                scale[i] = now
                codes[i][:, lo - p * page:hi - p * page] = _nearest64(part.transpose(0, 1) / now[:, None, None])
    return {"q": q, "k": k, "v": v, "k_scale": ks, "v_scale": vs}


def _exact_attend(s):
    c = s["case"]
    g = c["hq"] // c["hkv"]
    out = s["out"].double()
    for b, (n0, x) in enumerate(zip(lengths(c), node_counts(c))):
        m = x + 1
        ids = s["table"][b, :-(-(n0 + m) // c["page"])].long()
        k, v = ((t[0, ids].double() * sc[0, ids].double()[..., None, None]).transpose(0, 1).reshape(c["hkv"], -1, c["d"])[:, :n0 + m]
                for t, sc in ((s["k"], s["ks"]), (s["v"], s["vs"])))
        see = torch.ones((m, n0 + m), dtype=torch.bool, device="cuda")
        if s["mask"] is None:
            see[:, n0:] = torch.ones((m, m), device="cuda").tril().bool()
        else:
            bits = np.unpackbits(s["mask"][b].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:x, :x].astype(bool)
            see[0, n0 + 1:] = False
            see[1:, n0 + 1:] = torch.from_numpy(bits).cuda()
        for h in range(c["hkv"]):
            a = torch.einsum("tgd,sd->tgs", s["q"][b, :m, h * g:(h + 1) * g].double(), k[h]) / math.sqrt(c["d"])
            a = torch.softmax(a.masked_fill(~see[:, None], -math.inf), -1)
            out[b, :m, h * g:(h + 1) * g] = torch.einsum("tgs,sd->tgd", a, v[h])
    return {"out": out}


def _exact_compact(s):
    c = s["case"]
    page = c["page"]
    k, v, ks, vs = s["k"].float(), s["v"].float(), s["ks"].double(), s["vs"].double()
    table, gather, keep = s["table"].tolist(), s["gather"].tolist(), s["keep"].tolist()
    for b, n0 in enumerate(lengths(c)):
        for codes, scale in ((k, ks), (v, vs)):
            for p in range(n0 // page, (n0 + keep[b] - 1) // page + 1):
                i = table[b][p]
                rows = [(n0 + j, n0 + gather[b][j]) for j in range(keep[b]) if (n0 + j) // page == p]
                now = torch.stack([scale[:, i]] + [scale[:, table[b][f // page]] for _, f in rows]).amax(0)
                got = [codes[:, table[b][f // page], :, f % page].double() * (scale[:, table[b][f // page]] / now)[..., None] for _, f in rows]
                whole = codes[:, i].double() * (scale[:, i] / now)[..., None, None]
                for (t, _), x in zip(rows, got):
                    whole[:, :, t % page] = x
                codes[:, i] = _nearest64(whole).float()
                scale[:, i] = now
    return {"k": k, "v": v, "k_scale": ks, "v_scale": vs, "len": torch.tensor([a + m for a, m in zip(lengths(c), keep)])}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "compact": _exact_compact}[case["op"]](s)
