"""Plain 64-bit forms of the cache operators (NumPy, sequence by sequence) and the inputs of their tests."""
from __future__ import annotations

import numpy as np
import torch

BIG = 448.0
CODES = np.array([(-1 if c >> 7 else 1) * ((c & 7) / 8 * 2.0 ** -6 if (c >> 3 & 15) == 0 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3 & 15) - 7))
                  if c & 127 != 127 else np.nan for c in range(256)])
_VALUES = CODES[:127]                                   # 0 ... 448, ascending


def nearest(x: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value of each x: ties to the even code, saturating, NaN stays."""
    m = np.minimum(np.abs(x), BIG)
    hi = np.clip(np.searchsorted(_VALUES, np.nan_to_num(m)), 1, 126)
    below, above = m - _VALUES[hi - 1], _VALUES[hi] - m
    take_low = (below < above) | ((below == above) & ((hi - 1) % 2 == 0))
    r = np.copysign(np.where(take_low, _VALUES[hi - 1], _VALUES[hi]), x)
    return np.where(np.isnan(x), np.nan, r)


def scale_for(amax: float) -> float:
    """The smallest power of two >= amax / 448, at least 2^-64."""
    if amax <= 0:
        return 2.0 ** -64
    m, e = np.frexp(amax / BIG)
    return max(2.0 ** -64, 2.0 ** (int(e) - (1 if m == 0.5 else 0)))


def f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().double().numpy()


def f8(t: torch.Tensor) -> np.ndarray:
    """Values of a float8 tensor, from its bytes."""
    return CODES[t.detach().cpu().view(torch.uint8).numpy()]


def turned(x, weight, eps, cs, rot, interleaved):
    """Norm and rotation of x [..., D]; cs [..., rot] cosines then sines."""
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    if rot == 0:
        return x
    x, h = x.copy(), rot // 2
    c, s = cs[..., :h], cs[..., h:]
    a, b = (x[..., 0:rot:2].copy(), x[..., 1:rot:2].copy()) if interleaved else (x[..., :h].copy(), x[..., h:rot].copy())
    p, q = a * c - b * s, b * c + a * s
    if interleaved:
        x[..., 0:rot:2], x[..., 1:rot:2] = p, q
    else:
        x[..., :h], x[..., h:rot] = p, q
    return x


def positions(step, b, tokens):
    """Positions of a sequence's step tokens; step: dict of NumPy arrays."""
    base = step["base"][b] if step["base"] is not None else step["len"][b]
    if step["pos"] is None:
        return base + np.arange(tokens)
    return np.concatenate([[base], step["pos"][b, :tokens - 1]]).astype(int)[:tokens]


def sees(step, b, tokens):
    """[tokens][tokens] truth values of who sees whom inside the step."""
    if step["mask"] is None:
        return np.tril(np.ones((tokens, tokens), bool))
    bits = np.unpackbits(np.ascontiguousarray(step["mask"][b]).view(np.uint8), axis=1, bitorder="little").astype(bool)
    see = np.eye(tokens, dtype=bool)
    see[:, 0] = True
    see[1:, 1:] |= bits[:tokens - 1, :tokens - 1]
    return see


def append(codes, scale, table, step, x, page):
    """One side of an append into values codes [pages][heads][page][D] and scale [pages][heads], in place.  x: [B][T][heads][D], turned."""
    for b in range(len(step["len"])):
        n0, m = int(step["len"][b]), int(step["nodes"][b]) + 1
        for p in range(n0 // page, (n0 + m - 1) // page + 1) if m > 0 else []:
            lo, hi, i = max(n0, p * page), min(n0 + m, (p + 1) * page), int(table[b, p])
            part = x[b, lo - n0:hi - n0]
            for h in range(codes.shape[1]):
                v = part[:, h]
                fin = np.abs(v[np.isfinite(v)])
                s = scale_for(fin.max() if fin.size else 0.0)
                if lo > p * page:
                    s = max(s, scale[i, h])
                    codes[i, h, :lo - p * page] = nearest(codes[i, h, :lo - p * page] * (scale[i, h] / s))
                scale[i, h] = s
                codes[i, h, lo - p * page:hi - p * page] = nearest(v / s)


def attend(k, v, ks, vs, table, step, q, scale, page):
    """(out, lse, sum of p |v|) of every token of every sequence; None where a sequence has none."""
    found = []
    g = q.shape[2] // k.shape[1]
    for b in range(len(step["len"])):
        n0, m = int(step["len"][b]), int(step["nodes"][b]) + 1
        if m <= 0:
            found.append(None)
            continue
        slots = np.arange(n0 + m)
        ids, rows = table[b, slots // page], slots % page
        see = np.concatenate([np.ones((m, n0), bool), sees(step, b, m)], 1)
        out, lse, mass = np.zeros((m,) + q.shape[2:]), np.zeros((m, q.shape[2])), np.zeros((m,) + q.shape[2:])
        for h in range(q.shape[2]):
            kk, vv = (t[ids, h // g, rows] * s[ids, h // g][:, None] for t, s in ((k, ks), (v, vs)))
            a = np.where(see, scale * (q[b, :m, h] @ kk.T), -np.inf)
            top = a.max(1, keepdims=True)
            e = np.exp(a - top)
            p = e / e.sum(1, keepdims=True)
            for i in range(m):                                     # only what is seen, so that NaN elsewhere stays out
                w = see[i]
                out[i, h] = p[i, w] @ vv[w]
                mass[i, h] = p[i, w] @ np.abs(vv[w])
            lse[:, h] = top[:, 0] + np.log(e.sum(1))
        found.append((out, lse, mass))
    return found


def compact(codes, scale, table, lens, gather, keep, page):
    """One side of a compaction of one layer, in place."""
    for b in range(len(lens)):
        n0 = int(lens[b])
        for p in range(n0 // page, (n0 + int(keep[b]) - 1) // page + 1) if keep[b] > 0 else []:
            i = int(table[b, p])
            moves = [(n0 + j - p * page, *divmod(n0 + int(gather[b, j]), page)) for j in range(int(keep[b])) if (n0 + j) // page == p]
            now = np.maximum(scale[i], np.max([scale[table[b, sp]] for _, sp, _ in moves], axis=0))
            got = [codes[table[b, sp], :, r] * (scale[table[b, sp]] / now)[:, None] for _, sp, r in moves]
            whole = codes[i] * (scale[i] / now)[:, None, None]
            for (to, _, _), x in zip(moves, got):
                whole[:, to] = x
            codes[i] = nearest(whole)
            scale[i] = now


# ---- inputs --------------------------------------------------------------------------------------------------------

def random_tree(rs, n, nodes, depth):
    """(mask words [n][W] int64, position offsets [n]) of a random tree in packed order."""
    level = np.sort(np.concatenate([np.arange(1, min(depth, nodes) + 1), rs.randint(1, max(2, depth + 1), max(0, nodes - depth))]))[:nodes]
    see = np.zeros((n, (n + 63) // 64 * 64), bool)
    off = np.zeros(n, np.int32)
    for i in range(nodes):
        before = np.flatnonzero(level[:i] == level[i] - 1)
        if len(before):
            see[i] = see[rs.choice(before)]
        see[i, i] = True
        off[i] = level[i]
    return np.packbits(see, axis=1, bitorder="little").view(np.int64), off


class Case:
    """Sizes and seeded inputs of a test: kv_len and nodes as lists, T the padded length of the step."""

    def __init__(self, lens, nodes, T, hq=4, hkv=2, D=64, page=16, dtype=torch.bfloat16, tree=True, layers=1, spare=3, seed=0):
        self.B, self.T, self.hq, self.hkv, self.D, self.page, self.dtype, self.layers = len(lens), T, hq, hkv, D, page, dtype, layers
        rs = self.rs = np.random.RandomState(seed)
        self.max_pages = max((max(l, 0) + max(x, 0)) // page + 1 for l, x in zip(lens, nodes)) + 1
        self.num_pages = self.B * self.max_pages + spare
        self.table = rs.permutation(self.num_pages)[:self.B * self.max_pages].astype(np.int32).reshape(self.B, self.max_pages)
        self.step = dict(len=np.array(lens, np.int32), nodes=np.array(nodes, np.int32), base=None, pos=None, mask=None)
        if tree and T > 1:
            trees = [random_tree(rs, T - 1, max(0, x), 5) for x in nodes]
            self.step["mask"] = np.stack([m for m, _ in trees])
            self.step["base"] = (self.step["len"] + rs.randint(0, 3, self.B)).astype(np.int32)
            self.step["pos"] = (self.step["base"][:, None] + np.stack([o for _, o in trees])).astype(np.int32)
        self.max_pos = int(max(lens)) + T + 8

    def rows(self, heads, spread=1.0, pad=0):
        """Random rows [B][T][heads][D] of the case's type on the device; pad: a larger buffer's slice, off a 16-byte boundary if odd."""
        x = torch.from_numpy(self.rs.standard_normal((self.B, self.T, heads, self.D)) * spread).to(self.dtype).cuda()
        if pad:
            big = torch.zeros((self.B, self.T + 1, heads, self.D + 8 + pad), dtype=self.dtype, device="cuda")
            view = big[:, 1:, :, pad:pad + self.D]
            view.copy_(x)
            return view
        return x

    def cache(self, spread=60.0, scales=(-8, -5)):
        """Random finite codes and power-of-two scales."""
        shape = (self.layers, self.num_pages, self.hkv, self.page, self.D)
        side = lambda: torch.from_numpy(np.clip(self.rs.standard_normal(shape) * spread, -BIG, BIG)).float().to(torch.float8_e4m3fn).cuda()  # noqa: E731
        sc = lambda: torch.from_numpy(2.0 ** self.rs.randint(scales[0], scales[1] + 1, shape[:3])).float().cuda()  # noqa: E731
        return side(), side(), sc(), sc(), torch.from_numpy(self.table).cuda()

    def handle(self, binding, **more):
        return binding.TreeKV(self.hq, self.hkv, self.D, self.page, self.num_pages, self.max_pages, self.B, self.T, layers=self.layers,
                              dtype=self.dtype, **more)

    def dev_step(self, binding):
        t = {k: None if v is None else torch.from_numpy(v).cuda() for k, v in self.step.items()}
        return binding.KVStep(t["len"], t["nodes"], t["base"], t["pos"], t["mask"])

    def cos_sin(self, rot, base=10000.0):
        angle = np.arange(self.max_pos)[:, None] * base ** (-np.arange(0, rot, 2) / rot)
        return torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1)).float().cuda()
