"""A batch of sequences over pages, and what its operators compute, in 64 bits on the CPU."""
from __future__ import annotations

import math

import numpy as np
import torch

DEV = "cuda:0"


def random_parents(rows, g, reach=6):
    """A tree's parents: every row hangs under one of the `reach` rows before it."""
    return [-1] + [int(torch.randint(max(0, v - reach), v, (1,), generator=g)) for v in range(1, rows)]


def lines_of(parent):
    """Rows on the way from every row up to the root, itself first."""
    out = []
    for v, p in enumerate(parent):
        out.append([v] + (out[p] if p >= 0 else []))
    return out


def mask_words(lines):
    words = []
    for line in lines:
        u = sum(1 << v for v in line)
        words.append([w - (1 << 64) if w >> 63 else w for w in ((u >> 64 * i) & ((1 << 64) - 1) for i in range(4))])
    return torch.tensor(words, dtype=torch.int64).reshape(-1, 4)


class Case:
    """Sequences with `lens` cached slots and `counts` rows each over scattered pages; what no sequence owns holds NaN."""

    def __init__(self, lens, counts, Hkv, hd, page, dtype, seed, trees=True, layers=None, spare_rows=0, last_pages=False, pool=None):
        self.g = g = torch.Generator().manual_seed(seed)
        self.lens, self.counts, self.page, self.dtype, self.Hkv, self.hd = list(lens), list(counts), page, dtype, Hkv, hd
        self.seqs, self.used = len(lens), sum(counts)
        self.rows = max(self.used, 1) + spare_rows
        need = [-(-(n + t) // page) for n, t in zip(lens, counts)]
        self.pool = pool or sum(need) + 2
        self.max_rows, self.max_len = max(max(counts), 1), max(lens)
        width = max(-(-(self.max_len + self.max_rows) // page), 1)
        order = (torch.arange(self.pool - sum(need), self.pool) if last_pages else torch.arange(self.pool))[torch.randperm(sum(need) if last_pages else self.pool, generator=g)]
        self.table = torch.full((self.seqs, width), -1, dtype=torch.int32)
        at = 0
        for b, w in enumerate(need):
            self.table[b, :w] = order[at:at + w].to(torch.int32)
            at += w
        self.starts = np.concatenate([[0], np.cumsum(self.counts)]).tolist()
        if trees:
            self.parents = [random_parents(t, g) if t else [] for t in counts]
        else:
            self.parents = [list(range(-1, t - 1)) for t in counts]
        self.lines = [lines_of(p) for p in self.parents]
        self.trees, self.layers = trees, layers

    def normal(self, *shape, sigma=1.0, mean=0.0):
        return (torch.randn(*shape, generator=self.g) * sigma + mean).to(self.dtype)

    def new_pools(self):
        """(k, v) pools with normal values in every slot that a sequence has, NaN elsewhere."""
        lead = () if self.layers is None else (self.layers,)
        out = []
        for _ in range(2):
            pool = torch.full(lead + (self.pool, self.Hkv, self.page, self.hd), float("nan"), dtype=self.dtype)
            for b in range(self.seqs):
                S = self.lens[b] + self.counts[b]
                if S:
                    page, row = self.where(b, range(S))
                    x = self.normal(S, *lead, self.Hkv, self.hd)
                    if self.layers is None:
                        pool[page, :, row] = x
                    else:
                        pool[:, page, :, row] = x
            out.append(pool)
        return out

    def where(self, b, slots):
        s = torch.as_tensor(list(slots), dtype=torch.long)
        return self.table[b].long()[s // self.page], s % self.page

    def depth(self):
        d = [len(line) - 1 for lines in self.lines for line in lines]
        return torch.tensor(d + [0] * (self.rows - self.used), dtype=torch.int32)

    def anc(self):
        a = torch.cat([mask_words(lines) for lines in self.lines if lines] + [torch.full((self.rows - self.used, 4), -1, dtype=torch.int64)])
        return a

    def flat_parents(self):
        return torch.tensor([p for t in self.parents for p in t] + [7] * (self.rows - self.used), dtype=torch.int32)

    def batch(self, B, pools, **bounds):
        start = torch.tensor(self.starts, dtype=torch.int32, device=DEV)
        length = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        return B.PagedBatch(start, length, self.table.to(DEV), pools[0], pools[1], bounds.get("rows", self.rows),
                            bounds.get("max_rows", self.max_rows), bounds.get("max_len", self.max_len))

    def slots(self, pool, b):
        """[slots, Hkv, hd] of sequence b in 64 bits (pages that are none: NaN)."""
        S = self.lens[b] + self.counts[b]
        page, row = self.where(b, range(S))
        ok = (page >= 0) & (page < self.pool)
        x = pool.cpu()[page.clamp(0, self.pool - 1), :, row].double()
        x[~ok] = float("nan")
        return x, ok


def attention(case, q, k_pool, v_pool, anc=True, scale=None, masks=None):
    """(out, sum of p |v|, largest sum |q k| scale of a row) [used rows, Hq, hd] in 64 bits.  masks: rows x 256 truth values in
    place of the trees."""
    Hq, hd = q.shape[1], q.shape[2]
    G = Hq // case.Hkv
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    out = torch.zeros(case.used, Hq, hd, dtype=torch.float64)
    weight, size = torch.zeros_like(out), torch.zeros(case.used, Hq, 1, dtype=torch.float64)
    qd = q.double().cpu()
    for b in range(case.seqs):
        n, t, at = case.lens[b], case.counts[b], case.starts[b]
        if not t:
            continue
        k, ok = case.slots(k_pool, b)
        v, _ = case.slots(v_pool, b)
        seen = torch.zeros(t, n + t, dtype=torch.bool)
        seen[:, :n] = True
        for r in range(t):
            if masks is not None:
                seen[r, n:] = masks[at + r, :t]
            else:
                seen[r, [n + u for u in case.lines[b][r]]] = True
        seen &= ok[None, :]
        for h in range(Hq):
            for r in range(t):
                j = seen[r].nonzero()[:, 0]
                if not len(j):
                    continue
                kk, vv = k[j, h // G], v[j, h // G]
                z = kk @ qd[at + r, h] * scale
                p = torch.softmax(z, dim=0)
                out[at + r, h] = p @ vv
                weight[at + r, h] = p @ vv.abs()
                size[at + r, h, 0] = ((kk.abs() @ qd[at + r, h].abs()) * scale).max()
    return out, weight, size


def attention_bound(case, out, weight, size):
    """What the operator may be off by.  float32: the scores' sums (hd + 4 roundings of terms that add up to `size`), which the softmax
    turns into twice their relative error, and the sums over the keys.  bf16 adds the rounding of the result and of the
    probabilities, half a step (2^-8) each, and what lags behind in the reference point does not matter (a factor)."""
    keys = max(n + t for n, t in zip(case.lens, case.counts))
    f32 = (2.0 * (case.hd + 4) * size + keys + 32) * 2.0 ** -24 * weight
    if case.dtype == torch.float32:
        return f32 + 1e-30
    return f32 + 2.0 ** -8 * (out.abs() + 1.01 * weight) + 1e-30


def turned(x, gain, eps, pos, rot, interleaved, freq, amplitude):
    """[rows, heads, hd] in 64 bits: the norm of the head and the rotation; and a bound on each entry's size before rounding."""
    y = x.double().cpu()
    if gain is not None:
        y = y / (y.square().mean(2, keepdim=True) + eps).sqrt() * gain.double().cpu()
    half = rot // 2
    lo = torch.arange(half) * (2 if interleaved else 1)
    hi = lo + (1 if interleaved else half)
    t = pos.double().cpu()[:, None, None] * freq.double().cpu()
    a, b = y[..., lo], y[..., hi]
    z, size = y.clone(), y.abs()
    z[..., lo] = amplitude * (a * torch.cos(t) - b * torch.sin(t))
    z[..., hi] = amplitude * (b * torch.cos(t) + a * torch.sin(t))
    size[..., lo] = size[..., hi] = amplitude * (a.abs() + b.abs())
    return z, size


def accept(parent, tokens, answers, max_path):
    path = [0]
    while len(path) < max_path:
        kids = [u for u in range(len(parent)) if u > path[-1] and parent[u] == path[-1] and tokens[u] == answers[path[-1]]]
        if not kids:
            break
        path.append(kids[0])
    return path


def sample(z, u, T=1.0, k=0, p=1.0, mp=0.0):
    """(token, log share) of one row in 64 bits; and how near u is to a border of the running sums, relative to their total."""
    x = np.asarray(z, dtype=np.float64).copy()
    x[np.isnan(x)] = -np.inf
    if x.max() == -np.inf:
        return -1, -np.inf, 1.0
    if not T > 0:
        return int(np.argmax(x)), 0.0, 1.0
    if x.max() == np.inf:
        x = np.where(x == np.inf, 0.0, -np.inf)
    with np.errstate(all="ignore"):
        e = np.where(x == -np.inf, 0.0, np.where(x == x.max(), 1.0, np.exp((x - x.max()) / np.float64(T))))
    left = np.argsort(-x, kind="stable")
    left = left[:int((x > -np.inf).sum())]
    if k > 0:
        left = left[:k]
    if p < 1:
        mass = np.cumsum(e[left])
        left = left[:int(np.searchsorted(mass, max(p, 0.0) * mass[-1], side="left")) + 1]
    if mp > 0:
        left = left[e[left] >= min(mp, 1.0)]
    left = np.sort(left)
    mass = np.cumsum(e[left])
    target = max(u, 0.0) * mass[-1] if u == u else 0.0
    at = int(np.searchsorted(mass, target, side="right"))
    some = left[e[left] > 0]
    if at >= len(left):
        at = int(np.searchsorted(left, some[-1]))
    near = float(np.abs(mass - target).min() / mass[-1])
    return int(left[at]), float(np.log(e[left[at]] / mass[-1])), near
