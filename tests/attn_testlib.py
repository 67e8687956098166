"""Plain 64-bit forms of the operators over a paged cache and of the sampler, and the cases of their tests."""
from __future__ import annotations

import math

import numpy as np

# half a step of a rounding, relative to the value
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def torch_dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def tree(rng, n, reach=8):
    """Parents of a random topological tree (now and then a forest): a node hangs from one of the `reach` in front of it."""
    p = np.arange(n) - 1 - rng.integers(0, reach, n)
    return np.maximum(p, -1).astype(np.int32)


def depths(parent):
    out = np.zeros(len(parent), np.int64)
    for i, p in enumerate(parent):
        out[i] = 0 if p < 0 else out[p] + 1
    return out


def root_paths(parent, rng):
    """A root path of the tree, cut anywhere (possibly empty)."""
    if len(parent) == 0:
        return []
    node, chain = int(rng.integers(0, len(parent))), []
    while node >= 0:
        chain.append(node)
        node = int(parent[node])
    return chain[::-1][:int(rng.integers(0, len(chain) + 1))]


def ancestors(parent):
    n = len(parent)
    see = np.zeros((n, n), bool)
    for i, p in enumerate(parent):
        if p >= 0:
            see[i] = see[p]
        see[i, i] = True
    return see


def attend(q, k, v, see, scale):
    """q [n][h_q][d], k and v [L][h_kv][d], see [n][L] in 64 bits.  Returns the outputs, the same with |v|, and the largest sum of
    |q_i k_i| * scale of a seen token per row and head.  What a row does not see has no part in it, whatever its values."""
    n, h_q, d = q.shape
    G = h_q // k.shape[1] if k.shape[1] else 1
    o, a, big = np.zeros((n, h_q, d)), np.zeros((n, h_q, d)), np.zeros((n, h_q))
    for i in range(n):
        at = np.flatnonzero(see[i])
        if len(at) == 0:
            continue
        for h in range(h_q):
            kk, vv = k[at, h // G], v[at, h // G]
            with np.errstate(invalid="ignore"):
                s = kk @ q[i, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                o[i, h] = w @ vv
                a[i, h] = w @ np.abs(vv)
                big[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * abs(scale)
    return o, a, big


def allowed(o, a, big, dtype, d, n_tokens):
    """Bound of |got - o|.  A score is a sum of d products in fp32: off by at most (d + 2) 2^-24 of the sum of their absolute
    values, with scale, maximum and power another few steps of it; that much relative each weight is off, numerator and
    denominator, and the sums over the tokens another n 2^-24 each.  Where rows are bf16 the weights go into the second product
    as bf16, off by half a step each.  The result is rounded once."""
    score = (d + 8) * 2.0 ** -24 * big[..., None] + (n_tokens + 16) * 2.0 ** -24
    weight = 2 * score + (HALF_STEP["bf16"] if dtype == "bf16" else 0.0)
    return a * weight * 1.01 + np.abs(o) * HALF_STEP[dtype] * 1.01 + 1e-30


def rotated(x, pos, rope, rope_dim, interleaved):
    """x [n][heads][d] in 64 bits, turned by the table's rows."""
    y = x.copy()
    if rope_dim == 0:
        return y
    half = rope_dim // 2
    c, s = rope[pos, :half][:, None], rope[pos, half:rope_dim][:, None]
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


class Cache:
    """A paged cache with sequences of given capacity; pages in random order, what belongs to nobody is NaN."""

    def __init__(self, rng, capacity, h_kv, d, page, dtype, layout="token", max_pages=None, spare=2, strides=0):
        import torch
        self.page, self.dtype = page, dtype
        need = [-(-int(n) // page) for n in capacity]
        self.n_pages = sum(need) + spare
        self.max_pages = max(need + [1]) if max_pages is None else max_pages
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(need), self.max_pages), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        dims = (self.n_pages, page, h_kv) if layout == "token" else (self.n_pages, h_kv, page)
        def make():
            t = torch.full(dims + (d + strides,), float("nan"), dtype=torch_dtype(dtype), device="cuda")[..., :d]
            return t if layout == "token" else t.transpose(1, 2)
        self.k, self.v = make(), make()
        self.page_table = torch.from_numpy(self.table).cuda()

    def places(self, b, n):
        t = np.arange(n)
        return self.table[b, t // self.page].astype(np.int64), t % self.page

    def write(self, b, k, v):
        """Tokens 0 .. len(k) - 1 of sequence b (numpy, 64 bits), rounded to the cache's type."""
        import torch
        if len(k) == 0:
            return
        page, at = (torch.from_numpy(x).cuda() for x in self.places(b, len(k)))
        self.k[page, at] = torch.from_numpy(k).cuda().to(self.k.dtype)
        self.v[page, at] = torch.from_numpy(v).cuda().to(self.v.dtype)

    def read(self, b, n):
        import torch
        if n == 0:
            return (np.zeros((0,) + tuple(self.k.shape[2:])),) * 2
        page, at = (torch.from_numpy(x).cuda() for x in self.places(b, n))
        return self.k[page, at].double().cpu().numpy(), self.v[page, at].double().cpu().numpy()


def sample(x, u, T=1.0, k=0, p=1.0, m=0.0):
    """Token and probability of one row, in 64 bits."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    order = np.argsort(-x, kind="stable")
    top = x[order[0]]
    if top == -np.inf:
        return -1, 0.0
    if not T > 0:
        return int(order[0]), 1.0
    xs = x[order]
    with np.errstate(invalid="ignore"):
        w = np.where(xs == top, 1.0, np.exp((xs - top) / T) if math.isfinite(top) and math.isfinite(T) else
                     (np.where(xs > -np.inf, 1.0, 0.0) if math.isfinite(top) else 0.0))
    kept = np.arange(len(w)) < (k if 0 < k < len(w) else len(w))
    w = np.where(kept, w, 0.0)
    if p < 1.0:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        kept &= (before < p * w.sum()) | (np.arange(len(w)) == 0)
    kept &= w >= min(m, 1.0) if m > 0 else True
    kept &= w > 0
    mass = np.zeros(len(x))
    mass[order[kept]] = w[kept]
    total = np.cumsum(mass)
    at = int(np.flatnonzero((total > min(max(u, 0.0), 1.0) * total[-1]) & (mass > 0))[0]) if u < 1 else int(np.flatnonzero(mass > 0)[-1])
    return at, mass[at] / total[-1]
