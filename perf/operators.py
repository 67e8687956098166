"""The operators that a decode step of a hybrid model needs next to its GDN layers, for measuring and comparing them.

    append   gdn_kv_append / gdn_kv_commit: new rows' keys rotated by position and written, with their values, to a paged
             cache; the queries rotated on the way (append), or the rows of an accepted path alone (commit)
    decode   gdn_attn_decode: attention of one new token per sequence over its pages
    tree     gdn_attn_tree_verify: attention of the nodes of a draft tree, or of a prompt chunk, over pages
    sample   gdn_sample: tokens from logits by temperature, top-k, top-p and min-p, from given random numbers

A case is a dict of plain values:

    op            one of the above
    dtype         bf16 | f32, of rows, cache and outputs (sample: of the logits)
    n_seq         sequences; lo..hi: tokens in the cache before the call (decode: the new one included), per sequence
    rows_lo, rows_hi   rows of the call per sequence (append, tree)
    parents       tree: a draft tree | chain: rows follow one another (a prompt, a linear draft)
    commit        append: the rows of an accepted path of the tree are written, nothing else
    h_q, h_kv, d  heads and components;  page: tokens of a page;  layout: token | head, the outer one inside a page
    rope_dim, interleaved   components that are rotated, and how they pair up
    rows, vocab, filters    sample: rows, tokens, and which filters are set: all | top_p | top_k | none | greedy
    sizes         seed of the ragged sizes

Lengths, head counts and tree sizes are those of the benchmark configurations of ``synth`` (trees of up to 64 to 256
nodes, 128 components, 32 heads) and generic serving ones.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def _attn(name, op, n_seq, lo, hi, rows_lo=1, rows_hi=1, parents="chain", commit=False, dtype="bf16", h_q=32, h_kv=8, d=128,
          page=16, layout="token", rope_dim=0, interleaved=False, sizes=1):
    c = dict(op=op, dtype=dtype, n_seq=n_seq, lo=lo, hi=hi, rows_lo=rows_lo, rows_hi=rows_hi, parents=parents, commit=commit,
             h_q=h_q, h_kv=h_kv, d=d, page=page, layout=layout, rope_dim=rope_dim, interleaved=interleaved, sizes=sizes)
    return dict(c, name=name) if name else c


def _sample(name, rows, vocab, filters, dtype="f32"):
    c = dict(op="sample", rows=rows, vocab=vocab, filters=filters, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new token of one sequence: the cost of a call
        _attn("append_b1", "append", 1, 1000, 1000, rope_dim=128),
        # the accepted paths of a serving batch of 64-node trees
        _attn("append_commit_b64", "append", 64, 100, 4000, 32, 64, parents="tree", commit=True, rope_dim=64, sizes=2),
        # prompts of a batch going into the cache
        _attn("append_prompts_b16", "append", 16, 0, 0, 500, 2000, rope_dim=128, page=32, layout="head", sizes=3),
        # one sequence shortly behind its prompt: latency
        _attn("decode_b1_short", "decode", 1, 700, 700),
        # one sequence with a long context: the split over its length
        _attn("decode_b1_long", "decode", 1, 131000, 131000, page=64, layout="head"),
        # a serving batch with lengths of all sizes
        _attn("decode_b64_ragged", "decode", 64, 1, 9000, sizes=4),
        # an accuracy run in fp32 on a small batch, smaller heads
        _attn("decode_b8_f32", "decode", 8, 100, 3000, dtype="f32", h_q=16, h_kv=4, d=64, sizes=5),
        # the 64-node tree of one sequence (the headline tree) at a full-attention layer
        _attn("tree_b1_T64", "tree", 1, 4000, 4000, 64, 64, parents="tree"),
        # trees of a serving batch, pages of an odd size
        _attn("tree_b32_ragged", "tree", 32, 300, 6000, 5, 64, parents="tree", page=24, sizes=6),
        # a prompt chunk behind a cached prefix: bound by the products
        _attn("chunk_b2_T2000", "tree", 2, 1000, 3000, 1900, 2047, page=64, layout="head", sizes=7),
        # the next token of one sequence
        _sample("sample_b1", 1, 50000, "all"),
        # the target tokens at the nodes of a tree batch, large vocabulary
        _sample("sample_b256_top_p", 256, 131071, "top_p"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above (at most the work of the largest listed one of its operator and type)."""
    while True:
        op = rng.choice(["append", "decode", "decode", "tree", "tree", "sample", "sample"])
        if op == "sample":
            c = _sample(None, _log(rng, 1, 256), _log(rng, 1000, 131071), rng.choice(["all", "top_p", "top_k", "none", "greedy"]),
                        rng.choice(["f32", "f32", "bf16"]))
            return c
        h_kv = rng.choice([1, 2, 4, 8])
        heads = dict(h_kv=h_kv, h_q=h_kv * rng.choice([1, 2, 4, 8]), d=rng.choice([64, 128, 128]), page=rng.choice([16, 16, 24, 32, 64, 128]),
                     layout=rng.choice(["token", "head"]), sizes=rng.randrange(1, 1 << 20))
        if op == "append":
            parents = rng.choice(["chain", "tree"])
            hi = _log(rng, 1, 64 if parents == "tree" else 2000)
            c = _attn(None, op, _log(rng, 1, 64), 0, _log(rng, 1, 4000), _log(rng, 1, hi), hi, parents=parents,
                      commit=parents == "tree" and rng.random() < 0.5, dtype=rng.choice(["bf16", "bf16", "f32"]),
                      rope_dim=rng.choice([0, 32, 64]), interleaved=rng.random() < 0.3, **heads)
            most = 1.0e9
        elif op == "decode":
            dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
            hi = _log(rng, 1, 131000 if dtype == "bf16" else 9000)
            c = _attn(None, op, _log(rng, 1, 64), _log(rng, 1, hi), hi, dtype=dtype, **heads)
            most = 1.3e9 if dtype == "bf16" else 1e8
        else:
            dtype = rng.choice(["bf16", "bf16", "bf16", "bf16", "f32"])
            parents = rng.choice(["tree", "tree", "chain"])
            hi = _log(rng, 2, 256 if parents == "tree" else 2000) if dtype == "bf16" else _log(rng, 2, 32)
            c = _attn(None, op, _log(rng, 1, 32), 0, _log(rng, 1, 8000), _log(rng, 1, hi), hi, parents=parents, dtype=dtype, **heads)
            most = 1.3e9 if dtype == "bf16" else 1e8
        w = work(c)
        # the plain form holds its weights for every pair of a row and a token of the longest sequence
        pairs = c["n_seq"] * c["h_q"] * c["rows_hi"] * (c["hi"] + c["rows_hi"])
        if 256 <= w["bytes"] <= most and w["flops"] <= 1.2e11 and (op == "append" or pairs <= 9e8) and c["n_seq"] * c["hi"] * c["h_kv"] * c["d"] <= 1.5e9:
            return c


def _sizes(c):
    """Lengths before the call and rows of the call, per sequence (numpy)."""
    rng = np.random.default_rng(c["sizes"])
    lens = rng.integers(c["lo"], c["hi"] + 1, c["n_seq"])
    rows = rng.integers(c["rows_lo"], c["rows_hi"] + 1, c["n_seq"])
    return lens, rows


def _path_sizes(c, rows):
    """Nodes of the accepted path that are written, per sequence: at most the depth of a tree that grows as _parents() grows it."""
    return np.array([len(p) for p in _paths(c, rows)])


def _parents(c, rows):
    """Parents of every tree, local to it: a node hangs from one of the eight in front of it, the first from the root."""
    rng = np.random.default_rng(c["sizes"] + 1)
    out = []
    for n in rows:
        p = np.arange(n) - 1 - (rng.integers(0, 8, n) if c["parents"] == "tree" else 0)
        p[1:] = np.maximum(p[1:], 0)
        if n:
            p[0] = -1
        out.append(p.astype(np.int32))
    return out


def _paths(c, rows):
    """An accepted path of every tree, root first: from nothing to a whole root path."""
    rng = np.random.default_rng(c["sizes"] + 2)
    out = []
    for p in _parents(c, rows):
        chain, node = [], int(rng.integers(0, len(p)))
        while node >= 0:
            chain.append(node)
            node = int(p[node])
        chain = chain[::-1][:16]
        out.append(chain[:int(rng.integers(0, len(chain) + 1))])
    return out


def _offsets(sizes):
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def ints(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    if c["op"] == "sample":
        n, V = c["rows"], c["vocab"]
        logits = 2.2 * randn(n, V)
        likely = torch.randint(0, V, (n, 16), generator=g, device="cuda")
        logits.scatter_add_(1, likely, 4.0 + 3.0 * randn(n, 16))   # a few tokens stand out, as after training
        u = torch.rand(n, generator=g, device="cuda")
        r = torch.rand(3, n, generator=g, device="cuda")
        on = {"all": (1, 1, 1), "top_p": (0, 1, 0), "top_k": (1, 0, 0), "none": (0, 0, 0), "greedy": (0, 0, 0)}[c["filters"]]
        greedy = c["filters"] == "greedy"
        return dict(case=c, logits=logits.to(_TORCH[c["dtype"]]), uniform=u,
                    temperature=torch.zeros_like(u) if greedy else 0.6 + 0.7 * r[0],
                    top_k=(1 + 200 * r[1]).int() if on[0] else torch.zeros_like(u).int(),
                    top_p=0.7 + 0.29 * r[2] if on[1] else torch.ones_like(u),
                    min_p=0.05 * r[0] if on[2] else torch.zeros_like(u),
                    token=torch.full((n,), -2, dtype=torch.int32, device="cuda"), prob=torch.zeros_like(u),
                    status=torch.zeros(1, dtype=torch.int32, device="cuda"))

    dt = _TORCH[c["dtype"]]
    lens, rows = _sizes(c)
    if c["op"] == "decode":
        rows = np.ones_like(lens)
        held = lens
    else:
        held = lens + rows
    pages = -(-held // c["page"])
    n_pages, max_pages = int(pages.sum()) + 3, int(max(pages.max(), 1))
    order = np.random.default_rng(seed).permutation(n_pages)
    table = np.full((c["n_seq"], max_pages), -1, np.int32)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    dims = (n_pages, c["page"], c["h_kv"], c["d"]) if c["layout"] == "token" else (n_pages, c["h_kv"], c["page"], c["d"])
    k_cache, v_cache = randn(*dims).to(dt), randn(*dims).to(dt)
    if c["layout"] == "head":   # always seen as [page][token][head][component]
        k_cache, v_cache = k_cache.transpose(1, 2), v_cache.transpose(1, 2)
    N = int(rows.sum())
    state = dict(case=c, k_cache=k_cache, v_cache=v_cache, page_table=ints(table), seq_lens=ints(lens), row_offsets=ints(_offsets(rows)),
                 q=(1.5 * randn(N, c["h_q"], c["d"])).to(dt), max_len=int(held.max()), max_rows=int(max(rows.max(), 1)),
                 parent=ints(np.concatenate(_parents(c, rows))) if c["parents"] == "tree" else None,
                 out=torch.zeros(N, c["h_q"], c["d"], dtype=dt, device="cuda"),
                 status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if c["op"] == "append":
        state.update(k=randn(N, c["h_kv"], c["d"]).to(dt), v=randn(N, c["h_kv"], c["d"]).to(dt))
        half = c["rope_dim"] // 2
        angle = torch.arange(state["max_len"], device="cuda", dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / max(half, 1))
        state["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
        if c["commit"]:
            paths = _paths(c, rows)
            state["path"] = ints(np.concatenate([np.zeros(0, np.int32)] + [np.array(p, np.int32) for p in paths] + [np.zeros(1, np.int32)]))
            state["path_offsets"] = ints(_offsets([len(p) for p in paths]))
    return state


def _shape(s):
    """The shape argument and the workspace, which a program makes once."""
    import paper_2607_06763_b200 as gdn
    c = s["case"]
    shape = gdn.GdnAttnShape.from_cache(s["k_cache"], s["page_table"], h_q=c["h_q"], total_rows=s["q"].shape[0], max_rows=s["max_rows"],
                                        max_len=s["max_len"], scale=c["d"] ** -0.5)
    n = gdn.gdn_attn_workspace_bytes(shape)
    s["own"] = (gdn, shape, torch.empty(max(n, 256), dtype=torch.uint8, device="cuda"), n)


def _run_own(s):
    c = s["case"]
    if c["op"] == "sample":
        import paper_2607_06763_b200 as gdn
        if "own" not in s:
            s["own"] = gdn.GdnSampleShape.from_logits(s["logits"])
        gdn.gdn_sample(s["own"], s["logits"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["uniform"], s["token"], s["prob"],
                       s["status"], torch.cuda.current_stream())
        return {"token": s["token"], "prob": s["prob"]}
    if "own" not in s:
        _shape(s)
    gdn, shape, ws, n = s["own"]
    stream = torch.cuda.current_stream()
    if c["op"] == "append" and c["commit"]:
        gdn.gdn_kv_commit(shape, s["k"], s["v"], s["rope"], s["rope"].shape[0], c["rope_dim"], c["interleaved"], s["parent"],
                          s["row_offsets"], s["path"], s["path_offsets"], s["seq_lens"], s["page_table"], s["k_cache"], s["v_cache"],
                          s["status"], stream)
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if c["op"] == "append":
        gdn.gdn_kv_append(shape, s["q"], s["k"], s["v"], s["rope"], s["rope"].shape[0], c["rope_dim"], c["interleaved"], s["parent"],
                          s["row_offsets"], s["seq_lens"], s["page_table"], s["out"], s["k_cache"], s["v_cache"], s["status"], stream)
        return {"q": s["out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if c["op"] == "decode":
        gdn.gdn_attn_decode(shape, s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["seq_lens"], s["out"], ws, n, s["status"], stream)
    else:
        gdn.gdn_attn_tree_verify(shape, s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["seq_lens"], s["parent"], s["row_offsets"],
                                 s["out"], ws, n, s["status"], stream)
    return s["out"]


def _row_places(s):
    """For every packed row: its sequence, and its place among the sequence's rows."""
    rows = torch.arange(s["q"].shape[0], device="cuda")
    off = s["row_offsets"].long()
    seq = torch.searchsorted(off[1:], rows, right=True)
    return seq, rows - off[seq]


def _ancestors(s, seq, local):
    """[n_seq][T][T] truth values: node j is on the root path of node i (i itself included)."""
    B, T = s["case"]["n_seq"], s["max_rows"]
    if s["parent"] is None:
        return torch.ones(T, T, dtype=torch.bool, device="cuda").tril().expand(B, T, T)
    parent = s["parent"].long()
    child = parent >= 0
    edge = torch.zeros(B, T, T, dtype=torch.float64, device="cuda")
    edge[seq[child], local[child], parent[child]] = 1.0
    eye = torch.eye(T, dtype=torch.float64, device="cuda").expand(B, T, T)
    # 1 + E + E^2 + ... of the edges: every root path once
    return torch.linalg.solve_triangular(eye - edge, eye, upper=False, unitriangular=True) > 0.5


def _rotated(x, cos, sin, rope_dim, interleaved):
    """x [n][heads][d] in fp32 with the first rope_dim components turned."""
    if rope_dim == 0:
        return x
    y = x.clone()
    a, b = (x[..., 0:rope_dim:2], x[..., 1:rope_dim:2]) if interleaved else (x[..., :rope_dim // 2], x[..., rope_dim // 2:rope_dim])
    cos, sin = cos[:, None], sin[:, None]
    if interleaved:
        y[..., 0:rope_dim:2], y[..., 1:rope_dim:2] = a * cos - b * sin, b * cos + a * sin
    else:
        y[..., :rope_dim // 2], y[..., rope_dim // 2:rope_dim] = a * cos - b * sin, b * cos + a * sin
    return y


def _plain_append(s):
    c = s["case"]
    seq, local = _row_places(s)
    lens, R = s["seq_lens"].long(), c["rope_dim"]
    if c["commit"]:
        off = s["path_offsets"].long()
        n = s["path"].shape[0] - 1
        place = torch.arange(n, device="cuda")
        seq = torch.searchsorted(off[1:], place, right=True)
        step = place - off[seq]
        src = s["row_offsets"].long()[seq] + s["path"][:n].long()
        slot = pos = lens[seq] + step
    else:
        src = torch.arange(s["q"].shape[0], device="cuda")
        slot = lens[seq] + local
        pos = slot if s["parent"] is None else lens[seq] + _ancestors(s, seq, local).sum(-1)[seq, local] - 1
    cos, sin = s["rope"][pos, :R // 2], s["rope"][pos, R // 2:]
    page = s["page_table"][seq, slot // c["page"]].long()
    s["k_cache"][page, slot % c["page"]] = _rotated(s["k"][src].float(), cos, sin, R, c["interleaved"]).to(s["k_cache"].dtype)
    s["v_cache"][page, slot % c["page"]] = s["v"][src]
    if c["commit"]:
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    s["out"].copy_(_rotated(s["q"].float(), cos, sin, R, c["interleaved"]))
    return {"q": s["out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attention(s):
    c = s["case"]
    B, T, L, H = c["n_seq"], s["max_rows"], s["max_len"], c["h_kv"]
    G = c["h_q"] // H
    lens = s["seq_lens"].long()
    tok = torch.arange(L, device="cuda")
    page = s["page_table"][:, tok // c["page"]].long().clamp_min(0)
    held = lens if c["op"] == "decode" else lens + (s["row_offsets"][1:] - s["row_offsets"][:-1])
    there = (tok[None] < held[:, None])[..., None, None]
    k = torch.where(there, s["k_cache"][page, tok % c["page"]].float(), 0.0)
    v = torch.where(there, s["v_cache"][page, tok % c["page"]].float(), 0.0)
    seq, local = _row_places(s)
    q = torch.zeros(B, T, c["h_q"], c["d"], device="cuda")
    q[seq, local] = s["q"].float()
    score = torch.einsum("bthgd,blhd->bhgtl", q.view(B, T, H, G, c["d"]), k) * c["d"] ** -0.5
    seen = (tok[None] < lens[:, None])[:, None].expand(B, T, L)
    if c["op"] == "tree":
        node = tok[None] - lens[:, None]                       # of a cached token: which row of the call it is
        anc = _ancestors(s, seq, local).gather(2, node.clamp(0, T - 1)[:, None].expand(B, T, L))
        seen = seen | (anc & (node >= 0)[:, None] & (node < T)[:, None])
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = (score - torch.where(top > -math.inf, top, 0.0)).exp()
    total = weight.sum(-1, keepdim=True)
    o = torch.einsum("bhgtl,blhd->bthgd", weight / torch.where(total > 0, total, 1.0), v)
    s["out"].copy_(o.reshape(B, T, c["h_q"], c["d"])[seq, local])
    return s["out"]


def _plain_sample(s):
    """In 64 bits: a token next to the border of a filter or of its interval must fall on the same side everywhere."""
    x = s["logits"].double()
    n, V = x.shape
    T = s["temperature"].double()[:, None]
    top = x.amax(1, keepdim=True)
    w = ((x - top) / torch.where(T > 0, T, 1.0)).exp()
    order = torch.sort(x, dim=1, descending=True, stable=True)[1]      # ties: the lowest index first
    sorted_w = w.gather(1, order)
    rank = torch.arange(V, device="cuda")[None]
    k = s["top_k"].long()[:, None]
    sorted_w = torch.where((rank < k) | (k <= 0), sorted_w, 0.0)
    before = sorted_w.cumsum(1) - sorted_w
    p, total = s["top_p"].double()[:, None], sorted_w.sum(1, keepdim=True)
    keep = ((before < p * total) | (p >= 1.0)) & (sorted_w >= s["min_p"].double()[:, None]) & (sorted_w > 0)
    keep = torch.where(T > 0, keep, rank == 0)
    w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, sorted_w, 0.0))
    mass = w.cumsum(1)
    token = ((mass > s["uniform"].double()[:, None] * mass[:, -1:]) & (w > 0)).to(torch.uint8).argmax(1)
    s["token"].copy_(token)
    s["prob"].copy_((w.gather(1, token[:, None]) / mass[:, -1:])[:, 0])
    return {"token": s["token"], "prob": s["prob"]}


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    return _plain_append(state) if op == "append" else _plain_sample(state) if op == "sample" else _plain_attention(state)


def work(case):
    c = case
    if c["op"] == "sample":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * _BYTES[c["dtype"]] + c["rows"] * 28, "flops": 4 * n}
    lens, rows = _sizes(c)
    size, H, G, d = _BYTES[c["dtype"]], c["h_kv"], c["h_q"] // c["h_kv"], c["d"]
    if c["op"] == "append":
        n = int((_path_sizes(c, rows) if c["commit"] else rows).sum())
        heads = 2 * H + (0 if c["commit"] else c["h_q"])
        turned = H + (0 if c["commit"] else c["h_q"])
        return {"bytes": n * (2 * heads * d * size + 4 * c["rope_dim"] + 8), "flops": 3 * n * turned * c["rope_dim"]}
    if c["op"] == "decode":
        held, rows, pairs = lens, np.ones_like(lens), int(lens.sum())
    else:
        held = lens + rows
        own_pairs = rows * (rows + 1) // 2 if c["parents"] == "chain" else \
            np.array([sum(_depths(p)) for p in _parents(c, rows)])
        pairs = int((lens * rows + own_pairs).sum())
    n_pages = int((-(-held // c["page"])).sum())
    return {"bytes": int(held.sum()) * 2 * H * d * size + int(rows.sum()) * 2 * c["h_q"] * d * size + 4 * (n_pages + int(rows.sum()) + 2 * c["n_seq"]),
            "flops": 4 * pairs * H * G * d}


def _depths(parent):
    depth = []
    for p in parent:
        depth.append(1 + (depth[p] if p >= 0 else 0))
    return depth


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "sample":
        return _exact_sample(s)
    lens, rows = _sizes(c)
    if c["op"] == "append":
        return _exact_append(s, lens, rows)
    if work(case)["flops"] > 1e12:
        return None
    rows = np.ones_like(lens) if c["op"] == "decode" else rows
    parents = _parents(c, rows)
    table = s["page_table"].cpu().numpy()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    G, first = c["h_q"] // c["h_kv"], 0
    for b in range(c["n_seq"]):
        n, L = int(rows[b]), int(lens[b])
        held = L if c["op"] == "decode" else L + n
        if held == 0:
            first += n
            continue
        pages = torch.from_numpy(table[b, :-(-held // c["page"])].astype(np.int64)).cuda()
        see = np.zeros((n, held), bool)
        see[:, :L] = True
        if c["op"] == "tree" and c["parents"] == "chain":
            see[:, L:] = np.tri(n, dtype=bool)
        elif c["op"] == "tree":
            for i, p in enumerate(parents[b]):
                if p >= 0:
                    see[i, L:] = see[p, L:]
                see[i, L + i] = True
        hidden = torch.from_numpy(~see).cuda()
        for h in range(c["h_kv"]):
            k = s["k_cache"][pages][:, :, h].reshape(-1, c["d"])[:held].double()
            v = s["v_cache"][pages][:, :, h].reshape(-1, c["d"])[:held].double()
            for g in range(G):
                z = (s["q"][first:first + n, h * G + g].double() @ k.T / math.sqrt(c["d"])).masked_fill(hidden, -math.inf)
                out[first:first + n, h * G + g] = torch.softmax(z, 1) @ v
        first += n
    return out


def _exact_append(s, lens, rows):
    c = s["case"]
    table = s["page_table"].cpu().numpy()
    R, half = c["rope_dim"], c["rope_dim"] // 2
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    src, slot, pos, seq = [], [], [], []
    first = 0
    for b, (n, parent, path) in enumerate(zip(rows, _parents(c, rows), _paths(c, rows))):
        nodes = path if c["commit"] else range(n)
        depth = range(len(path)) if c["commit"] else [x - 1 for x in _depths(parent)]
        for t, node in enumerate(nodes):
            src.append(first + node)
            slot.append(lens[b] + t)
            pos.append(lens[b] + depth[t])
            seq.append(b)
        first += n
    src, slot, pos, seq = (np.array(a, np.int64) for a in (src, slot, pos, seq))
    page, at = (torch.from_numpy(a.astype(np.int64)).cuda() for a in (table[seq, slot // c["page"]], slot % c["page"]))
    place = torch.from_numpy(pos).cuda()
    # the pair (a, b) as a + ib, times the table's cos + i sin
    turn = torch.complex(s["rope"][place, :half].double(), s["rope"][place, half:].double())[:, None]

    def turned(x):
        x = x.double()
        if R == 0:
            return x
        head = x[..., :R]
        pair = head.unflatten(-1, (half, 2)) if c["interleaved"] else torch.stack([head[..., :half], head[..., half:]], -1)
        y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        y = y.flatten(-2) if c["interleaved"] else torch.cat([y[..., 0], y[..., 1]], -1)
        return torch.cat([y, x[..., R:]], -1)

    src = torch.from_numpy(src).cuda()
    k_cache[page, at] = turned(s["k"][src])
    v_cache[page, at] = s["v"][src].double()
    out = {"k_cache": k_cache, "v_cache": v_cache}
    return out if c["commit"] else {"q": turned(s["q"]), **out}


def _exact_sample(s):
    x = s["logits"].double().cpu().numpy()
    u, T, k, p, m = (s[n].double().cpu().numpy() for n in ("uniform", "temperature", "top_k", "top_p", "min_p"))
    token, prob = np.zeros(len(x), np.int32), np.zeros(len(x))
    for r, row in enumerate(x):
        order = np.argsort(-row, kind="stable")
        if T[r] <= 0:
            token[r], prob[r] = order[0], 1.0
            continue
        w = np.exp((row[order] - row[order[0]]) / T[r])
        kept = np.arange(len(w)) < (k[r] if k[r] > 0 else len(w))
        w = np.where(kept, w, 0.0)
        if p[r] < 1.0:
            kept &= np.concatenate([[0.0], np.cumsum(w)[:-1]]) < p[r] * w.sum()
        kept &= w >= m[r]
        chosen = np.sort(order[kept])
        mass = np.exp((row[chosen] - row[order[0]]) / T[r])
        total = np.cumsum(mass)
        at = min(int(np.searchsorted(total, u[r] * total[-1], side="right")), len(chosen) - 1)
        token[r], prob[r] = chosen[at], mass[at] / total[-1]
    return {"token": torch.from_numpy(token), "prob": torch.from_numpy(prob)}
