"""The operators over a paged cache against a plain 64-bit implementation, and run together as a decode step runs them."""
import numpy as np
import pytest

from tests import attn_testlib as at

pytestmark = pytest.mark.gpu


def _ints(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _rounded(a, dtype):
    """A numpy array rounded to `dtype`, as a device tensor and in 64 bits."""
    import torch
    t = torch.from_numpy(a).cuda().to(at.torch_dtype(dtype))
    return t, t.double().cpu().numpy()


class Call:
    """Sequences with `lens` committed tokens and trees of `rows` nodes behind them in a paged cache."""

    def __init__(self, seed, lens, rows, h_q, h_kv, d, dtype="bf16", page=16, layout="token", chain=False, slack=0, spare_rows=0,
                 decode=False, q_gap=0, strides=0, max_rows=None):
        import torch
        import paper_2607_06763_b200 as gdn
        rng = np.random.default_rng(seed)
        self.gdn, self.lens, self.rows, self.d, self.dtype, self.decode = gdn, list(lens), list(rows), d, dtype, decode
        self.h_q, self.h_kv, self.scale = h_q, h_kv, d ** -0.5
        held = self.lens if decode else [a + b for a, b in zip(lens, rows)]
        self.held = held
        self.cache = at.Cache(rng, [n + slack for n in held], h_kv, d, page, dtype, layout, strides=strides)
        self.parents = [np.arange(n, dtype=np.int32) - 1 if chain else at.tree(rng, n) for n in rows]
        self.k64, self.v64 = [], []
        for b, n in enumerate(held):
            self.cache.write(b, rng.standard_normal((n, h_kv, d)), rng.standard_normal((n, h_kv, d)))
        self.N = sum(rows)
        q, q64 = _rounded(1.5 * rng.standard_normal((self.N + spare_rows, h_q, d)), dtype)
        self.q64 = q64[:self.N]
        if q_gap:   # rows inside a wider projection
            wide = torch.full((self.N + spare_rows, h_q * d + q_gap), float("nan"), dtype=q.dtype, device="cuda")
            wide[:, :h_q * d] = q.view(len(q), -1)
            q = wide
        self.q = q
        self.offsets = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.parent = None if chain else _ints(np.concatenate(self.parents + [np.full(spare_rows, 77, np.int32)]))
        self.seq_lens, self.row_offsets = _ints(lens), _ints(self.offsets)
        max_len = max(held + [1]) + slack
        self.shape = gdn.GdnAttnShape.from_cache(self.cache.k, self.cache.page_table, h_q, self.N + spare_rows,
                                                 max(list(rows) + [1]) if max_rows is None else max_rows, max_len=min(max_len, self.cache.max_pages * page),
                                                 q_stride=h_q * d + q_gap)
        self.o = torch.full((self.N + spare_rows, h_q, d), 7.0, dtype=at.torch_dtype(dtype), device="cuda")
        self.ws_bytes = gdn.gdn_attn_workspace_bytes(self.shape)
        assert self.ws_bytes > 0
        self.ws = torch.full((self.ws_bytes,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN patterns: nothing of it counts
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(self, stream=None):
        if self.decode:
            return self.gdn.gdn_attn_decode(self.shape, self.q, self.cache.k, self.cache.v, self.cache.page_table, self.seq_lens, self.o,
                                            self.ws, self.ws_bytes, self.status, stream)
        return self.gdn.gdn_attn_tree_verify(self.shape, self.q, self.cache.k, self.cache.v, self.cache.page_table, self.seq_lens,
                                             self.parent, self.row_offsets, self.o, self.ws, self.ws_bytes, self.status, stream)

    def device_status(self):
        import torch
        torch.cuda.synchronize()
        return int(self.status.item())

    def see(self, b):
        n, L = self.rows[b], self.lens[b]
        if self.decode:
            return np.ones((1, L), bool)
        return np.concatenate([np.ones((n, L), bool), at.ancestors(self.parents[b])], 1)

    def check(self, what="", only=None):
        got = self.o.double().cpu().numpy()
        worst = 0.0
        for b in range(len(self.lens)) if only is None else only:
            k, v = self.cache.read(b, self.held[b])
            rows = slice(int(self.offsets[b]), int(self.offsets[b + 1]))
            o, a, big = at.attend(self.q64[rows], k, v, self.see(b), self.scale)
            bound = at.allowed(o, a, big, self.dtype, self.d, self.held[b])
            assert np.array_equal(np.isfinite(got[rows]), np.isfinite(o)), f"{what}: finite in other places, sequence {b}"
            fine = np.isfinite(o)
            if fine.any():
                ratio = np.abs(got[rows] - o)[fine] / bound[fine]
                worst = max(worst, float(ratio.max()))
        assert (got[self.N:] == 7.0).all(), f"{what}: rows behind the last sequence were written"
        assert worst <= 1.0, f"{what}: {worst:.3f} of the allowed error"

    def verify(self, what=""):
        assert self.run() == 0
        assert self.device_status() == 0
        self.check(what)


HEADS = [(1, 1, 64), (4, 4, 128), (8, 2, 64), (8, 1, 128), (16, 1, 128), (12, 4, 128), (40, 2, 64), (6, 2, 40), (4, 4, 8), (14, 2, 96)]


@pytest.mark.parametrize("h_q,h_kv,d", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode(cuda_device, h_q, h_kv, d, dtype):
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 300, 1000]
    Call(1, lens, [1] * len(lens), h_q, h_kv, d, dtype, decode=True).verify()


@pytest.mark.parametrize("page,layout", [(1, "token"), (7, "head"), (16, "head"), (24, "token"), (64, "head"), (100, "token"), (512, "token")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_pages(cuda_device, page, layout, dtype):
    lens = [700, 3, 0, 128, 257, 64]
    Call(2, lens, [1] * 6, 8, 2, 128, dtype, page=page, layout=layout, slack=40, decode=True, q_gap=64, strides=16).verify()


@pytest.mark.parametrize("lens", [[5000], [0], [1], [33, 8000], [4097, 0, 1, 2, 3] * 30, [64] * 500], ids=str)
def test_decode_splits(cuda_device, lens):
    """One long sequence over all SMs, next to short ones, and more units than SMs."""
    Call(3, lens, [1] * len(lens), 8, 2, 64, page=32, decode=True).verify()


@pytest.mark.parametrize("rows", [[1], [2], [5, 0, 3], [16], [17], [31, 33], [64], [64, 1, 40], [65], [100, 64, 3], [200], [129, 0]], ids=str)
@pytest.mark.parametrize("h_q,h_kv,d,dtype", [(4, 4, 64, "bf16"), (8, 2, 128, "bf16"), (8, 1, 128, "bf16"), (6, 2, 40, "bf16"), (4, 2, 64, "f32")])
def test_trees(cuda_device, rows, h_q, h_kv, d, dtype):
    lens = [70, 0, 131][:len(rows)]
    Call(4, lens, rows, h_q, h_kv, d, dtype, spare_rows=3).verify()


@pytest.mark.parametrize("rows", [[1], [7, 0, 64], [65], [130, 250], [600]], ids=str)
@pytest.mark.parametrize("h_q,h_kv,d,dtype", [(4, 4, 64, "bf16"), (8, 2, 128, "bf16"), (4, 2, 128, "f32")])
def test_chunks_of_a_prompt(cuda_device, rows, h_q, h_kv, d, dtype):
    lens = [0, 200, 77][:len(rows)]
    Call(5, lens, rows, h_q, h_kv, d, dtype, chain=True, page=24, layout="head", spare_rows=2, q_gap=16).verify()


@pytest.mark.parametrize("lens,rows", [([1500, 0, 3000], [64, 64, 20]), ([900] * 20, [16] * 20), ([2500], [200]), ([6000], [3])], ids=str)
@pytest.mark.parametrize("h_q,h_kv,d", [(8, 2, 128), (8, 1, 64)])
def test_trees_behind_long_caches(cuda_device, lens, rows, h_q, h_kv, d):
    Call(6, lens, rows, h_q, h_kv, d, page=64, slack=100).verify()


@pytest.mark.parametrize("page,layout", [(1, "token"), (7, "head"), (8, "token"), (24, "head"), (100, "token"), (256, "head")])
@pytest.mark.parametrize("h_q,h_kv,d", [(8, 1, 128), (8, 1, 64), (2, 2, 128)])
def test_tree_pages(cuda_device, page, layout, h_q, h_kv, d):
    """Units of more than 64 rows by tensor copies (pages that a power of two from 8 on divides) and by rows."""
    Call(15, [300, 0, 65], [60, 64, 17], h_q, h_kv, d, page=page, layout=layout, strides=8, spare_rows=1).verify()
    Call(16, [300, 40], [90, 130], h_q, h_kv, d, page=page, layout=layout, chain=True).verify()


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("h_q,h_kv,d", [(80, 1, 64), (160, 1, 128), (300, 1, 64)])
def test_many_heads_share_one(cuda_device, decode, h_q, h_kv, d):
    lens = [0, 1, 127, 700]
    Call(17, lens, [1] * 4 if decode else [3, 1, 0, 2], h_q, h_kv, d, decode=decode).verify()


@pytest.mark.parametrize("scale", [0.0, -0.1, 1e-30])
@pytest.mark.parametrize("rows", [[5, 2], [70, 30]], ids=str)
def test_scales_that_hide_or_turn_the_order(cuda_device, scale, rows):
    c = Call(18, [90, 300], rows, 8, 2, 64)
    c.shape.scale = c.scale = scale
    c.verify()


def test_many_sequences_of_all_lengths(cuda_device):
    """More units than runs, of a tile to a hundred: runs over many units and units over many runs."""
    rng = np.random.default_rng(19)
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(9000), 60))]
    Call(20, lens, [1] * 60, 4, 2, 64, decode=True, page=64).verify()
    Call(21, lens, [int(x) for x in rng.integers(0, 20, 60)], 8, 2, 64, page=32).verify()
    Call(22, lens[:30], [int(x) for x in rng.integers(20, 64, 30)], 8, 2, 128, page=32).verify()


@pytest.mark.parametrize("chain", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_more_units_than_two_per_cta(cuda_device, chain, d):
    """Units that are not split: chunks and trees of many sequences, some without rows, one that is no tree."""
    rng = np.random.default_rng(24)
    lens = [int(x) for x in rng.integers(0, 200, 16)]
    rows = [int(x) for x in rng.integers(0, 90, 16)]
    rows[3], rows[5] = 0, 100
    c = Call(25, lens, rows, 32, 8, d, page=16, chain=chain, spare_rows=2)
    c.verify()
    if not chain:
        c.o.fill_(7.0)
        c.parent[int(c.offsets[5]) + 50] = 60
        assert c.run() == 0 and c.device_status() == -7
        c.check(only=[b for b in range(16) if b != 5])
        assert (c.o[int(c.offsets[5]):int(c.offsets[6])] == 7.0).all()


@pytest.mark.parametrize("h_q,h_kv,d,dtype", [(4, 4, 64, "bf16"), (8, 1, 128, "bf16"), (4, 2, 64, "f32")])
@pytest.mark.parametrize("rows", [[9], [40, 64], [150]], ids=str)
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")], ids=str)
def test_values_that_a_row_does_not_see(cuda_device, rows, h_q, h_kv, d, dtype, value):
    """Infinities and NaN in the keys and values of some nodes: rows that do not see them are what they are without them."""
    c = Call(7, [50, 20][:len(rows)], rows, h_q, h_kv, d, dtype)
    for b, n in enumerate(rows):
        k, v = c.cache.read(b, c.held[b])
        hit = [c.lens[b] + i for i in (n // 2, n - 1)]
        v[hit[0], :, ::3] = value
        v[hit[1]] = value
        if n > 20:
            k[c.lens[b] + n // 3] = value
        c.cache.write(b, k, v)
    c.verify(str(value))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores_and_equal_scores(cuda_device, dtype):
    """Scores of several hundred (the maximum moves far from tile to tile) and all-zero queries (every token weighs the same)."""
    c = Call(8, [600, 300], [20, 3], 8, 2, 64, dtype)
    c.q[:10] *= 60
    c.q[10:12] = 0
    c.q64 = c.q[:c.N].double().cpu().numpy().reshape(c.N, 8, 64)
    c.verify()


@pytest.mark.parametrize("decode", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_device_side_faults_are_reported(cuda_device, decode, dtype):
    """A sequence that cannot be: its rows are left alone, the others are right."""
    def call():
        rows = [1, 1, 1, 1] if decode else [8, 70, 3, 5]
        return Call(9, [100, 50, 20, 300], rows, 4, 2, 64, dtype, decode=decode, slack=20)
    for change, code in ((lambda c: c.seq_lens.__setitem__(1, -1), -12), (lambda c: c.seq_lens.__setitem__(1, c.shape.max_len + 1), -12)):
        c = call()
        change(c)
        assert c.run() == 0 and c.device_status() == code
        c.check("length", only=[0, 2, 3])
        assert (c.o[int(c.offsets[1]):int(c.offsets[2])] == 7.0).all()
    for bad_page in (-1, 1 << 30):
        c = call()
        c.cache.page_table[1, 0] = bad_page
        assert c.run() == 0 and c.device_status() == -12
        c.check("page", only=[0, 2, 3])
    if not decode:
        for node, parent in ((5, 5), (0, 0), (7, 60), (3, -2)):
            c = call()
            c.parent[node] = parent
            assert c.run() == 0 and c.device_status() == -7
            c.check("parent", only=[1, 2, 3])
            assert (c.o[:8] == 7.0).all()
        for at_, value in ((1, -3), (2, 1 << 30), (4, 1 << 20)):
            c = call()
            c.row_offsets[at_] = value
            assert c.run() == 0 and c.device_status() == -7


def test_small_trees_with_bad_parents(cuda_device):
    """Trees of at most 64 nodes are checked without a plan of their own."""
    c = Call(10, [500, 20, 700], [8, 60, 3], 4, 2, 64)
    c.parent[30] = 40
    assert c.run() == 0 and c.device_status() == -7
    c.check(only=[0, 2])
    assert (c.o[8:68] == 7.0).all()


def test_offsets_above_32_bits(cuda_device):
    """Pages so far apart that the elements between them do not fit 32 bits."""
    import torch
    import paper_2607_06763_b200 as gdn
    d, page, n_pages = 128, 16, 40
    apart = (1 << 32) // (n_pages - 2) // 8 * 8
    base = torch.empty(apart * (n_pages - 1) + page * d, dtype=torch.bfloat16, device="cuda")
    cache = base.as_strided((n_pages, page, 1, d), (apart, d, d, 1))
    torch.manual_seed(0)
    values = torch.randn(n_pages, page, 1, d, device="cuda").bfloat16()
    cache.copy_(values)
    table = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device="cuda")[None].contiguous()
    L = n_pages * page - 3
    q = torch.randn(1, 4, d, device="cuda").bfloat16()
    outs = []
    for c in (cache, values):
        s = gdn.GdnAttnShape.from_cache(c, table, 4, 1, 1)
        n = gdn.gdn_attn_workspace_bytes(s)
        o, ws, status = torch.zeros_like(q), torch.empty(n, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        assert gdn.gdn_attn_decode(s, q, c, c, table, _ints([L]), o, ws, n, status) == 0
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        outs.append(o)
    assert torch.equal(outs[0], outs[1]) and bool(outs[0].abs().sum() > 0)
    # a row behind them all, to the last page's place
    s = gdn.GdnAttnShape.from_cache(cache, table.flip(1).contiguous(), 4, 1, 1)
    k = torch.randn(1, 1, d, device="cuda").bfloat16()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert gdn.gdn_kv_append(s, None, k, k, None, 0, 0, 0, None, _ints([0, 1]), _ints([L]), table.flip(1).contiguous(), None, cache, cache, status) == 0
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and torch.equal(cache[n_pages - 1, L % page], k[0])


@pytest.mark.parametrize("decode", [True, False])
def test_captured_calls_follow_their_arrays(cuda_device, decode):
    """Two captured calls with a workspace between them, replayed after lengths, pages and trees have changed; and a call on a
    stream of its own."""
    import torch
    a = Call(11, [900, 40, 0], [1, 1, 1] if decode else [64, 10, 3], 8, 2, 128, decode=decode, slack=100)
    b = Call(12, [30, 300, 500], [1, 1, 1] if decode else [64, 64, 1], 8, 2, 128, decode=decode, slack=100)
    n = max(a.ws_bytes, b.ws_bytes)
    a.ws = b.ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    a.ws_bytes = b.ws_bytes = n
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert a.run(side) == 0 and b.run(side) == 0
    side.synchronize()
    a.check("stream")
    b.check("stream")
    graphs = []
    for c in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            assert c.run(torch.cuda.current_stream()) == 0
        graphs.append(g)
    for step in range(3):
        for c, g in zip((a, b), graphs):
            c.o.fill_(7.0)
            g.replay()
        for c in (a, b):
            assert c.device_status() == 0
            c.check(f"replay {step}")
            # shorter caches, other trees
            c.lens = [max(0, x - 13 * (step + 1)) for x in c.lens]
            if decode:
                c.held = c.lens
            else:
                rng = np.random.default_rng(step)
                c.parents = [at.tree(rng, len(p)) for p in c.parents]
                c.parent.copy_(_ints(np.concatenate(c.parents)))
                c.held = [x + r for x, r in zip(c.lens, c.rows)]
            c.seq_lens.copy_(_ints(c.lens))


def test_results_do_not_change_from_call_to_call(cuda_device):
    import torch
    for c in (Call(13, [3000, 100], [1, 1], 8, 2, 128, decode=True), Call(14, [2000, 50], [64, 30], 8, 2, 128), Call(14, [100], [20], 4, 2, 64, "f32")):
        outs = []
        for _ in range(4):
            assert c.run() == 0
            outs.append(c.o.clone())
        assert all(torch.equal(outs[0], o) for o in outs[1:])


# ---- rows into the cache


def _rope(n, rope_dim, seed=0):
    import torch
    angle = np.random.default_rng(seed).uniform(-3.0, 3.0, (n, max(rope_dim // 2, 1)))[:, :rope_dim // 2]
    t = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1)).float().cuda().contiguous()
    return t, t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h_q,h_kv,d,rope_dim,interleaved", [(8, 2, 128, 128, 0), (4, 4, 64, 32, 1), (8, 1, 128, 64, 0), (2, 2, 64, 0, 0), (6, 2, 40, 10, 0),
                                                            (6, 2, 40, 12, 1), (2, 1, 128, 96, 0), (3, 1, 8, 8, 1), (4, 2, 128, 8, 0)])
@pytest.mark.parametrize("chain", [True, False])
def test_append(cuda_device, dtype, h_q, h_kv, d, rope_dim, interleaved, chain):
    import torch
    import paper_2607_06763_b200 as gdn
    rng = np.random.default_rng(20)
    lens, rows = [0, 5, 100, 33, 7], [3, 0, 70, 64, 1]
    cache = at.Cache(rng, [a + b for a, b in zip(lens, rows)], h_kv, d, 24, dtype, "head" if chain else "token")
    held = []
    for b, n in enumerate(lens):
        kv = rng.standard_normal((2, n, h_kv, d))
        cache.write(b, kv[0], kv[1])
        held.append(cache.read(b, n))
    parents = [np.arange(n, dtype=np.int32) - 1 if chain else at.tree(rng, n) for n in rows]
    N = sum(rows)
    gap = 48
    wide, wide64 = _rounded(rng.standard_normal((N + 2, (h_q + 2 * h_kv) * d + gap)), dtype)
    stride = wide.stride(0)
    q, k, v = wide, wide[:, h_q * d:], wide[:, (h_q + h_kv) * d:]
    max_len = max(a + b for a, b in zip(lens, rows))
    rope, rope64 = _rope(max_len, rope_dim)
    shape = gdn.GdnAttnShape.from_cache(cache.k, cache.page_table, h_q, N + 2, max(rows), max_len=max_len, q_stride=stride, k_stride=stride, v_stride=stride)
    q_out = torch.full((N + 2, h_q, d), 7.0, dtype=wide.dtype, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    offsets = np.concatenate([[0], np.cumsum(rows)])
    rc = gdn.gdn_kv_append(shape, q, k, v, rope if rope_dim else None, max_len, rope_dim, interleaved, None if chain else _ints(np.concatenate(parents)),
                           _ints(offsets), _ints(lens), cache.page_table, q_out, cache.k, cache.v, status)
    torch.cuda.synchronize()
    assert rc == 0 and int(status.item()) == 0
    assert bool((q_out[N:] == 7.0).all())
    step = at.HALF_STEP[dtype]
    for b, n in enumerate(rows):
        r = slice(int(offsets[b]), int(offsets[b + 1]))
        pos = lens[b] + at.depths(parents[b])
        parts = [wide64[r, i * d:j * d].reshape(n, j - i, d) for i, j in ((0, h_q), (h_q, h_q + h_kv), (h_q + h_kv, h_q + 2 * h_kv))]
        got_k, got_v = cache.read(b, lens[b] + n)
        assert np.array_equal(got_k[:lens[b]], held[b][0]) and np.array_equal(got_v[:lens[b]], held[b][1])
        assert np.array_equal(got_v[lens[b]:], parts[2])
        for got, x in ((q_out[r].double().cpu().numpy(), parts[0]), (got_k[lens[b]:], parts[1])):
            want = at.rotated(x, pos, rope64, rope_dim, interleaved)
            # two products and a sum in fp32, at most 2^-24 of the products' sizes each; one rounding
            size = at.rotated(np.abs(x), pos, np.abs(rope64), rope_dim, interleaved)
            size = np.maximum(np.abs(size), np.abs(want)) + (np.abs(x).max(-1, keepdims=True) if rope_dim else 0.0)
            assert (np.abs(got - want) <= 3 * 2.0 ** -24 * size + step * 1.01 * np.abs(want)).all()
            assert np.array_equal(got[..., rope_dim:], x[..., rope_dim:])
    # what belongs to nobody is as it was
    used = np.zeros((cache.n_pages, cache.page), bool)
    for b in range(len(rows)):
        page, place = cache.places(b, lens[b] + rows[b])
        used[page, place] = True
    assert bool(torch.isnan(cache.k[torch.from_numpy(~used).cuda()]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("with_parents", [True, False])
def test_commit_writes_the_accepted_path(cuda_device, dtype, with_parents):
    """Over the nodes that append had put there; a broken path leaves its sequence alone."""
    import torch
    import paper_2607_06763_b200 as gdn
    rng = np.random.default_rng(21)
    lens, rows, h_kv, d, rope_dim = [0, 5, 100, 33, 7, 9], [3, 0, 70, 64, 1, 12], 2, 64, 64
    parents = [at.tree(rng, n) for n in rows]
    paths = [at.root_paths(p, rng) for p in parents]
    paths[2] = [x for x in range(70) if at.ancestors(parents[2])[69, x]]
    N = sum(rows)
    (k, k64), (v, v64) = _rounded(rng.standard_normal((N, h_kv, d)), dtype), _rounded(rng.standard_normal((N, h_kv, d)), dtype)
    max_len = 170
    rope, rope64 = _rope(max_len, rope_dim)
    offsets = np.concatenate([[0], np.cumsum(rows)])
    for broken in (False, True):
        cache = at.Cache(np.random.default_rng(1), [a + b for a, b in zip(lens, rows)], h_kv, d, 16, dtype)
        p = [list(x) for x in paths]
        if broken:
            p[5] = [0, 3, 2] if with_parents else [0, 2, 2]
            p[3] = [0, 64]
        shape = gdn.GdnAttnShape.from_cache(cache.k, cache.page_table, 4, N, max(rows), max_len=max_len)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        rc = gdn.gdn_kv_commit(shape, k, v, rope, max_len, rope_dim, 0, _ints(np.concatenate(parents)) if with_parents else None, _ints(offsets),
                               _ints(np.concatenate([np.array(x, np.int32) for x in p])), _ints(np.concatenate([[0], np.cumsum([len(x) for x in p])])),
                               _ints(lens), cache.page_table, cache.k, cache.v, status)
        torch.cuda.synchronize()
        assert rc == 0 and int(status.item()) == (-9 if broken else 0)
        for b, path in enumerate(p):
            got_k, got_v = cache.read(b, lens[b] + rows[b])
            n = 0 if broken and b in (3, 5) else len(path)
            assert np.isnan(got_k[:lens[b]]).all() and np.isnan(got_k[lens[b] + n:]).all() and np.isnan(got_v[lens[b] + n:]).all()
            if n:
                src = offsets[b] + np.array(path)
                assert np.array_equal(got_v[lens[b]:lens[b] + n], v64[src])
                want = at.rotated(k64[src], lens[b] + np.arange(n), rope64, rope_dim, 0)
                assert np.abs(got_k[lens[b]:lens[b] + n] - want).max() <= (at.HALF_STEP[dtype] + 2.0 ** -22) * np.abs(k64[src]).max() * 2


def test_append_in_place_and_faults(cuda_device):
    import torch
    import paper_2607_06763_b200 as gdn
    rng = np.random.default_rng(22)
    lens, rows, h_q, h_kv, d = [10, 20, 30], [4, 80, 2], 4, 2, 64
    N = sum(rows)
    parents = [at.tree(rng, n) for n in rows]
    offsets = np.concatenate([[0], np.cumsum(rows)])
    (q, _), (k, _), (v, _) = (_rounded(rng.standard_normal((N, h, d)), "bf16") for h in (h_q, h_kv, h_kv))
    rope, _ = _rope(128, 64)

    def run(cache, q_in, q_out, lens=lens, parents=parents):
        shape = gdn.GdnAttnShape.from_cache(cache.k, cache.page_table, h_q, N, max(rows), max_len=112)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        assert gdn.gdn_kv_append(shape, q_in, k, v, rope, 128, 64, 0, _ints(np.concatenate(parents)), _ints(offsets), _ints(lens),
                                 cache.page_table, q_out, cache.k, cache.v, status) == 0
        torch.cuda.synchronize()
        return int(status.item())

    def cache():
        return at.Cache(np.random.default_rng(1), [112] * 3, h_kv, d, 16, "bf16")

    a, b = cache(), cache()
    out, same = torch.zeros_like(q), q.clone()
    assert run(a, q, out) == 0 and run(b, same, same) == 0
    assert torch.equal(out, same) and torch.equal(torch.nan_to_num(a.k), torch.nan_to_num(b.k))
    c = cache()
    assert run(c, q, torch.zeros_like(q), lens=[10, -1, 30]) == -12 and run(c, q, torch.zeros_like(q), lens=[10, 40, 30]) == -12
    assert np.isnan(c.read(1, 112)[0]).all() and not np.isnan(c.read(2, 32)[0][30:]).any()
    c = cache()
    c.page_table[2, 1] = 1 << 20   # where rows 30, 31 of the last sequence would go
    out2 = torch.zeros_like(q)
    assert run(c, q, out2) == -12 and np.isnan(c.read(0, 112)[0]).sum() < 112 * h_kv * d
    for wrong in ([2, 4, 84, 86], [0, 4, 84, 1 << 20], [0, 84, 4, 86], [-5, 4, 84, 86], [0, 4, 84, 87]):
        c = cache()
        shape = gdn.GdnAttnShape.from_cache(c.k, c.page_table, h_q, N, max(rows), max_len=112)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out3 = torch.zeros_like(q)
        assert gdn.gdn_kv_append(shape, q, k, v, rope, 128, 64, 0, None, _ints(wrong), _ints(lens), c.page_table, out3, c.k, c.v, status) == 0
        assert gdn.gdn_kv_commit(shape, k, v, rope, 128, 64, 0, None, _ints(offsets), _ints([0] * 200), _ints(wrong), _ints(lens), c.page_table,
                                 c.k, c.v, status) == 0
        torch.cuda.synchronize()
        assert int(status.item()) in (-7, -9), wrong
    bad = [p.copy() for p in parents]
    bad[1][40] = 50
    c = cache()
    assert run(c, q, torch.zeros_like(q), parents=bad) == -7
    assert np.isnan(c.read(1, 61)[0][60]).all() and not np.isnan(c.read(1, 21)[0][20]).any()


def test_decode_steps_as_a_model_runs_them(cuda_device):
    """Prompt, then steps of: rows of a draft tree into the cache, the tree's attention, tokens at every node, the accepted path,
    its commit, the next length -- against the attention of the accepted tokens alone, computed densely in 64 bits."""
    import torch
    import paper_2607_06763_b200 as gdn
    rng = np.random.default_rng(30)
    B, h_q, h_kv, d, vocab, page = 3, 8, 2, 64, 50, 16
    embed = rng.standard_normal((vocab, (h_q + 2 * h_kv) * d))
    head = torch.from_numpy(rng.standard_normal((h_q * d, vocab))).float().cuda()
    rows_of, rows64 = _rounded(embed, "bf16")
    rope, rope64 = _rope(512, d)
    cache = at.Cache(rng, [400] * B, h_kv, d, page, "bf16")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tokens = [list(rng.integers(0, vocab, n)) for n in (1, 40, 100)]       # accepted so far
    seq_lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def forward(new, parents):
        """Rows of the tokens `new` [per sequence] into the cache and through the attention; (fused rows, outputs, shape, offsets)."""
        flat = np.concatenate(new).astype(np.int64)
        x = rows_of[torch.from_numpy(flat).cuda()].contiguous()
        n, w = len(flat), x.shape[1]
        offsets = _ints(np.concatenate([[0], np.cumsum([len(t) for t in new])]))
        shape = gdn.GdnAttnShape.from_cache(cache.k, cache.page_table, h_q, n, max(len(t) for t in new), q_stride=h_q * d, k_stride=w, v_stride=w)
        fused = gdn.GdnAttnShape.from_cache(cache.k, cache.page_table, h_q, n, max(len(t) for t in new), q_stride=w, k_stride=w, v_stride=w)
        par = None if parents is None else _ints(np.concatenate(parents))
        q = torch.empty(n, h_q, d, dtype=x.dtype, device="cuda")
        o = torch.empty_like(q)
        k, v = x[:, h_q * d:], x[:, (h_q + h_kv) * d:]
        assert gdn.gdn_kv_append(fused, x, k, v, rope, 512, d, 0, par, offsets, seq_lens, cache.page_table, q, cache.k, cache.v, status) == 0
        need = gdn.gdn_attn_workspace_bytes(shape)
        assert need <= ws.numel()
        assert gdn.gdn_attn_tree_verify(shape, q, cache.k, cache.v, cache.page_table, seq_lens, par, offsets, o, ws, ws.numel(), status) == 0
        return (fused, x, k, v, par, offsets), o

    def check_against_dense(b, o_row, history):
        """Outputs of the last of `history` at sequence b, whose tokens attend to one another as a plain sequence."""
        x = rows64[np.array(history)]
        n = len(x)
        pos = np.arange(n)
        round_ = lambda a: _rounded(a, "bf16")[1]
        q, k, v = (x[:, i * d:j * d].reshape(n, j - i, d) for i, j in ((0, h_q), (h_q, h_q + h_kv), (h_q + h_kv, h_q + 2 * h_kv)))
        q, k = round_(at.rotated(q, pos, rope64, d, 0)), round_(at.rotated(k, pos, rope64, d, 0))
        want, a, big = at.attend(q[-1:], k, v, np.ones((1, n), bool), d ** -0.5)
        # a rotated component next to a rounding border may fall on its other side: half a step more of query and key each
        bound = at.allowed(want, a, big, "bf16", d, n) + a * 4 * 2.0 ** -8 * big[..., None]
        assert (np.abs(o_row.double().cpu().numpy()[None] - want) <= bound).all()

    forward([t[:-1] for t in tokens], None)          # the prompts, as chunks; the last token is the first step's root
    seq_lens += _ints([len(t) - 1 for t in tokens])
    for step in range(4):
        parents = [np.concatenate([[-1], np.maximum(at.tree(rng, n), 0)]).astype(np.int32)[:n] for n in (9, 30, 64)]
        draft = [np.concatenate([[t[-1]], rng.integers(0, vocab, len(p) - 1)]) for t, p in zip(tokens, parents)]
        call, o = forward(draft, parents)
        logits = o.float().reshape(len(o), -1) @ head
        n = len(o)
        u = torch.rand(n, device="cuda")
        token = torch.full((n,), -9, dtype=torch.int32, device="cuda")
        prob = torch.empty(n, device="cuda")
        full = lambda x, dt=torch.float32: torch.full((n,), x, dtype=dt, device="cuda")
        assert gdn.gdn_sample(gdn.GdnSampleShape.from_logits(logits), logits, full(0.9), full(20, torch.int32), full(0.95), full(0.01), u, token,
                              prob, status) == 0
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        got, lg = token.cpu().numpy(), logits.double().cpu().numpy()
        for r in range(n):
            assert got[r] == at.sample(lg[r], float(u[r]), float(np.float32(0.9)), 20, float(np.float32(0.95)), float(np.float32(0.01)))[0]
        # the accepted path: from the root along children whose token was sampled at their parent (some accepted anyhow)
        fused, x, k, v, par, offsets = call
        paths, first = [], 0
        for b, p in enumerate(parents):
            path = [0]
            while True:
                kids = [c for c in range(len(p)) if p[c] == path[-1]]
                hit = [c for c in kids if draft[b][c] == got[first + path[-1]]] or (kids[:1] if rng.random() < 0.7 else [])
                if not hit:
                    break
                path.append(hit[0])
            check_against_dense(b, o[first + path[-1]], tokens[b][:-1] + [draft[b][i] for i in path])
            tokens[b] = tokens[b][:-1] + [int(draft[b][i]) for i in path] + [int(got[first + path[-1]])]
            paths.append(path)
            first += len(p)
        assert gdn.gdn_kv_commit(fused, k, v, rope, 512, d, 0, par, offsets, _ints(np.concatenate(paths)),
                                 _ints(np.concatenate([[0], np.cumsum([len(x) for x in paths])])), seq_lens, cache.page_table, cache.k, cache.v, status) == 0
        seq_lens += _ints([len(x) for x in paths])
    # one plain token behind it all, by the decode call
    x = rows_of[torch.tensor([t[-1] for t in tokens]).cuda()].contiguous()
    w = x.shape[1]
    shape = gdn.GdnAttnShape.from_cache(cache.k, cache.page_table, h_q, B, 1, q_stride=w, k_stride=w, v_stride=w)
    q, o = torch.empty(B, h_q, d, dtype=x.dtype, device="cuda"), torch.empty(B, h_q, d, dtype=x.dtype, device="cuda")
    assert gdn.gdn_kv_append(shape, x, x[:, h_q * d:], x[:, (h_q + h_kv) * d:], rope, 512, d, 0, None, _ints(np.arange(B + 1)), seq_lens, cache.page_table, q,
                             cache.k, cache.v, status) == 0
    seq_lens += 1
    shape.q_stride = h_q * d
    assert gdn.gdn_attn_decode(shape, q, cache.k, cache.v, cache.page_table, seq_lens, o, ws, ws.numel(), status) == 0
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for b in range(B):
        assert int(seq_lens[b]) == len(tokens[b])
        check_against_dense(b, o[b], tokens[b])


@pytest.mark.parametrize("h_q,h_kv,d,dtype", [(4, 4, 64, "bf16"), (8, 2, 128, "bf16"), (6, 2, 40, "bf16"), (4, 2, 64, "f32")])
@pytest.mark.parametrize("rows", [7, 64])
def test_bad_trees_between_good_ones(cuda_device, rows, h_q, h_kv, d, dtype):
    """Runs of many short units, every second of them of a tree that is none: what one unit's check of its tree says must not be
    taken for the next one's by any warp."""
    rng = np.random.default_rng(40)
    n = 300
    c = Call(41, [int(x) for x in rng.integers(0, 200, n)], [rows] * n, h_q, h_kv, d, dtype, slack=20)
    broken = [b for b in range(n) if b % 2 == 1 and b % 5 != 0]
    for b in broken:
        c.parent[int(c.offsets[b]) + rows - 1] = rows
    good = [b for b in range(n) if b not in broken]
    for _ in range(5):
        c.o.fill_(7.0)
        c.status.zero_()
        assert c.run() == 0 and c.device_status() == -7
    c.check(only=good[::7])
    first = c.o.clone()
    for b in broken:
        assert bool((first[int(c.offsets[b]):int(c.offsets[b + 1])] == 7.0).all())
    c.o.fill_(7.0)
    assert c.run() == 0 and c.device_status() == -7
    assert bool((first == c.o).all())


@pytest.mark.parametrize("h_q,h_kv,d,dtype,rows,chain", [(8, 1, 128, "bf16", 3, False), (8, 1, 64, "bf16", 8, True), (8, 1, 128, "bf16", 40, False),
                                                         (8, 1, 64, "bf16", 70, True), (2, 1, 128, "bf16", 200, True), (4, 2, 64, "f32", 5, False),
                                                         (4, 2, 40, "bf16", 20, True)])
@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")], ids=str)
def test_committed_keys_that_are_no_numbers(cuda_device, h_q, h_kv, d, dtype, rows, chain, value, many):
    """One component of one committed key, at each place modulo 16 of tiles that all rows see: a row whose score there is +inf or NaN
    is NaN (inf - inf, as in 64 bits), one whose score is -inf is what it is without the token.  In units that several runs share, and
    (many) in units of one run."""
    n, L, e = (320, 150, 5) if many else (17, 400, 5)
    lens = [L] * (n - 1) + [150 if many else 3000]
    c = Call(42, lens, [rows] * n, h_q, h_kv, d, dtype, chain=chain)
    at_ = [b % 128 for b in range(n)] if many else [129 + b if b % 2 else b for b in range(n - 1)] + [1500]
    clean = []
    for b in range(n):
        k, v = c.cache.read(b, c.held[b])
        clean.append((k.copy(), v))
        k[at_[b], :, e] = value
        c.cache.write(b, k, v)
    assert c.run() == 0 and c.device_status() == 0
    got = c.o.double().cpu().numpy()
    for b in range(n) if rows <= 8 and not many else range(40, 60) if rows <= 40 and many else range(0, n, n // 5):
        q = c.q64[c.offsets[b]:c.offsets[b + 1]]
        o = got[c.offsets[b]:c.offsets[b + 1]]
        gone = q[..., e] * value == -np.inf          # (nothing else is: a query's component is 0 nowhere)
        assert (np.isnan(o).all(-1) == ~gone).all() and (np.isfinite(o).all(-1) == gone).all(), b
        k, v = clean[b]
        see = c.see(b)
        see[:, at_[b]] = False
        want, a, big = at.attend(q, k, v, see, c.scale)
        assert (np.abs(o - want) <= at.allowed(want, a, big, dtype, d, c.held[b]))[gone].all(), b


@pytest.mark.parametrize("h_q,h_kv,d,dtype,rows", [(8, 1, 128, "bf16", 3), (8, 1, 128, "bf16", 40), (8, 1, 64, "bf16", 70), (4, 2, 64, "f32", 5),
                                                   (4, 2, 40, "bf16", 20)])
@pytest.mark.parametrize("n", [1, 150])
def test_rows_whose_scores_are_all_minus_infinity(cuda_device, h_q, h_kv, d, dtype, rows, n):
    """Zeros, as where a row sees nothing; where they are all +inf, NaN."""
    c = Call(43, [300, 0, 2000] if n == 1 else [140] * n, [rows] * (3 if n == 1 else n), h_q, h_kv, d, dtype)
    c.q[:, :, 7] = -1.0
    c.q[::3, :, 7] = 1.0
    for b in range(len(c.lens)):
        k, v = c.cache.read(b, c.held[b])
        k[..., 7] = -np.inf
        c.cache.write(b, k, v)
    assert c.run() == 0 and c.device_status() == 0
    got = c.o[:c.N].double().cpu().numpy()
    assert (got[::3] == 0.0).all()
    assert np.isnan(np.delete(got, np.arange(0, c.N, 3), 0)).all()
