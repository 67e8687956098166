"""What the calls over a paged cache and the sampler refuse, and the size of their workspace.  No kernel is launched here."""
import ctypes
import os
import re

import pytest

import paper_2607_06763_b200 as gdn
from paper_2607_06763_b200 import build

A = 1 << 20   # an address that is aligned for everything; nothing is read there
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build_library()
    return gdn.load_library()


def shape(**kw):
    s = gdn.GdnAttnShape(4, 32, 8, 128, 1, 64, 16, 100, 16, 64, 1000, 0.088, 16 * 8 * 128, 8 * 128, 128, 32 * 128, 8 * 128, 8 * 128)
    for k, v in kw.items():
        assert hasattr(s, k)
        setattr(s, k, v)
    return s


def decode(s, q=A, k=A, v=A, table=A, lens=A, o=A, ws=A, n=1 << 40, status=A):
    return gdn.gdn_attn_decode(s, q, k, v, table, lens, o, ws, n, status)


def tree(s, q=A, k=A, v=A, table=A, lens=A, parent=A, offsets=A, o=A, ws=A, n=1 << 40, status=A):
    return gdn.gdn_attn_tree_verify(s, q, k, v, table, lens, parent, offsets, o, ws, n, status)


def append(s, q=A, k=A, v=A, rope=A, rope_len=1000, rope_dim=64, parent=A, offsets=A, lens=A, table=A, q_out=2 * A, kc=A, vc=A, status=A):
    return gdn.gdn_kv_append(s, q, k, v, rope, rope_len, rope_dim, 0, parent, offsets, lens, table, q_out, kc, vc, status)


def commit(s, k=A, v=A, rope=A, rope_len=1000, rope_dim=64, parent=A, offsets=A, path=A, path_offsets=A, lens=A, table=A, kc=A, vc=A, status=A):
    return gdn.gdn_kv_commit(s, k, v, rope, rope_len, rope_dim, 0, parent, offsets, path, path_offsets, lens, table, kc, vc, status)


@pytest.mark.parametrize("name,pattern", [("GdnAttnShape", "gdn_attn_shape"), ("GdnSampleShape", "gdn_sample_shape")])
def test_struct_matches_header(name, pattern):
    text = open(os.path.join(ROOT, "include", "gdn_tree.h")).read()
    body = re.search(r"typedef struct %s \{(.*?)\} %s_t;" % (pattern, pattern), text, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields = [(t, f.strip()) for t, names in re.findall(r"(int32_t|int64_t|float)\s+([^;]+);", body) for f in names.split(",")]
    kinds = {"int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float}
    assert [(f, kinds[t]) for t, f in fields] == [(f, t) for f, t in getattr(gdn, name)._fields_]


BAD = [(dict(dtype=2), -3), (dict(n_seq=-1), -2), (dict(h_q=30), -2), (dict(h_kv=0), -2), (dict(h_q=0), -2), (dict(d=4), -2),
       (dict(d=132), -2), (dict(d=136), -2), (dict(total_rows=-1), -2), (dict(max_rows=0), -2), (dict(n_pages=0), -2), (dict(page_size=0), -2),
       (dict(max_pages=0), -2), (dict(max_len=0), -2), (dict(max_len=1025), -2), (dict(scale=float("nan")), -2), (dict(page_stride=-8), -2),
       (dict(token_stride=1028), -2), (dict(head_stride=130), -2), (dict(q_stride=4088), -2), (dict(q_stride=4100), -2), (dict(k_stride=1016), -2),
       (dict(v_stride=1028), -2)]


@pytest.mark.parametrize("change,code", BAD, ids=[str(c) for c, _ in BAD])
def test_bad_shapes_are_refused(change, code):
    s = shape(**change)
    assert tree(s) == code and append(s) == code and commit(s) == code
    assert gdn.gdn_attn_workspace_bytes(s) == 0


def test_missing_and_misaligned_pointers_are_refused():
    d = shape(max_rows=1, total_rows=4)
    for name in ("q", "k", "v", "table", "lens", "o", "status"):
        assert decode(d, **{name: None}) == -1, name
        assert decode(d, **{name: A + 2}) == -4, name
    for name in ("q", "k", "v", "table", "lens", "offsets", "o", "status"):
        assert tree(shape(), **{name: None}) == -1, name
        assert tree(shape(), **{name: A + 2}) == -4, name
    for call, names in ((append, ("k", "v", "rope", "offsets", "lens", "table", "kc", "vc", "status", "q_out", "q")),
                        (commit, ("k", "v", "rope", "offsets", "path", "path_offsets", "lens", "table", "kc", "vc", "status"))):
        for name in names:
            assert call(shape(), **{name: None}) == -1, name
            assert call(shape(), **{name: A + 2}) == -4, name
    for name in ("q", "k", "v", "o"):
        assert decode(d, **{name: A + 8}) == -4
    assert decode(d, ws=A + 16) == -4 and decode(d, ws=None) == -10
    need = gdn.gdn_attn_workspace_bytes(d)
    assert need % 256 == 0 and decode(d, n=need - 1) == -10


def test_sizes_that_do_not_go_together_are_refused():
    assert decode(shape()) == -2                                      # more than one row of a sequence
    assert decode(shape(max_rows=1, total_rows=5)) == -2
    assert tree(shape(max_rows=4097, total_rows=5000)) == -2          # a tree; a chunk may be longer:
    assert append(shape(), rope_len=999) == -2 and append(shape(), rope_dim=63) == -2 and append(shape(), rope_dim=130) == -2
    assert append(shape(q_stride=32 * 128 + 8), q_out=A) == -2        # in place, rows apart


def test_empty_calls_return_at_once():
    s = shape(n_seq=0, total_rows=0)
    assert gdn.gdn_attn_tree_verify(s, *[None] * 9, 0, None) == 0
    assert gdn.gdn_kv_commit(s, None, None, None, 1000, 64, 0, *[None] * 9) == 0
    assert gdn.gdn_attn_decode(shape(n_seq=0, total_rows=0, max_rows=1), *[None] * 7, 0, None) == 0
    assert gdn.gdn_sample(gdn.GdnSampleShape(0, 100, 0, 0, 100), *[None] * 9) == 0


def test_workspace_follows_the_shape():
    one = gdn.gdn_attn_workspace_bytes(shape(max_rows=1, total_rows=4))
    assert one > 0
    assert gdn.gdn_attn_workspace_bytes(shape(max_rows=1, total_rows=4, max_len=8)) <= 256 * 2
    big = shape(max_rows=200, total_rows=800)
    assert gdn.gdn_attn_workspace_bytes(big) >= 800 * 7 * 4           # ancestors of trees above 64 nodes


def test_sampler_refusals():
    def call(s, logits=A, uniform=A, token=A, status=A, T=A):
        return gdn.gdn_sample(s, logits, T, A, A, A, uniform, token, A, status)
    ok = (8, 1000, 0, 0, 1000)
    for i, v, code in ((0, -1, -2), (1, 0, -2), (1, (1 << 18) + 1, -2), (2, 2, -3), (4, 999, -2)):
        s = gdn.GdnSampleShape(*[v if i == j else x for j, x in enumerate(ok)])
        if i == 1 and v > 0:
            s.row_stride = v
        assert call(s) == code
    s = gdn.GdnSampleShape(*ok)
    for name in ("logits", "uniform", "token", "status"):
        assert call(s, **{name: None}) == -1
        assert call(s, **{name: A + 1}) == -4
    assert call(s, T=A + 2) == -4


def test_shapes_of_the_other_calls_are_refused():
    for wrong in (gdn.GdnShape(), gdn.GdnSampleShape(), None, 5):
        with pytest.raises(TypeError, match="GdnAttnShape"):
            decode(wrong)
    with pytest.raises(TypeError, match="GdnSampleShape"):
        gdn.gdn_sample(shape(), A, A, A, A, A, A, A, A, A)
    with pytest.raises(TypeError, match="GdnShape"):
        gdn.gdn_tree_verify_static(shape(), *[A] * 10)


def test_shapes_from_tensors():
    import torch
    cache = torch.zeros(7, 2, 16, 64).transpose(1, 2)
    s = gdn.GdnAttnShape.from_cache(cache, torch.zeros(3, 5, dtype=torch.int32), h_q=8, total_rows=3, max_rows=1)
    assert (s.n_seq, s.h_q, s.h_kv, s.d, s.dtype, s.n_pages, s.page_size, s.max_pages, s.max_len) == (3, 8, 2, 64, 0, 7, 16, 5, 80)
    assert (s.page_stride, s.token_stride, s.head_stride, s.q_stride) == (2048, 64, 1024, 512) and abs(s.scale - 0.125) < 1e-7
    with pytest.raises(ValueError):
        gdn.GdnAttnShape.from_cache(cache.transpose(2, 3), torch.zeros(3, 5), 8, 3, 1)
    with pytest.raises(ValueError):
        gdn.GdnAttnShape.from_cache(cache.half(), torch.zeros(3, 5), 8, 3, 1)
    x = torch.zeros(4, 10, dtype=torch.bfloat16)[:, :7]
    s = gdn.GdnSampleShape.from_logits(x)
    assert (s.n_rows, s.vocab, s.dtype, s.row_stride) == (4, 7, 1, 10)
    with pytest.raises(ValueError):
        gdn.GdnSampleShape.from_logits(x.T)


def test_tensors_that_do_not_fit_the_shape_are_refused():
    import torch
    table, lens = torch.zeros(3, 5, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    cache = torch.zeros(7, 16, 2, 64)
    wide = torch.zeros(9, (8 + 2 * 2) * 64 + 16)
    make = lambda **kw: gdn.GdnAttnShape.from_cache(kw.pop("k_cache", cache), kw.pop("table", table), 8, 9, 4, **kw)
    s = make(v_cache=cache.clone(), q=wide, k=wide[:, 8 * 64:], v=wide[:, 10 * 64:], seq_lens=lens)
    assert (s.q_stride, s.k_stride, s.v_stride) == (784, 784, 784)
    s = make(q=wide[:, :8 * 64].view(9, 8, 64), k=torch.zeros(9, 2, 64), v=wide[:1, 10 * 64:])
    assert (s.q_stride, s.k_stride, s.v_stride) == (784, 128, 128)
    assert make(q=wide[:1], q_stride=784).q_stride == 784
    for wrong in (dict(v_cache=torch.zeros(7, 2, 16, 64).transpose(1, 2)), dict(v_cache=cache.bfloat16()), dict(v_cache=cache[:6]),
                  dict(table=table.long()), dict(table=torch.zeros(3, 9, dtype=torch.int32)[:, :5]), dict(table=table[0]),
                  dict(seq_lens=lens.long()), dict(seq_lens=lens[:2]), dict(seq_lens=torch.zeros(6, dtype=torch.int32)[::2]),
                  dict(q=wide.bfloat16()), dict(q=wide, q_stride=512), dict(q=torch.zeros(9, 8, 128)[..., :64]), dict(q=torch.zeros(9, 4, 64)),
                  dict(k=wide[:, ::2]), dict(k=wide[:, 11 * 64:11 * 64 + 64]), dict(v=torch.zeros(9, 2, 2, 64))):
        with pytest.raises(ValueError):
            make(**wrong)
