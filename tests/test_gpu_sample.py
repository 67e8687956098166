"""The sampler against a plain 64-bit implementation: the same token everywhere, its probability to fp32."""
import numpy as np
import pytest

from tests import attn_testlib as at

pytestmark = pytest.mark.gpu


def _check(x, u, T=None, k=None, p=None, m=None, stride=0, first=0):
    """x: [rows][vocab] fp32 or bf16 tensor on the device; the parameters per row, or None."""
    import torch
    import paper_2607_06763_b200 as gdn
    n, vocab = x.shape
    if stride or first:
        wide = torch.full((n * (vocab + stride) + first + 8,), float("inf"), dtype=x.dtype, device="cuda")
        view = wide.as_strided((n, vocab), (vocab + stride, 1), first)
        view.copy_(x)
        x = view
    dev = lambda a, dt=torch.float32: None if a is None else torch.as_tensor(np.asarray(a), dtype=dt).cuda().contiguous()
    uu, TT, kk, pp, mm = dev(u), dev(T), dev(k, torch.int32), dev(p), dev(m)
    token = torch.full((n + 1,), -9, dtype=torch.int32, device="cuda")
    prob = torch.full((n + 1,), -9.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    shape = gdn.GdnSampleShape.from_logits(x)
    assert gdn.gdn_sample(shape, x, TT, kk, pp, mm, uu, token, prob, status) == 0
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and int(token[n]) == -9 and float(prob[n]) == -9.0
    got, gp, rows = token.cpu().numpy(), prob.cpu().numpy(), x.double().cpu().numpy()
    host = lambda t, r, off: off if t is None else float(t[r])
    for r in range(n):
        want, wp = at.sample(rows[r], float(uu[r]), host(TT, r, 1.0), int(host(kk, r, 0)), host(pp, r, 1.0), host(mm, r, 0.0))
        assert got[r] == want, (r, got[r], want)
        # weights are formed to 1e-9 of themselves and summed exactly; the quotient is rounded to fp32
        assert abs(gp[r] - wp) <= (2.0 ** -24 + 1e-8) * wp + 1e-12, (r, gp[r], wp)
    again = torch.empty_like(token)
    assert gdn.gdn_sample(shape, x, TT, kk, pp, mm, uu, again, None, status) == 0   # without probabilities
    assert torch.equal(again[:n], token[:n])


def _logits(seed, n, vocab, dtype="f32", spread=2.2):
    import torch
    rng = np.random.default_rng(seed)
    x = spread * rng.standard_normal((n, vocab))
    return torch.from_numpy(x).cuda().to(at.torch_dtype(dtype)), rng


@pytest.mark.parametrize("vocab", [1, 2, 31, 100, 4095, 4097, 8193, 33333, 131071])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_filters(cuda_device, vocab, dtype):
    n = 12
    x, rng = _logits(vocab, n, vocab, dtype)
    u, T = rng.random(n), rng.uniform(0.3, 1.5, n)
    k = rng.integers(1, min(vocab, 300) + 1, n)
    p, m = rng.uniform(0.3, 0.999, n), rng.uniform(0.0, 0.1, n)
    _check(x, u)
    _check(x, u, T)
    _check(x, u, T, k)
    _check(x, u, T, None, p)
    _check(x, u, T, None, None, m)
    _check(x, u, T, k, p)
    _check(x, u, T, k, p, m)
    _check(x, u, np.where(np.arange(n) % 3 == 0, 0.0, T), np.where(np.arange(n) % 4 == 0, 0, k), np.where(np.arange(n) % 5 == 0, 1.0, p), m)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("stride,first", [(0, 1), (1, 0), (3, 5), (8, 3)])
def test_rows_that_lie_apart(cuda_device, dtype, stride, first):
    x, rng = _logits(5, 7, 5003, dtype)
    _check(x, rng.random(7), None, [40] * 7, [0.9] * 7, stride=stride, first=first)


def test_many_rows(cuda_device):
    for n, vocab in ((700, 700), (300, 9000), (150, 20000)):
        x, rng = _logits(n, n, vocab)
        _check(x, rng.random(n), rng.uniform(0.5, 1.2, n), rng.integers(0, 60, n), rng.uniform(0.5, 1.05, n))


@pytest.mark.parametrize("vocab", [10, 3000, 40000, 131071])
def test_equal_logits(cuda_device, vocab):
    """All equal, two values, and a few values: prefixes end inside ties, lowest index first."""
    import torch
    rng = np.random.default_rng(1)
    n = 8
    u = rng.random(n)
    flat = torch.full((n, vocab), 1.25, device="cuda")
    some = torch.from_numpy(rng.integers(0, 5, (n, vocab))).float().cuda()
    two = torch.where(torch.rand(n, vocab, device="cuda") < 0.5, 1.0, 1.01)
    for x in (flat, some, two):
        _check(x, u)
        _check(x, u, None, [1, 2, 7, vocab - 1, vocab, vocab // 2 + 1, max(1, vocab // 3), 5])
        _check(x, u, None, None, [0.0, 1e-9, 0.25, 0.5, 0.9, 0.999, 1.0, -1.0])
        _check(x, u, [0.5] * n, [vocab // 2 + 1] * n, [0.3, 0.5, 0.7, 0.75, 0.8, 0.85, 0.9, 0.95])
        _check(x, u, [0.0] * n)


def test_values_that_are_no_numbers(cuda_device):
    import torch
    inf, nan = float("inf"), float("nan")
    rng = np.random.default_rng(2)
    x = torch.from_numpy(rng.standard_normal((10, 6000))).float().cuda()
    x[0] = -inf
    x[1] = nan
    x[2, ::2] = -inf
    x[3, 5] = nan
    x[4, [7, 4000]] = inf
    x[5] = -inf
    x[5, 5999] = -3.0
    x[6, 100:5000] = nan
    x[7] = torch.finfo(torch.float32).min
    x[8, 1:] = torch.finfo(torch.float32).min
    x[9] *= 1e30
    u = rng.random(10)
    for T in (None, [1.0] * 10, [0.0] * 10, [1e-30] * 10):
        _check(x, u, T)
        _check(x, u, T, [3] * 10, [0.8] * 10, [0.1] * 10)
    b = x[:9].bfloat16()
    _check(b, u[:9])
    _check(b, u[:9], None, [3] * 9, [0.8] * 9)


def test_random_numbers_and_parameters_at_their_ends(cuda_device):
    import torch
    nan = float("nan")
    x, rng = _logits(3, 9, 5000)
    u = [0.0, 1.0 - 2.0 ** -24, 0.5, 0.0, 1.0 - 2.0 ** -24, 0.25, 0.75, 0.1, 0.9]
    _check(x, u)
    _check(x, u, None, [1] * 9)
    _check(x, u, [0.7] * 9, [-5, 0, 5000, 6000, 1, 2, 3, 4999, 5], [nan, 1.0, 2.0, 0.0, -1.0, 1e-30, 0.5, 0.9999999, 0.1], [nan, -1.0, 0.0, 1.0, 2.0, 0.5, 1e-30, 0.01, 0.99])
    _check(x, u, [nan, -1.0, float("inf"), 1e30, 1e-20, 5.0, 0.01, 1.0, 100.0])


def test_captured_sampling_follows_its_arrays(cuda_device):
    import torch
    import paper_2607_06763_b200 as gdn
    x, rng = _logits(4, 6, 30000)
    u = torch.rand(6, device="cuda")
    p = torch.full((6,), 0.9, device="cuda")
    token = torch.empty(6, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    shape = gdn.GdnSampleShape.from_logits(x)
    call = lambda: gdn.gdn_sample(shape, x, None, None, p, None, u, token, None, status, torch.cuda.current_stream())
    assert call() == 0
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        assert call() == 0
    for _ in range(3):
        x.copy_(2.0 * torch.randn_like(x))
        u.copy_(torch.rand_like(u))
        g.replay()
        torch.cuda.synchronize()
        got = token.cpu().numpy()
        for r in range(6):
            assert got[r] == at.sample(x[r].double().cpu().numpy(), float(u[r]), p=float(p[r]))[0]


def _next_to_borders(cum, bound, rng, n, low=0.0):
    """Random numbers (fp32) that lie `bound` to 4 `bound` of the sum behind, or in front of, the end of a token's interval."""
    z = cum[-1]
    out = []
    for j in rng.permutation(len(cum) - 1):
        near = np.float32(cum[j] / z)
        for u in (near, np.nextafter(near, np.float32(0)), np.nextafter(near, np.float32(1))):
            if low <= u < 1.0 and bound < abs(float(u) - cum[j] / z) < 4 * bound:
                out.append(u)
                break
        if len(out) == n:
            return np.array(out, np.float32)
    raise AssertionError("too few")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("top", [0.0, -3.0, 5.0], ids=str)
def test_random_numbers_next_to_a_tokens_end(cuda_device, dtype, top):
    """A likely token behind a hundred thousand unlikely ones of few values, so that errors of their weights add up.  Each weight may be
    off by 2^-46 of the likeliest one's (half a unit), all of them together by vocab 2^-46: tokens are the ones of 64 bits wherever the
    random number is further than that from a border."""
    import torch
    n, vocab = 24, 100003
    rng = np.random.default_rng(50)
    x = torch.empty(n, vocab, dtype=at.torch_dtype(dtype), device="cuda")
    u = np.zeros(n, np.float32)
    for r in range(n):
        values = torch.from_numpy(top - rng.uniform(9.0, 12.5, 1 if r % 2 else 5)).to(x.dtype)
        row = values[torch.from_numpy(rng.integers(0, len(values), vocab))]
        row[-1] = top
        x[r] = row.cuda()
        w = np.exp(row.double().numpy() - top)
        cum = np.cumsum(w)
        u[r] = _next_to_borders(cum, vocab * 2.0 ** -46 / cum[-1], rng, 1)[0]
    _check(x, u)


def test_random_numbers_next_to_a_tokens_end_in_spread_logits(cuda_device):
    """Logits of a normal distribution, positive and negative ones, far below zero (log-probabilities) too."""
    import torch
    n, vocab = 24, 50000
    rng = np.random.default_rng(51)
    x = 2.2 * rng.standard_normal((n, vocab))
    x[8:16] -= 11.0
    x[16:] = x[16:] - np.log(np.exp(x[16:]).sum(1, keepdims=True))
    x = torch.from_numpy(x).float().cuda()
    u = np.zeros(n, np.float32)
    for r in range(n):
        row = x[r].double().cpu().numpy()
        cum = np.cumsum(np.exp(row - row.max()))
        u[r] = _next_to_borders(cum, vocab * 2.0 ** -46 / cum[-1], rng, 1)[0]
    _check(x, u)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_filters_that_end_next_to_a_border(cuda_device, dtype):
    """top_p just in front of, or behind, the share at which a prefix has one token more."""
    import torch
    n, vocab = 24, 60000
    rng = np.random.default_rng(52)
    x = torch.from_numpy(1.5 * rng.standard_normal((n, vocab)) - np.where(np.arange(n) % 2, 9.0, 0.0)[:, None]).to(at.torch_dtype(dtype)).cuda()
    p, u = np.zeros(n, np.float32), np.zeros(n, np.float32)
    for r in range(n):
        row = x[r].double().cpu().numpy()
        order = np.argsort(-row, kind="stable")
        w = np.exp(row[order] - row[order[0]])
        cum, bound = np.cumsum(w), vocab * 2.0 ** -46
        p[r] = _next_to_borders(cum, bound / cum[-1], rng, 1, 0.3)[0]
        kept = np.sort(order[:int(np.searchsorted(cum, float(p[r]) * cum[-1])) + 1])
        mass = np.cumsum(np.exp(row[kept] - row[order[0]]))
        u[r] = _next_to_borders(mass, bound / mass[-1], rng, 1)[0]
    _check(x, u, None, None, p)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_far_below_the_likeliest(cuda_device, dtype):
    """Weights down to 2^-45 of the likeliest one's are taken (half a unit of 2^-45 is rounded off); what is below 2^-46 is not."""
    import torch
    n, vocab = 8, 3000
    nats = np.array([26.5, 27.0, 27.5, 28.0, 28.25, 28.5, 29.0, 30.5])
    x = torch.full((n, vocab), -40.0, dtype=at.torch_dtype(dtype), device="cuda")
    x[:, 1] = torch.from_numpy(-nats).to(x.dtype).cuda()
    x[:, -1] = 0.0
    w = np.exp(x[:, 1].double().cpu().numpy())
    _check(x, 0.5 * w)           # inside the interval of token 1, for what lies in front of it weighs nothing
    _check(x, 2.0 * w)           # behind it
    far = torch.full((2, vocab), -32.0, dtype=x.dtype, device="cuda")     # 2^-46.2 each
    far[:, -1] = 0.0
    status, token = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    import paper_2607_06763_b200 as gdn
    assert gdn.gdn_sample(gdn.GdnSampleShape.from_logits(far), far, None, None, None, None, torch.tensor([0.0, 1e-13], device="cuda"), token, None,
                          status) == 0
    assert token.tolist() == [vocab - 1] * 2
