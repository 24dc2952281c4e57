"""Tokens by temperature, top-k, top-p and min-p against the plain form in binary64: the
same tokens, wherever a choice is not within the units of the weights of turning."""
import numpy as np
import pytest
import torch

import step_ref as step
from layer_cases import DEV
from paper_2504_15299_amd import api

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def gpu(a, dtype=None):
    return None if a is None else torch.as_tensor(a, dtype=dtype).to(DEV)


def run(logits, u, t=None, k=None, p=None, m=None, least_room=1e-9):
    """logits: a host tensor.  A weight is off by half a unit of 2^-38 at most (the
    longest rows allowed), a running sum of V of them, of which the largest is 1, by less
    than V 2^-39 of itself: below 1e-9 for all rows here but those longer than 500, whose
    unit is 2^-45 and smaller."""
    B = len(logits)
    f = lambda a, d: None if a is None else torch.as_tensor(np.broadcast_to(a, B).copy(), dtype=d)  # noqa: E731
    tt, kk, pp, mm, uu = f(t, F32), f(k, I32), f(p, F32), f(m, F32), f(u, F32)
    tokens, probs = api.sample(logits.to(DEV), gpu(uu), gpu(tt), gpu(kk), gpu(pp), gpu(mm))
    tokens, probs = tokens.cpu().numpy(), probs.cpu().numpy()
    rows = logits.float().numpy()
    near = 0
    for b in range(B):
        one = lambda a, d: d if a is None else float(a[b])  # noqa: E731
        tok, share, room = step.sample(rows[b], one(uu, 0.0), one(tt, 1.0), int(one(kk, 0)),
                                       one(pp, 1.0), one(mm, 0.0))
        if room < least_room:
            near += 1
            continue
        assert tokens[b] == tok, (b, tokens[b], tok, room)
        # binary64 but for the kept sum's units, then one rounding
        assert abs(probs[b] - share) <= (2.0 ** -24 + 1e-9) * share + 1e-45
    assert near <= B // 8, near
    return tokens, probs


def normal(B, V, dtype=F32, std=3.0, seed=0):
    g = torch.Generator().manual_seed(seed + V)
    return (torch.randn((B, V), generator=g) * std).to(dtype)


def settings(B, rng, **kw):
    s = dict(u=rng.random(B), t=rng.uniform(0.3, 1.5, B), k=rng.integers(1, 100, B),
             p=rng.uniform(0.3, 1.0, B), m=rng.uniform(0, 0.1, B))
    return {**s, **kw}


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 63, 64, 65, 1000, 1023, 1025, 4096, 4099, 8193,
                               32000, 50257, 131072])
def test_lengths_and_types(V, dtype):
    rng = np.random.default_rng(V)
    run(normal(12, V, dtype), **settings(12, rng))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("bounds", ["", "k", "p", "m", "kp", "km", "pm", "kpm"])
def test_bounds(bounds, dtype):
    rng = np.random.default_rng(len(bounds))
    s = settings(40, rng)
    run(normal(40, 3001, dtype), **{n: v if n in "ut" or n in bounds else None
                                    for n, v in s.items()})


@pytest.mark.parametrize("t", [1e-30, 1e-3, 0.1, 1.0, 5.0, 1000.0, 1e30])
@pytest.mark.parametrize("k,p", [(0, 1.0), (0, 0.7), (1500, 1.0), (1500, 0.7), (8000, 0.9)])
def test_temperatures(t, k, p):
    """The highest of them put all tokens into one bin of the histogram."""
    rng = np.random.default_rng(3)
    run(normal(16, 9001), rng.random(16), t, k, p)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("k", [None, 3, 500, 512, 513, 2000])
@pytest.mark.parametrize("p", [None, 0.2, 0.999])
@pytest.mark.parametrize("m", [None, 0.9, 0.05, 1e-6])
def test_bounds_of_flat_rows(m, p, k, dtype):
    """Rows of which min-p or top-k leave a few tokens, some hundred or thousands, and in
    which top-p ends before or after them; logits that fill one bin, or many."""
    rng = np.random.default_rng(9)
    for V, std in ((700, 0.5), (6001, 0.02), (6001, 1.0), (20000, 4.0)):
        run(normal(6, V, dtype, std), rng.random(6), rng.uniform(0.5, 1.5, 6), k, p, m)


def test_temperature_zero_takes_the_largest():
    x = normal(9, 5000)
    x[3, 77] = x[3, 4000] = 50.0
    tokens, probs = api.sample(gpu(x), torch.full((9,), 0.99, device=DEV),
                               temperature=gpu([0.0, -1.0, float("nan")] * 3, F32))
    want = x.argmax(1)
    want[3] = 77
    assert torch.equal(tokens.cpu().long(), want) and (probs == 1).all()


@pytest.mark.parametrize("V", [1000, 1024, 1025, 5000, 30011])
@pytest.mark.parametrize("value", [0.0, -0.0, -2.5, 3e38, -3e38])
def test_equal_logits(V, value):
    """All weights are 1, everything is exact: token floor(u n) of the first n."""
    u = np.array([0.0, 1 / 1024, 0.25, 0.5, 0.75, 1023 / 1024])
    x = torch.full((6, V), value)
    for k, p, n in ((0, 1.0, V), (700, 1.0, 700), (0, 0.5, -(-V // 2)), (600, 0.25, 150),
                    (V - 1, 0.125, -(-(V - 1) // 8))):
        tokens, probs = api.sample(gpu(x), gpu(u, F32), top_k=gpu([k] * 6, I32),
                                   top_p=gpu([p] * 6, F32))
        assert tokens.tolist() == [int(a * n) for a in u]
        assert probs.tolist() == [float(np.float32(1 / n))] * 6


@pytest.mark.parametrize("V", [600, 40000])
def test_signed_zeros_are_equal(V):
    x = torch.zeros((2, V))
    x[:, ::2] = -0.0
    tokens, _ = api.sample(gpu(x), gpu([0.0, 0.5], F32), top_k=gpu([4, 4], I32))
    assert tokens.tolist() == [0, 2]


@pytest.mark.parametrize("dtype", [F32, BF])
def test_few_distinct_logits(dtype):
    """Thousands of equal ones around every border."""
    rng = np.random.default_rng(0)
    x = torch.from_numpy(rng.integers(-3, 1, (24, 20000)).astype(np.float32)).to(dtype)
    run(x, rng.random(24), 1.0, rng.integers(1, 20000, 24), rng.uniform(0.2, 1, 24))
    run(x, rng.random(24), 20.0, None, rng.uniform(0.2, 1, 24))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("mask", [-float("inf"), float("nan"), torch.finfo(BF).min])
def test_masked_logits(dtype, mask):
    """Masked tokens are not chosen, whichever way they are masked; a row of nothing
    else gives -1 (where the mask is a number, it is the row's only value)."""
    rng = np.random.default_rng(1)
    x = normal(20, 2000, dtype)
    x[torch.from_numpy(rng.random((20, 2000)) < 0.9)] = mask
    x[7], x[8, 1:] = mask, mask
    s = settings(20, rng, k=rng.integers(0, 2000, 20))
    tokens, probs = run(x, **s)
    if mask == torch.finfo(BF).min:
        assert 0 <= tokens[7]
    else:
        assert tokens[7] == -1 and probs[7] == 0.0
    assert tokens[8] == 0 and probs[8] == 1.0
    real = x.float().numpy()
    for b in set(range(20)) - {7}:
        assert np.isfinite(real[b, tokens[b]]) and real[b, tokens[b]] > -1e30


def test_infinite_logits_share_everything():
    x = normal(4, 3000)
    x[:, [5, 100, 2900]] = float("inf")
    tokens, probs = api.sample(gpu(x), gpu([0.0, 0.4, 0.7, 0.9999], F32),
                               temperature=gpu([1.0, 0.1, 1e38, float("inf")], F32))
    assert tokens.tolist() == [5, 100, 2900, 2900]
    assert probs.tolist() == [float(np.float32(1 / 3))] * 4


def test_bounds_outside_their_ranges():
    """u as the nearest number of [0, 1), p <= 0 one token, bounds that are NaN none, min-p
    above 1 the largest only."""
    x = normal(1, 500).expand(8, 500).contiguous()
    x[:, 10] = x[:, 20] = 40.0
    nan, inf = float("nan"), float("inf")
    tokens, _ = api.sample(gpu(x), gpu([-1.0, nan, 1.0, inf, 0.9, 0.9, 0.9, 0.0], F32),
                           top_p=gpu([nan, 1.0, 1.0, 2.0, 0.0, -3.0, 1.0, nan], F32),
                           min_p=gpu([nan, 0.0, 0.5, 7.0, 0.0, 0.0, 1.0, -1.0], F32),
                           top_k=gpu([-5, 0, 0, 0, 0, 0, 0, 10 ** 9], I32))
    assert tokens.tolist() == [10, 10, 20, 20, 10, 10, 20, 10]


@pytest.mark.parametrize("dtype", [F32, BF])
def test_rows_at_any_address(dtype):
    """Rows of a wider tensor that begin anywhere within 16 bytes; what lies beside them
    is not looked at."""
    rng = np.random.default_rng(5)
    for off in range(9):
        wide = torch.full((6, 1111 + 17), float("nan"), dtype=dtype, device=DEV)
        x = normal(6, 1111, dtype, seed=off)
        wide[:, :off] = 1e4
        wide[:, off + 1111:] = 1e4
        view = wide[:, off:off + 1111]
        view.copy_(x)
        u = gpu(rng.random(6), F32)
        got, want = api.sample(view, u), api.sample(gpu(x), u)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_frequencies():
    """Over evenly spread u a token comes up as often as its share says."""
    B, V = 4096, 50
    x = normal(1, V, std=1.5)
    u = (torch.arange(B) + 0.5) / B
    tokens, probs = api.sample(gpu(x.expand(B, V).contiguous()), gpu(u, F32))
    p = torch.softmax(x[0].double(), 0)
    n = torch.bincount(tokens.cpu().long(), minlength=V)
    assert ((n - B * p).abs() <= 1).all()
    assert ((probs.cpu() - p[tokens.cpu().long()]).abs() <= 1e-7).all()


def test_many_rows_and_none():
    x = torch.zeros((70001, 3), device=DEV)
    u = torch.rand(70001, device=DEV)
    tokens, _ = api.sample(x, u)
    assert torch.equal(tokens, (u.double() * 3).floor().to(I32))
    tokens, probs = api.sample(x[:0], u[:0])
    assert tokens.shape == probs.shape == (0,)


def test_rows_past_32_bit_offsets():
    V = 1 << 24
    x = torch.full((130, V), -10.0, dtype=BF, device=DEV)
    at = torch.randint(0, V, (130,), device=DEV)
    x[torch.arange(130, device=DEV), at] = 100.0
    tokens, _ = api.sample(x, torch.full((130,), 0.999, device=DEV))
    assert torch.equal(tokens.long(), at)
    # the longest row, all of them equal
    tokens, _ = api.sample(torch.zeros((1, V), dtype=BF, device=DEV), gpu([0.75], F32))
    assert tokens.tolist() == [V * 3 // 4]


def test_graph_and_another_stream():
    x, u = normal(5, 32000).to(DEV), torch.rand(5, device=DEV)
    p = torch.full((5,), 0.9, device=DEV)
    tokens, probs = api.sample(x, u, top_p=p)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        api.sample(x, u, top_p=p, tokens=tokens, probs=probs)
    s = torch.cuda.Stream()
    for _ in range(3):
        x.normal_(0, 3)
        u.uniform_()
        g.replay()
        torch.cuda.synchronize()
        other = api.sample(x, u, top_p=p, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(tokens, other[0]) and torch.equal(probs, other[1])
