"""Tokens whose choice is looked for among the least weights, or among more tokens than
one list holds, against the plain form in binary64."""
import math

import numpy as np
import pytest
import torch

from layer_cases import DEV
from paper_2504_15299_amd import api
from test_gpu_sample import BF, F32, I32, gpu, normal, run

pytestmark = pytest.mark.gpu

LIST = 512      # tokens that one list holds


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("V,std", [(1500, 1e-3), (32000, 0.003), (50257, 0.02), (131072, 0.1)])
def test_top_p_in_bins_of_many_tokens(V, std, dtype):
    """Top-p over flat rows, whose bins (of 4/256 in units of log2) hold more than a
    list: the search starts over, with an empty list that every wave has seen full.  Many
    rows, twice: equal calls give equal tokens."""
    x = normal(24, V, dtype, std)
    width = 4 / 256 * np.log(2)
    top = x.float().amax(1, keepdim=True)
    assert all(torch.bincount(((t - r) / width).long()).max() > LIST
               for t, r in zip(top, x.float()))
    rng = np.random.default_rng(V)
    u, p = rng.random(24), rng.uniform(0.3, 0.95, 24)
    want = run(x, u, None, None, p)[0]
    many = x.repeat(40, 1).to(DEV)
    for _ in range(3):
        got, _ = api.sample(many, gpu(np.tile(u, 40), F32), top_p=gpu(np.tile(p, 40), F32))
        assert (got.view(40, 24).cpu().numpy() == want).all()


@pytest.mark.parametrize("dtype", [F32, BF])
def test_top_p_of_equal_logits(dtype):
    """All tokens in one bin, and of one key."""
    u = np.array([0.0, 0.25, 0.5, 0.75] * 64)
    x = torch.zeros((256, 4096), dtype=dtype)
    tokens, probs = api.sample(gpu(x), gpu(u, F32), top_p=gpu([0.5] * 256, F32))
    assert tokens.tolist() == [int(a * 2048) for a in u] and (probs == 2.0 ** -11).all()


def temperature_for(row, k):
    """The temperature at which a row's k-th largest weighs 2^-33.5 of the largest: below
    2^-31.98 one bin takes all that follows."""
    d = np.sort(row[row > -1e30].astype(np.float64))[::-1]
    assert len(row) - k > LIST
    return (d[0] - d[k - 1]) / (33.5 * math.log(2))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("mask", [-float("inf"), float("nan"), torch.finfo(BF).min])
@pytest.mark.parametrize("p,m", [(None, None), (0.9, None), (None, 0.01), (0.7, 0.001)])
@pytest.mark.parametrize("k", [513, 600, 1500, 12000])
def test_top_k_among_the_least_weights(k, p, m, mask, dtype):
    """Half of a vocabulary masked, a low temperature and a top-k that ends far below the
    largest: the masked tokens are not looked through."""
    V, B = 32000, 6
    x = normal(B, V, dtype)
    x[torch.rand((B, V), generator=torch.Generator().manual_seed(1)) < 0.5] = mask
    rows = x.float().numpy()
    t = [temperature_for(r, k) for r in rows]
    tokens, _ = run(x, np.random.default_rng(k).random(B), t, k, p, m)
    for b in range(B):
        assert 0 <= tokens[b] < V and rows[b, tokens[b]] > -100.0


@pytest.mark.parametrize("mask", [-float("inf"), float("nan")])
@pytest.mark.parametrize("p", [1.0 - 2.0 ** -24, 1.0])
def test_tokens_of_the_least_weights(mask, p):
    """One large logit, thousands of 2^-33 of its weight and thousands masked: what is
    drawn past the first is one of the thousands, in the order of their indexes.

    A weight is off by 2^-48 (half a unit) and 2^-42 of itself, so the running sum of n
    of them by n (2^-15 + 2^-42) of one."""
    V, n = 32000, 20000
    g = torch.Generator().manual_seed(3)
    at = torch.randperm(V, generator=g)[:n].sort().values
    x = torch.full((V,), mask)
    x[at] = -33 * math.log(2)
    first = 17
    x[first] = 0.0
    w = math.exp(float(x[at[at != first][0]]))
    rest = at[at != first].numpy()
    us = np.array([0.5, 1 - 2.0 ** -23, 1 - 2.0 ** -24], np.float32)
    tokens, probs = api.sample(gpu(x.expand(3, V).contiguous()), gpu(us),
                               top_p=gpu([p] * 3, F32))
    tokens, probs = tokens.tolist(), probs.tolist()
    whole = 1 + w * len(rest)
    kept = whole if p == 1.0 else 1 + w * math.ceil((p * whole - 1) / w)
    assert tokens[0] == first
    for u, token in zip(us[1:], tokens[1:]):
        i = int((float(u) * kept - 1) / w) if float(u) * kept >= 1 else -1
        if i < 0:
            assert token == first
            continue
        near = abs(int(np.searchsorted(rest, token)) - i)
        assert token in rest and near <= 2 + len(rest) * (2.0 ** -15 + 2.0 ** -42)
    for token, share in zip(tokens, probs):
        want = (1.0 if token == first else w) / kept
        assert abs(share - want) <= (2.0 ** -24 + 2.0 ** -14) * want


@pytest.mark.parametrize("dtype", [F32, BF])
def test_rows_of_more_than_one_launch(dtype):
    """More rows than one launch has threads for, each with settings of its own."""
    B, V = (1 << 22) + 3, 3
    x = torch.zeros((B, V), dtype=dtype, device=DEV)
    i = torch.arange(B, device=DEV)
    u = (i % 8).float() / 8
    k = (i % 4).to(I32)                 # 0: all three
    t = (i % 5 > 0).float()             # 0: the first
    tokens, probs = api.sample(x, u, temperature=t, top_k=k)
    n = torch.where(k == 0, 3, k.long())
    n = torch.where(t == 0, 1, n)
    assert torch.equal(tokens.long(), (u.double() * n).floor().long())
    assert torch.equal(probs, (1.0 / n.double()).float())
