"""Attention over a bf16 cache where its probabilities' last bits, the smallest of
them and the largest values show."""
import numpy as np
import pytest
import torch

import decoder_ref as ref
from layer_cases import DEV
from paper_2504_15299_amd import api

pytestmark = pytest.mark.gpu

BF, I32 = torch.bfloat16, torch.int32


def bf(a):
    return ref.f64(ref.as_type(a, BF))


def attend(scores, v, Hq):
    """scores [B][H][n], v [B][n][H][D], both of bf16 values: the result of queries
    that are 1 in their first place over keys that hold the score there."""
    B, H, n = scores.shape
    D = v.shape[3]
    cache = api.KVCache.empty(B, n, H, D, device=DEV)
    k = torch.zeros((B, n, H, D))
    k[..., 0] = torch.from_numpy(scores.transpose(0, 2, 1)).float()
    cache.k.copy_(k)
    cache.v.copy_(torch.from_numpy(v).float())
    q = torch.zeros((B, Hq, D), dtype=BF, device=DEV)
    q[..., 0] = 1.0
    table = torch.arange(B, dtype=I32, device=DEV)[:, None]
    return ref.f64(api.attn_decode(q, cache, table, torch.full((B,), n, dtype=I32, device=DEV),
                                   scale=1.0))


@pytest.mark.parametrize("D", [16, 64, 128, 256])
def test_probabilities_keep_24_bits(D):
    """Values that cancel in the sum of p V down to 2^-18 of the sum of p |V|, so that
    the result's own rounding does not hide the terms' errors.

    A score is one product, exact.  Its exponent is off by two roundings (|score| <= 1,
    in units of log2) and that of the difference to the maximum, 4.4 U in all, the
    probability by 3.1 U of itself for it and 2 U for exp2; what is common to all of them
    cancels.  The sum has 5 keys of three pieces, each addition off by 2 U at most of
    the sum of magnitudes: 36 U together, 2^-18.8.  (Two pieces: up to 2^-16.)"""
    rng = np.random.default_rng(D)
    B, H, Hq, n = 16, 2, 4, 5
    scores = bf(-rng.random((B, H, n)))
    p = np.exp(scores)
    v = bf(rng.uniform(1, 2, (B, n, H, D)) * rng.choice([-1, 1], (B, n, H, D)))
    pt = p.transpose(0, 2, 1)[..., None]
    for j in (2, 3, 4):
        v[:, j] = bf(-(pt[:, :j] * v[:, :j]).sum(1) / pt[:, j])
    total = p.sum(2)[..., None]
    want = (pt * v).sum(1) / total
    mag = (pt * np.abs(v)).sum(1) / total
    assert np.median(np.abs(want) / mag) < 2.0 ** -17
    got = attend(scores, v, Hq)
    want, mag = np.repeat(want, Hq // H, 1), np.repeat(mag, Hq // H, 1)
    assert (np.abs(got - want) <= 36 * ref.U * mag + (ref.HALF[BF] + 8 * ref.U) * np.abs(want)).all()


def test_values_of_keys_without_weight():
    """A probability of zero adds nothing, whatever the value's size; one of 2^-124
    adds what it should, within the 2^-132 that its last pieces may lack."""
    scores = np.array([[[0.0, -300.0]], [[0.0, -86.0]]])
    v = np.ones((2, 2, 1, 16))
    v[0, 1] = bf(1e38)
    v[1, 1] = 2.0 ** 124
    v[:, :, :, 1] *= -1
    got = attend(scores, v, 1)
    sign = np.where(np.arange(16) == 1, -1.0, 1.0)
    assert np.array_equal(got[0, 0], sign)
    # the exponent 86 log2(e) is off by 3 U of itself
    term = np.exp(-86.0) * 2.0 ** 124
    room = term * 3 * 125 * ref.U + 2.0 ** -8 + ref.HALF[BF] * (1 + term)
    assert (np.abs(got[1, 0] - sign * (1 + term)) <= room).all()


@pytest.mark.parametrize("score", [0.0, -1.0, -50.0, -75.0, -87.0])
def test_infinite_value_of_any_weight(score):
    """An infinite value stays one whatever its probability, down to the least."""
    scores = np.array([[[0.0, score, score / 2]]])
    v = np.ones((1, 3, 1, 16))
    v[0, 1, 0, 3], v[0, 1, 0, 4] = np.inf, -np.inf
    got = attend(scores, v, 1)[0, 0]
    assert got[3] == np.inf and got[4] == -np.inf
    assert (np.delete(got, [3, 4]) == 1.0).all()
