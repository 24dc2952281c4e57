"""Queries, keys and values that are NaN or infinite reach the results that attend them,
and no others.

The others are held to the bound of their arithmetic, not to the same bits: the
references of a wave's exponents move together."""
import numpy as np
import pytest
import torch

import decoder_ref as ref
import step_ref as step
from paper_2504_15299_amd import api
from test_gpu_attn_prefix import BF, F32, make

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def plain(q, cache, table, lengths, ptab, shared):
    """The binary64 form and its bound."""
    return step.attn_prefix(ref.f64(q), ref.f64(cache.k), ref.f64(cache.v), table.cpu().numpy(),
                            lengths.cpu().numpy(), ptab.cpu().numpy(), shared.cpu().numpy(),
                            q.shape[2] ** -0.5)


def check_others(out, want, touched):
    """The results outside `touched` (rows or elements) are the plain form's, those in it
    are not finite."""
    got = ref.f64(out)
    assert not np.isfinite(got[touched]).any(), np.argwhere(np.isfinite(got) & touched)[:3].tolist()
    ref.close(np.where(touched, want[0], got), *want, out.dtype)


def rows_of(out):
    return np.zeros(out.shape, bool)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,H", [(4, 2), (12, 2), (34, 2)])
def test_nan_query(Hq, H, D, dtype):
    """One query head of one sequence: its row is NaN."""
    a = make([150] * 5, [150, 151, 183, 300, 170], Hq, H, D, 16, dtype, seed=D)
    want = plain(*a)
    for b, h in ((0, 0), (2, Hq - 1), (4, Hq // 2)):
        kept = a[0][b, h].clone()
        a[0][b, h] = NAN
        out = api.attn_prefix(*a)
        touched = rows_of(out)
        touched[b, h] = True
        check_others(out, want, touched)
        a[0][b, h] = kept


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("prefix", [0, 128, 200])
def test_nan_key_alone_behind_the_prefix(prefix, dtype):
    """The one token that a sequence has of its own."""
    a = make([prefix] * 4, [prefix + 1, prefix + 1, prefix + 40, prefix + 1], 8, 2, 64, 16, dtype,
             seed=prefix)
    want = plain(*a)
    cache, table = a[1:3]
    cache.k[int(table[1, prefix // 16]), prefix % 16, 1] = NAN
    out = api.attn_prefix(*a)
    touched = rows_of(out)
    touched[1, 4:] = True
    check_others(out, want, touched)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("token", [0, 64, 128, 130])
def test_nan_key_of_the_prefix(token, dtype):
    """Alone in a run of it, or among others: NaN for all that share it."""
    shared = [131, token, 131, token + 1, 0]
    a = make(shared, [131, 140, 160, 145, 9], 8, 2, 64, 16, dtype, prefix=131, seed=token)
    want = plain(*a)
    cache, ptab = a[1], a[4]
    cache.k[int(ptab[token // 16]), token % 16, 0] = NAN
    out = api.attn_prefix(*a)
    touched = rows_of(out)
    touched[np.array(shared) > token, :4] = True
    check_others(out, want, touched)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [40, 64, 128, 256])
@pytest.mark.parametrize("Hq,H", [(4, 2), (12, 2), (34, 2)])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
def test_values_of_keys_of_other_sequences(value, Hq, H, D, dtype):
    """The prefix's keys and values, and the own ones of other sequences, past what a
    sequence shares, whatever they hold: sequences that end before, inside and behind the
    tiles and runs where they lie."""
    shared = [300, 170, 0, 131, 130, 129, 64, 300, 1, 170]
    lengths = [300, 180, 20, 131, 200, 129, 64, 340, 1, 170]
    a = make(shared, lengths, Hq, H, D, 16, dtype, prefix=300, seed=D)
    want = plain(*a)
    q, cache, table, _, ptab, _ = a
    touched = np.zeros(q.shape, bool)
    G = Hq // H
    for token, head, d in ((130, 0, 3), (131, 1, D - 1), (171, 0, 0), (250, 1, 8)):
        cache.v[int(ptab[token // 16]), token % 16, head, d] = value
        touched[np.array(shared) > token, head * G:(head + 1) * G, d] = True
    cache.v[int(table[7, 310 // 16]), 310 % 16, 0, 5] = value
    touched[7, :G, 5] = True
    check_others(api.attn_prefix(*a), want, touched)
    # keys too: NaN scores for those who attend them
    cache.k[int(ptab[180 // 16]), 180 % 16, 1, 2] = NAN
    touched[np.array(shared) > 180, G:] = True
    check_others(api.attn_prefix(*a), want, touched)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_sequences_without_a_share_beside_a_prefix_of_nan(dtype):
    shared = [200, 0, 200, 0, 0]
    a = make(shared, [200, 50, 210, 1, 0], 8, 2, 128, 16, dtype, seed=1)
    want = plain(*a)
    cache, ptab = a[1], a[4]
    cache.k[ptab.long()] = NAN
    cache.v[ptab.long()] = NAN
    out = api.attn_prefix(*a)
    touched = rows_of(out)
    touched[[0, 2]] = True
    check_others(out, want, touched)
    assert (out[4] == 0).all()
