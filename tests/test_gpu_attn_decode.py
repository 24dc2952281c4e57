"""Attention of one new token over the paged cache against binary64 within the
bound of its arithmetic.  Every cache row that is not attended holds NaN."""
import numpy as np
import pytest
import torch

import decoder_ref as ref
from layer_cases import DEV
from paper_2504_15299_amd import api

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def make(lengths, Hq, H, D, page, dtype, order="pthd", seed=0, width=None, window=0, spread=1.0):
    """(q, cache, table, lengths) on the device: pages in random places of a
    pool filled with NaN, rows only where a token is attended."""
    rng = np.random.default_rng(seed)
    B = len(lengths)
    width = width or max(1, -(-max(max(lengths), 1) // page))
    pool = B * width + 2
    table = rng.permutation(pool)[:B * width].reshape(B, width).astype(np.int32)
    if order == "joint":
        both = torch.full((pool, 2, page, H, D), float("nan"), dtype=dtype)
        k, v = both[:, 0], both[:, 1]
    else:
        names = {"p": pool, "t": page, "h": H, "d": D}
        k, v = (torch.full([names[c] for c in order], float("nan"), dtype=dtype)
                .permute([order.index(c) for c in "pthd"]) for _ in range(2))
    for b, n in enumerate(lengths):
        n = min(max(n, 0), width * page)
        j = np.arange(max(0, n - window) if window else 0, n)
        at = (torch.from_numpy(table[b][j // page].astype(np.int64)), torch.from_numpy(j % page))
        k[at] = ref.as_type(rng.standard_normal((len(j), H, D)) * spread, dtype)
        v[at] = ref.as_type(rng.standard_normal((len(j), H, D)), dtype)
    dev = lambda t: t.to(DEV)  # noqa: E731
    if order == "joint":
        both = dev(both)
        cache = api.KVCache(both[:, 0], both[:, 1])
    else:
        cache = api.KVCache(*(dev(t.permute([("pthd").index(c) for c in order]).contiguous())
                              .permute([order.index(c) for c in "pthd"]) for t in (k, v)))
    q = dev(ref.as_type(rng.standard_normal((B, Hq, D)) * spread, dtype))
    return (q, cache, dev(torch.from_numpy(table)),
            dev(torch.tensor(lengths, dtype=torch.int32)))


def check(q, cache, table, lengths, window=0, scale=None, **kw):
    out = api.attn_decode(q, cache, table, lengths, scale, window, **kw)
    want, err = ref.attn(ref.f64(q), ref.f64(cache.k), ref.f64(cache.v), table.cpu().numpy(),
                         lengths.cpu().numpy(),
                         q.shape[2] ** -0.5 if scale is None else scale, window)
    ref.close(out, want, err, q.dtype)
    return out


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 64, 100, 127, 128, 129, 257, 300]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [8, 16, 40, 64, 72, 80, 96, 128, 136, 192, 248, 256])
def test_dims(D, dtype):
    check(*make([0, 1, 33, 150], 4, 2, D, 16, dtype))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [1, 3, 16, 24, 64, 500])
def test_lengths_and_pages(page, dtype):
    check(*make(LENGTHS, 4, 1, 64, page, dtype, seed=page))


@pytest.mark.parametrize("Hq,H", [(1, 1), (3, 1), (7, 7), (16, 1), (17, 1), (40, 2), (64, 8),
                                  (96, 2)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_heads(Hq, H, dtype):
    check(*make([0, 5, 200], Hq, H, 128, 16, dtype, seed=Hq))


@pytest.mark.parametrize("order", ["pthd", "phtd", "joint", "hptd"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_orders(order, dtype):
    check(*make([40, 7, 0, 160], 6, 3, 64, 8, dtype, order))


# longer than the offsets held at a time, with few and many splits
@pytest.mark.parametrize("max_len", [0, 1, 1000, 2600, 100000])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_long_and_the_length_expected(max_len, dtype):
    """max_len only divides the work: results hold for longer sequences too."""
    check(*make([2600, 1025, 1, 0], 2, 1, 64, 16, dtype), max_len=max_len)


# the work in equal shares over all sequences, or whole per key head: batches of
# empty, short and long sequences, more of them than a wave has lanes and than a
# split call may have, key heads with more than 16 query heads
@pytest.mark.parametrize("B,Hq,H,D", [(2, 8, 8, 64), (70, 4, 2, 64), (256, 2, 1, 16),
                                      (257, 2, 1, 16), (30, 20, 1, 136), (5, 34, 2, 128)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("max_len", [100, 4000])
def test_shares(B, Hq, H, D, dtype, max_len):
    rng = np.random.default_rng(B)
    lengths = rng.integers(0, 60, B)
    lengths[rng.random(B) < 0.3] = 0
    lengths[rng.integers(0, B, max(1, B // 20))] = rng.integers(300, 700)
    check(*make(lengths.tolist(), Hq, H, D, 16, dtype, seed=B), max_len=max_len)


# more short units than the chip takes at a time; one sequence longer than expected
@pytest.mark.parametrize("G", [1, 6])
@pytest.mark.parametrize("D", [40, 64, 80, 128, 256])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_short_units(G, D, dtype):
    rng = np.random.default_rng(D + G)
    lengths = rng.integers(0, 50, 130)
    lengths[77] = 1100
    check(*make(lengths.tolist(), 4 * G, 4, D, 16, dtype, seed=D), max_len=30)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_all_empty(dtype):
    for max_len in (10, 5000):
        out = check(*make([0, 0, 0], 4, 2, 64, 16, dtype), max_len=max_len)
        assert (out == 0).all()


@pytest.mark.parametrize("window", [1, 2, 16, 31, 100, 128, 299, 300, 301, 5000])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_window(window, dtype):
    check(*make(LENGTHS, 4, 2, 64, 16, dtype, window=window), window=window)


def test_window_of_a_long_sequence():
    check(*make([5000, 3000], 4, 2, 128, 64, BF, window=1500), window=1500)
    check(*make([5000, 3000], 4, 2, 128, 64, BF, window=1500), window=1500, max_len=100)


def test_lengths_beyond_the_table_and_below_zero():
    check(*make([-5, 100, 47, 48, 2 ** 31 - 1, -2 ** 31], 2, 2, 64, 16, BF, width=3))


@pytest.mark.parametrize("scale", [0.0, 1.0, -0.7, 3.0])
def test_scales(scale):
    """From a plain mean to scores where one key takes all."""
    check(*make([1, 70, 200], 4, 2, 64, 16, F32), scale=scale)
    check(*make([1, 70, 200], 4, 2, 64, 16, BF), scale=scale)


def test_scores_that_fall_and_grow_along_the_sequence():
    """The running maximum changes at every tile, or never."""
    for slope in (-1.0, 1.0):
        q, cache, table, lengths = make([400], 2, 1, 64, 16, F32)
        j = torch.arange(400, device=DEV)
        rows = (table[0][j // 16].long(), j % 16, 0)
        cache.k[rows] = slope * 0.05 * j[:, None] * torch.ones(64, device=DEV)
        q[:] = 0.3
        check(q, cache, table, lengths)


def test_bad_pages_count_as_masked():
    q, cache, table, lengths = make([100, 64, 30], 4, 2, 64, 16, BF, width=7)
    table[0, 2], table[0, 5] = -1, cache.n_pages
    table[1, :] = 2 ** 31 - 1
    table[2, 0], table[2, 1] = -2 ** 31, cache.n_pages + 5
    out = check(q, cache, table, lengths)
    assert (out[1:] == 0).all()


def test_infinities():
    """An infinite value reaches the result with the sign it has; an infinite
    score leaves no number; neither touches another sequence."""
    q, cache, table, lengths = make([50, 50, 50], 2, 1, 64, 16, BF)
    clean = api.attn_decode(q, cache, table, lengths)
    cache.v[table[1, 0], 3, 0, 5] = float("inf")
    cache.v[table[1, 0], 3, 0, 6] = -float("inf")
    cache.k[table[2, 0], 3, 0, 5] = float("nan")
    out = api.attn_decode(q, cache, table, lengths)
    assert torch.equal(out[0], clean[0])
    assert (out[1, :, 5] == float("inf")).all() and (out[1, :, 6] == -float("inf")).all()
    others = [d for d in range(64) if d not in (5, 6)]
    assert torch.equal(out[1][:, others], clean[1][:, others])
    assert torch.isnan(out[2]).all()


def test_strided_queries():
    q, cache, table, lengths = make([40, 41, 42], 4, 2, 64, 16, BF)
    wide = torch.zeros((3, 9, 64), dtype=BF, device=DEV)
    wide[:, 2:6] = q
    out = check(wide[:, 2:6], cache, table, lengths)
    assert torch.equal(out, api.attn_decode(q, cache, table, lengths))


def test_cache_beyond_32_bit_offsets():
    """The last pages of a cache of over 2^32 elements and 2^33 bytes."""
    page, H, D = 64, 8, 128
    n = (1 << 32) // (page * H * D) + 3
    k = torch.empty((n, page, H, D), dtype=BF, device=DEV)
    v = torch.empty_like(k)
    small = api.KVCache.empty(4, page, H, D, device=DEV)
    for t in (small.k, small.v):
        t.normal_()
    k[-4:], v[-4:] = small.k, small.v
    q = torch.randn((1, 16, D), dtype=BF, device=DEV)
    near = torch.tensor([[2, 0, 3, 1]], dtype=torch.int32, device=DEV)
    lengths = torch.tensor([230], dtype=torch.int32, device=DEV)
    cache, far = api.KVCache(k, v), near + (n - 4)
    want = api.attn_decode(q, small, near, lengths)
    assert torch.equal(api.attn_decode(q, cache, far, lengths), want)
    x = torch.randn((1, H, D), dtype=BF, device=DEV)
    pos = lengths - 1
    api.kv_append(None, x, x, cache, far, pos)
    api.kv_append(None, x, x, small, near, pos)
    assert torch.equal(k[-4:], small.k) and torch.equal(v[-4:], small.v)


def test_two_streams_with_a_workspace_each():
    a, b = (make([700, 300, 900], 8, 2, 128, 16, BF, seed=s) for s in (1, 2))
    want = [check(*c) for c in (a, b)]
    need = api.attn_decode_workspace(3, 8, a[1], 1000)
    ws = [torch.empty(need, dtype=torch.uint8, device=DEV) for _ in range(2)]
    s = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[api.attn_decode(*c, max_len=1000, workspace=w, stream=t) for c, w, t in zip((a, b), ws, s)]
           for _ in range(4)]
    torch.cuda.synchronize()
    first = got[0]
    for pair in got:
        for x, y, z in zip(pair, first, want):
            assert torch.equal(x, y)
            assert (x.float() - z.float()).abs().max() <= 2.0 ** -7 * z.float().abs().max()


def test_captured_call_follows_its_inputs():
    q, cache, table, lengths = make([200, 100, 40], 8, 2, 64, 16, BF)
    ws = torch.empty(api.attn_decode_workspace(3, 8, cache, 208), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)
    api.attn_decode(q, cache, table, lengths, max_len=208, out=out, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        api.attn_decode(q, cache, table, lengths, max_len=208, out=out, workspace=ws)
    for n in ([200, 100, 40], [3, 0, 40], [150, 100, 1]):
        lengths.copy_(torch.tensor(n, dtype=torch.int32))
        ws.fill_(255)
        want = api.attn_decode(q, cache, table, lengths, max_len=208)
        out.fill_(-7)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_no_sequences():
    q, cache, table, lengths = make([5], 2, 1, 64, 16, BF)
    out = api.attn_decode(q[:0], cache, table[:0], lengths[:0])
    assert out.shape == (0, 2, 64)


def test_rejects_wrong_arguments():
    q, cache, table, lengths = make([50, 60], 4, 2, 64, 16, BF)
    ok = dict(q=q, cache=cache, block_table=table, lengths=lengths)
    for bad in (dict(q=q.float()), dict(q=q[:, :, :32]), dict(lengths=lengths[:1]),
                dict(lengths=lengths.long()), dict(block_table=table[:1]), dict(q=q.cpu()),
                dict(out=q[:1]), dict(block_table=table.t().contiguous().t())):
        with pytest.raises(ValueError):
            api.attn_decode(**{**ok, **bad})
    for bad in (dict(window=-1), dict(max_len=-1), dict(q=q[:, :3].contiguous()),
                dict(scale=float("nan")), dict(scale=float("inf"))):
        with pytest.raises(api.D2MoEError) as e:
            api.attn_decode(**{**ok, **bad})
        assert e.value.status == api.EINVAL
    with pytest.raises(api.D2MoEError) as e:
        api.attn_decode(**ok, max_len=4000, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    assert e.value.status == api.EWORKSPACE
    with pytest.raises(ValueError):
        api.KVCache(cache.k, cache.v[:1])
    with pytest.raises(ValueError):
        api.KVCache(cache.k.transpose(2, 3), cache.v.transpose(2, 3))
