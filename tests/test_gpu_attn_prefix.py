"""Attention of one new token per sequence behind a shared prefix against binary64 within
the bound of its arithmetic.  Every cache row that is not attended holds NaN."""
import numpy as np
import pytest
import torch

import decoder_ref as ref
import step_ref as step
from layer_cases import DEV
from paper_2504_15299_amd import api

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def make(shared, lengths, Hq, H, D, page, dtype, prefix=None, seed=0, spread=1.0, order="pthd"):
    """(q, cache, table, lengths, prefix_table, prefix_lens) on the device: pages in random
    places of a pool filled with NaN, rows only where a token is attended, entries of
    pages that a sequence shares whole -1."""
    rng = np.random.default_rng(seed)
    B = len(lengths)
    prefix = max(max(shared), 1) if prefix is None else prefix
    head = -(-prefix // page)
    width = max(1, -(-max(max(lengths), 1) // page))
    pool = head + B * width + 2
    pages = rng.permutation(pool)
    ptab, table = pages[:head].astype(np.int32), np.full((B, width), -1, np.int32)
    names = {"p": pool, "t": page, "h": H, "d": D}
    k, v = (torch.full([names[c] for c in order], float("nan"), dtype=dtype)
            .permute([order.index(c) for c in "pthd"]) for _ in range(2))

    def fill(p, slot):
        at = torch.from_numpy(p.astype(np.int64)), torch.from_numpy(slot)
        k[at] = ref.as_type(rng.standard_normal((len(slot), H, D)) * spread, dtype)
        v[at] = ref.as_type(rng.standard_normal((len(slot), H, D)), dtype)

    s = [min(a, n, head * page) for a, n in zip(shared, lengths)]
    j = np.arange(max(max(s), 0))
    fill(ptab[j // page], j % page)
    for b in range(B):
        j = np.arange(max(s[b], 0), max(lengths[b], 0))
        if len(j):
            first = j[0] // page
            table[b, first:] = pages[head + b * width + first:head + (b + 1) * width]
            fill(table[b][j // page], j % page)
    dev = lambda t: t.to(DEV)  # noqa: E731
    cache = api.KVCache(*(dev(t.permute(["pthd".index(c) for c in order]).contiguous())
                          .permute([order.index(c) for c in "pthd"]) for t in (k, v)))
    ints = lambda a: dev(torch.tensor(a, dtype=I32))  # noqa: E731
    q = dev(ref.as_type(rng.standard_normal((B, Hq, D)) * spread, dtype))
    return (q, cache, dev(torch.from_numpy(table)), ints(lengths), dev(torch.from_numpy(ptab)),
            ints(shared))


def check(q, cache, table, lengths, ptab, shared, scale=None, **kw):
    out = api.attn_prefix(q, cache, table, lengths, ptab, shared, scale, **kw)
    want, err = step.attn_prefix(ref.f64(q), ref.f64(cache.k), ref.f64(cache.v),
                                 table.cpu().numpy(), lengths.cpu().numpy(), ptab.cpu().numpy(),
                                 shared.cpu().numpy(), q.shape[2] ** -0.5 if scale is None else scale)
    ref.close(out, want, err, q.dtype)
    return out


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [8, 16, 40, 64, 72, 80, 96, 128, 136, 192, 248, 256])
@pytest.mark.parametrize("Hq,H", [(4, 2), (10, 2), (36, 2)])
def test_dims(D, Hq, H, dtype):
    """Up to 16, up to 32 and more queries of a key head."""
    check(*make([150] * 5, [150, 151, 183, 300, 170], Hq, H, D, 16, dtype, seed=D))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [1, 3, 16, 24, 64, 500])
@pytest.mark.parametrize("prefix", [1, 15, 16, 17, 31, 33, 64, 65, 127, 128, 129, 257, 300])
def test_prefixes_and_pages(prefix, page, dtype):
    own = [0, 1, 2, 15, 16, 17, 33, 64, 100, 129]
    check(*make([prefix] * 10, [prefix + n for n in own], 4, 1, 64, page, dtype, seed=page))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hq,H", [(1, 1), (3, 1), (7, 7), (16, 1), (17, 1), (40, 2), (64, 8),
                                  (96, 2)])
@pytest.mark.parametrize("B", [1, 2, 9, 33])
def test_batches_and_heads(B, Hq, H, dtype):
    rng = np.random.default_rng(B)
    check(*make([70] * B, (70 + rng.integers(0, 40, B)).tolist(), Hq, H, 128, 16, dtype, seed=Hq))


# sequences that share a part, nothing, more than the prefix's table or their own length
# says, that are empty, or end inside the prefix
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("G", [1, 4, 13])
def test_shares_of_any_length(G, D, dtype):
    shared = [200, 0, 1, 63, 64, 65, 200, 199, 128, 0, 200, 5, -3, 1000, 100]
    lengths = [200, 0, 1, 64, 64, 200, 350, 199, 300, 77, 0, -5, 40, 300, 50]
    check(*make(shared, lengths, 2 * G, 2, D, 16, dtype, prefix=200, seed=G))


def test_nothing_at_all():
    out = check(*make([0, 5, -1], [0, 0, -1], 4, 2, 64, 16, BF))
    assert (out == 0).all()


# the lengths expected only divide the work
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("max_prefix,max_rest", [(0, 0), (1, 10 ** 6), (10 ** 6, 1), (500, 100),
                                                 (1 << 30, 1 << 30)])
def test_lengths_expected(max_prefix, max_rest, dtype):
    check(*make([1300, 900, 1300], [2100, 1000, 1301], 6, 2, 128, 16, dtype),
          max_prefix=max_prefix, max_rest=max_rest)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_many_runs_and_row_tiles(D, dtype):
    """70 queries of a key head, a prefix in tens of runs."""
    check(*make([4000] * 10, [4000 + 30 * i for i in range(10)], 7, 1, D, 16, dtype, seed=D))


@pytest.mark.parametrize("order", ["phtd", "hptd"])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_orders(order, dtype):
    check(*make([60] * 3, [90, 61, 100], 6, 3, 64, 8, dtype, order=order))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [0.0, 1.0, -0.3, 1e-30])
def test_scales(scale, dtype):
    check(*make([90] * 3, [130, 91, 200], 8, 2, 64, 16, dtype), scale=scale)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_large_scores(dtype):
    """Scores of hundreds: nearly all weight on single keys, anywhere."""
    check(*make([300] * 6, [330, 301, 450, 300, 310, 600], 8, 2, 128, 16, dtype, spread=6.0))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_masked_pages(dtype):
    """Pages outside the pool count as masked, in either table; a sequence with nothing
    else gives zeros."""
    q, cache, table, lengths, ptab, shared = make([100] * 4, [140, 200, 100, 150], 8, 2, 64, 16,
                                                  dtype)
    table[0, 7], table[1, 9], table[1, 10] = 10 ** 6, -1, -2147483648
    table[3, 6:] = -1
    ptab[2], ptab[4] = -7, cache.n_pages
    check(q, cache, table, lengths, ptab, shared)
    ptab[:] = -1
    out = check(q, cache, table, lengths, ptab, shared)
    assert (out[2] == 0).all() and (out[3] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinite_scores_that_mask(dtype):
    """Keys whose scores are -infinity add nothing; where all are, zeros."""
    q, cache, table, lengths, ptab, shared = make([40] * 3, [50, 45, 60], 4, 2, 64, 8, dtype)
    q[1] = 0
    q[1, :, 0] = 1.0
    cache.k[..., 0] = -float("inf")
    q[0, :, 0] = q[0, :, 0].abs()
    q[2, :, 0] = q[2, :, 0].abs()
    out = api.attn_prefix(q, cache, table, lengths, ptab, shared)
    assert (out == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_tables_without_columns(dtype):
    """No prefix, or no own pages: the attention of single sequences, and zeros."""
    q, cache, table, lengths, ptab, shared = make([0] * 3, [40, 1, 70], 4, 2, 64, 8, dtype)
    check(q, cache, table, lengths, ptab[:0], shared)
    check(q, cache, table, lengths, ptab[:0], shared + 50)
    q, cache, table, lengths, ptab, shared = make([70] * 3, [70] * 3, 4, 2, 64, 8, dtype)
    check(q, cache, table[:, :0].contiguous(), lengths, ptab, shared)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_over_its_queries(dtype):
    a = make([90] * 9, list(range(90, 135, 5)), 8, 2, 64, 16, dtype)
    want = api.attn_prefix(*a)
    assert torch.equal(api.attn_prefix(*a, out=a[0]), want)
    # queries in rows of a wider tensor, the result where they begin
    q = want.new_empty((9, 24, 64))
    q[:, :8] = make([90] * 9, list(range(90, 135, 5)), 8, 2, 64, 16, dtype)[0]
    out = q.view(-1)[:9 * 8 * 64].view(9, 8, 64)
    assert torch.equal(api.attn_prefix(q[:, :8], *a[1:], out=out), want)


def test_like_single_sequences():
    """The same batch through attn_decode, whose own rounding may differ by its last bit."""
    q, cache, table, lengths, ptab, shared = make([500] * 12, list(range(500, 860, 30)), 8, 2, 128,
                                                  16, F32)
    full = table.clone()
    for b in range(12):
        full[b, :31] = ptab[:31]      # whole pages
    a = check(q, cache, table, lengths, ptab, shared)
    whole = torch.full((12,), 496, dtype=I32, device=DEV)
    has = lengths > 500
    for t in (cache.k, cache.v):
        t[table[has, 31].long(), :4] = t[ptab[31].long(), :4]
    b = check(q[has], cache, table[has], lengths[has], ptab, whole[has])
    c = api.attn_decode(q[has], cache, full[has].contiguous(), lengths[has])
    assert (a[has] - b).abs().max() < 1e-5 and (b - c).abs().max() < 1e-5


def test_prefix_past_32_bit_offsets():
    """Pages of both tables behind the first 2^31 elements of the cache."""
    H, D, page = 2, 128, 16
    n = (1 << 31) // (page * H * D) + 40
    cache = api.KVCache.empty(n, page, H, D, device=DEV)
    rows = torch.arange(n - 30, n, device=DEV)
    cache.k[rows] = torch.randn((30, page, H, D), device=DEV).to(BF)
    cache.v[rows] = torch.randn((30, page, H, D), device=DEV).to(BF)
    small = api.KVCache(cache.k[n - 30:].clone(), cache.v[n - 30:].clone())
    ptab = torch.arange(12, dtype=I32, device=DEV)
    table = torch.full((3, 18), -1, dtype=I32, device=DEV)
    table[:, 12:] = torch.arange(12, 30, dtype=I32, device=DEV).view(3, 6)
    lengths = torch.tensor([280, 193, 230], dtype=I32, device=DEV)
    shared = torch.full((3,), 192, dtype=I32, device=DEV)
    q = torch.randn((3, 8, D), device=DEV).to(BF)
    off = n - 30
    got = api.attn_prefix(q, cache, table + off, lengths, ptab + off, shared)
    assert torch.equal(got, api.attn_prefix(q, small, table, lengths, ptab, shared))


@pytest.mark.parametrize("Hq,H", [(1, 1), (34, 2)])
def test_the_most_sequences(Hq, H):
    """65535 sequences behind three shared tokens, each with one or no token of its own in
    pages of one token, and two tiles of heads where there are 17 to a key head."""
    B, D, G = 65535, 8, Hq // H
    torch.manual_seed(Hq)
    cache = api.KVCache.empty(B + 3, 1, H, D, F32, DEV)
    cache.k.normal_()
    cache.v.normal_()
    q = torch.randn((B, Hq, D), device=DEV)
    order = torch.randperm(B + 3, device=DEV).to(I32)
    table = torch.full((B, 4), -1, dtype=I32, device=DEV)
    table[:, 3] = order[3:]
    lengths = 3 + (torch.arange(B, device=DEV) % 3 > 0).to(I32)
    out = api.attn_prefix(q, cache, table, lengths, order[:3].contiguous(),
                          torch.full((B,), 3, dtype=I32, device=DEV))
    at = order.long()
    k, v = (torch.cat([t[at[:3], 0].double().expand(B, 3, H, D), t[at[3:], 0].double()[:, None]], 1)
            .permute(0, 2, 1, 3) for t in (cache.k, cache.v))
    x = q.double().view(B, H, G, 1, D)
    s = (x * k[:, :, None]).sum(-1) * D ** -0.5
    s[lengths == 3, :, :, 3] = -float("inf")
    p = torch.softmax(s, -1)
    want = (p[..., None] * v[:, :, None]).sum(3).view(B, Hq, D)
    # scores of 8 products: off by 9 2^-24 of the sum of |products|; a weight by twice that, the
    # exponents' own 2^-22, the joins' products and the sums of 4 keys
    ds = 9 * 2.0 ** -24 * (x * k[:, :, None]).abs().sum(-1).amax(-1) * D ** -0.5
    mag = (p[..., None] * v[:, :, None].abs()).sum(3)
    err = mag * (2 * ds[..., None] + 2.0 ** -20)
    assert ((out.double() - want).abs() <= err.view(B, Hq, D)).all()


def test_graphs_over_one_workspace_and_another_stream():
    """Two captured calls over one workspace, replayed in turn with eager work between,
    follow their lengths, shares and queries."""
    sets = [make([300] * 5, [310, 300, 450, 333, 301], 8, 2, 128, 16, BF, seed=i) for i in range(2)]
    need = api.attn_prefix_workspace(5, 8, sets[0][1], 300, 200)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    outs, graphs = [torch.empty_like(a[0]) for a in sets], []
    kw = dict(max_prefix=300, max_rest=200)
    for a, out in zip(sets, outs):
        api.attn_prefix(*a, out=out, workspace=ws, **kw)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            api.attn_prefix(*a, out=out, workspace=ws, **kw)
        graphs.append(g)
    s = torch.cuda.Stream()
    for i in range(4):
        ws.fill_(255)
        for a in sets:
            a[0].normal_()
            a[3].copy_(torch.tensor([310, 300 - i, 450, 310 + i, 0], dtype=I32))
            a[5].copy_(torch.tensor([300, 300, 300, 300, 300], dtype=I32))
        for g, out in zip(graphs, outs):
            out.fill_(-7)
            g.replay()
        torch.cuda.synchronize()
        for a, out in zip(sets, outs):
            other = api.attn_prefix(*a, stream=s, **kw)
            torch.cuda.synchronize()
            assert torch.equal(out, other)
            check(*a, **kw)
