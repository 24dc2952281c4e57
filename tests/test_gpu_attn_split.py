"""Attention over the paged cache whose keys are divided over all workgroups: shares
of thousands of keys (several rounds of the row offsets held at a time), that begin
inside a key head's keys, hold several key heads' or only masked ones.  Pages that
no token is read from hold NaN, and the workspace is NaN before every call.

References are sums in binary64 on the GPU, one head at a time."""
import numpy as np
import pytest
import torch

import decoder_ref as ref
from layer_cases import DEV
from paper_2504_15299_amd import api

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
NAN = float("nan")


class Case:
    """Sequences of the given lengths in random pages, with a workspace for all of them."""

    def __init__(self, lengths, Hq, H, D, page, dtype, seed=0, fill="random"):
        g = torch.Generator(DEV).manual_seed(seed)
        self.H, self.D, self.page = H, D, page
        width = -(-max(lengths) // page)
        used = [-(-n // page) for n in lengths]
        pool = sum(used) + 3
        ids = torch.randperm(pool, generator=g, device=DEV).to(I32)
        self.table = torch.full((len(lengths), width), -7, dtype=I32, device=DEV)
        k = torch.full((pool, page, H, D), NAN, dtype=dtype, device=DEV)
        v = torch.full_like(k, NAN)
        at = 0
        for b, (n, u) in enumerate(zip(lengths, used)):
            self.table[b, :u] = ids[at:at + u]
            at += u
            spots = self.spots(b, n)
            k.view(-1, H, D)[spots] = torch.randn((n, H, D), generator=g, device=DEV).to(dtype)
            if fill == "random":
                new = torch.randn((n, H, D), generator=g, device=DEV)
            else:
                new = torch.zeros((n, H, D), device=DEV)
                if n:
                    where = torch.randint(0, n, (200, H, D), generator=g, device=DEV)
                    sign = torch.randint(0, 2, (200, H, D), generator=g, device=DEV) * 2.0 - 1
                    new.scatter_(0, where, sign)
            v.view(-1, H, D)[spots] = new.to(dtype)
        self.cache = api.KVCache(k, v)
        self.lengths = torch.tensor(lengths, dtype=I32, device=DEV)
        self.q = torch.randn((len(lengths), Hq, D), generator=g, device=DEV).to(dtype)
        self.longest = max(lengths)
        need = api.attn_decode_workspace(len(lengths), Hq, self.cache, self.longest)
        self.ws = torch.empty(need, dtype=torch.uint8, device=DEV)

    def spots(self, b, n, first=0):
        j = torch.arange(first, n, device=DEV)
        return self.table[b].long()[j // self.page] * self.page + j % self.page

    def run(self, ws=None, used=True, **kw):
        """The call, over a workspace whose parts were NaN and must have been written."""
        ws = self.ws if ws is None else ws
        ws.fill_(255)
        kw = {"max_len": self.longest, "q": self.q, **kw}
        out = api.attn_decode(kw.pop("q"), self.cache, self.table, self.lengths, workspace=ws, **kw)
        assert bool((ws != 255).any()) == used
        return out

    def keys_of_a_share(self, dtype):
        """The keys of all key heads over the 256 or 512 shares."""
        units = len(self.lengths) * self.H
        return int(self.lengths.sum()) * self.H // (512 if self.D <= 64 or units > 512 else 256)

    def want(self, scale, window=0, path=0):
        """(result, bound on the error before the result's rounding), heads of pages that
        are not there left out.  A score of D products is off by 2 U (D + 2) of the sum of
        their magnitudes, the exponent by 8 U of its size, a probability and the sum of all
        relatively by twice that, a sum by 2 U per addition on a term's way through it, of
        which `path` counts the most (three pieces of bf16 probabilities)."""
        B, Hq, D = self.q.shape
        out = torch.zeros((B, Hq, D), dtype=torch.float64, device=DEV)
        err, G, pages = torch.zeros_like(out), Hq // self.H, self.cache.n_pages
        for b, n in enumerate(self.lengths.tolist()):
            n = min(n, self.table.shape[1] * self.page)
            first = max(0, n - window) if window else 0
            j = torch.arange(first, n, device=DEV)
            p = self.table[b].long()[j // self.page]
            ok = (p >= 0) & (p < pages)
            at = p[ok] * self.page + j[ok] % self.page
            if not len(at):
                continue
            for h in range(self.H):
                k, v = (t.view(-1, self.H, D)[at, h].double() for t in (self.cache.k, self.cache.v))
                qs = self.q[b, h * G:(h + 1) * G].double()
                s = qs @ k.t().contiguous() * scale
                off = (qs.abs() @ k.abs().t().contiguous()).amax(1, keepdim=True) * abs(scale) * \
                    2 * ref.U * (D + 2) + 8 * ref.U * s.abs().amax(1, keepdim=True)
                w = torch.exp(s - s.amax(1, keepdim=True))  # (exact where the scale is 0)
                total = w.sum(1, keepdim=True)
                out[b, h * G:(h + 1) * G] = (w @ v) / total
                err[b, h * G:(h + 1) * G] = (2 * torch.expm1(2 * off) + 2 * ref.U * path) * \
                    (w @ v.abs()) / total
        return out, err


def close(got, want, err=0.0):
    assert got.shape == want.shape
    bad = ~((got.double() - want).abs() <= err + (ref.HALF[got.dtype] + 8 * ref.U) * want.abs())
    assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:3].tolist())


# one or two long sequences, some hundred that end inside shares, empty and short ones
# between, key heads with more than 16 query heads, dimensions that are filled up
LAYOUTS = {
    "two long": ([200001, 37, 0, 151010], 4, 2, 128, 48),
    "heads": ([60000, 1, 33333, 50000, 20000, 59999], 32, 8, 128, 64),
    "segments": ([1500 + 97 * i % 2600 for i in range(100)], 16, 8, 128, 16),
    "one head": ([800003], 5, 1, 64, 24),
    "padded": ([150000, 90001], 20, 1, 80, 16),
    "wide": ([70000, 0, 50001], 34, 2, 256, 16),
}


@pytest.mark.parametrize("name", LAYOUTS)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_every_key_counts_once(name, dtype):
    """With scale 0 every probability is 1 and the result the mean of the values, of
    which each dimension has 200 of 1 or -1: multiples of 2^-16 (the last piece of 1) of
    at most 200, so every sum is exact and the result has its own roundings only."""
    c = Case(*LAYOUTS[name], dtype, fill="few")
    assert c.keys_of_a_share(dtype) > 3 * 512 or name in ("wide", "padded")
    want, _ = c.want(0.0)
    close(c.run(scale=0.0), want)


@pytest.mark.parametrize("name", LAYOUTS)
@pytest.mark.parametrize("dtype", [BF, F32])
def test_long_shares(name, dtype):
    """A term goes through the additions of one wave's quarter of a share, three a key,
    then four waves' and at most 512 parts'."""
    c = Case(*LAYOUTS[name], dtype, seed=1)
    scale = c.D ** -0.5
    close(c.run(scale=scale), *c.want(scale, path=3 * c.keys_of_a_share(dtype) // 4 + 3 * 32 + 520))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_window_over_long_shares(dtype):
    window = 140000
    c = Case([200001, 37, 150000], 4, 2, 128, 16, dtype, seed=2, fill="few")
    close(c.run(scale=0.0, window=window), c.want(0.0, window)[0])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_longer_than_expected(dtype):
    """max_len only divides the work."""
    c = Case([120000, 90000], 4, 2, 128, 16, dtype, seed=3, fill="few")
    close(c.run(scale=0.0, max_len=5000), c.want(0.0)[0])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_shares_whose_pages_are_all_masked(dtype):
    """The first shares of a sequence, some in its middle and its last ones have no
    page in the cache; another sequence has none at all."""
    c = Case([300000, 100000, 160000], 4, 1, 128, 16, dtype, seed=4, fill="few")
    share = c.keys_of_a_share(dtype) // 16
    c.table[0, :3 * share] = -1
    c.table[0, 60 * share:63 * share + 5] = 2 ** 31 - 1
    c.table[0, -4 * share:] = c.cache.n_pages
    c.table[1] = -1
    out = c.run(scale=0.0)
    close(out, c.want(0.0)[0])
    assert (out[1] == 0).all() and (out[0] != 0).any()
    out = c.run()
    close(out, *c.want(128 ** -0.5, path=3 * 16 * share // 4 + 3 * 32 + 520))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_infinities_in_one_share(dtype):
    """An infinite value reaches the joined result with its sign, a score that is no
    number its own query heads alone; scores of -infinity in all shares but one leave
    that one's mean, in all of them zeros."""
    c = Case([200000, 200000, 120000, 120000, 700], 6, 2, 128, 16, dtype, seed=5, fill="few")
    clean = c.run(scale=1.0)
    k, v = (t.view(-1, 2, 128) for t in (c.cache.k, c.cache.v))
    at = c.spots(0, 200000)
    v[at[150001], 0, 5], v[at[12345], 0, 6] = float("inf"), -float("inf")
    k[c.spots(1, 200000)[99999], 1, 3] = NAN
    c.q[2:4, :, 0] = 1.0
    k[c.spots(2, 120000)[:100000], :, 0] = -float("inf")
    k[c.spots(3, 120000), :, 0] = -float("inf")
    out = c.run(scale=1.0)
    assert (out[0, :3, 5] == float("inf")).all() and (out[0, :3, 6] == -float("inf")).all()
    same = torch.ones_like(out, dtype=torch.bool)
    same[0, :3, 5:7] = False
    same[1, 3:] = False
    same[2:4] = False
    assert torch.equal(out[same], clean[same])
    assert torch.isnan(out[1, 3:]).all()
    assert (out[3] == 0).all() and torch.isfinite(out[2]).all()
    # the sequence without its first keys
    rest = c.table.clone()
    rest[2, :100000 // 16] = -1
    alone = api.attn_decode(c.q, c.cache, rest, c.lengths, scale=1.0, max_len=100)
    # U for each of the two orders of the same sums, of magnitudes of up to 1
    room = 4 * ref.U * (3 * 120000 / 4) * alone[2].float().abs().amax() + ref.HALF[dtype] * 2
    assert ((out[2].float() - alone[2].float()).abs() <= room).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strided_queries(dtype):
    c = Case([100000, 130001, 20], 4, 2, 64, 16, dtype, seed=6)
    wide = torch.full((3, 9, 64), NAN, dtype=dtype, device=DEV)
    wide[:, 2:6] = c.q
    assert torch.equal(c.run(q=wide[:, 2:6]), c.run())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_two_streams_with_a_workspace_each(dtype):
    cases = [Case([100000, 3000, 40000], 8, 2, 128, 16, dtype, seed=s) for s in (7, 8)]
    want = [c.run() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    for c in cases:
        c.ws.fill_(255)
    torch.cuda.synchronize()
    got = [[api.attn_decode(c.q, c.cache, c.table, c.lengths, max_len=c.longest, workspace=c.ws, stream=s)
            for c, s in zip(cases, streams)] for _ in range(4)]
    torch.cuda.synchronize()
    for pair in got:
        for x, y in zip(pair, want):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_captured_call_follows_its_inputs(dtype):
    c = Case([150000, 60000, 3000], 4, 2, 128, 16, dtype, seed=9)
    out = torch.empty_like(c.q)
    c.run(out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        api.attn_decode(c.q, c.cache, c.table, c.lengths, max_len=c.longest, out=out, workspace=c.ws)
    other = torch.empty_like(c.ws)
    for n in ([150000, 60000, 3000], [3, 0, 2999], [149999, 1, 0], [100000, 60000, 2000]):
        c.lengths.copy_(torch.tensor(n, dtype=I32))
        c.q.normal_()
        c.ws.fill_(255)
        out.fill_(-7)
        g.replay()
        got = out.clone()
        want = c.run(ws=other)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
