"""Calls of the decode operators that only their surroundings make hard: other
streams with memory just freed, the largest sizes, results over their inputs."""
import pytest
import torch

from layer_cases import DEV
from paper_2504_15299_amd import api

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def cache_of(n_pages, page, H, D, dtype=BF):
    c = api.KVCache.empty(n_pages, page, H, D, dtype, DEV)
    c.k.normal_()
    c.v.normal_()
    return c


def on_stream(name, s):
    """One call of the operator on stream s, its result and workspace its own."""
    cache = cache_of(8, 16, 2, 64)
    table = torch.arange(8, dtype=I32, device=DEV).view(2, 4)
    q = torch.randn((2, 4, 64), dtype=BF, device=DEV)
    pos = torch.tensor([3, 60], dtype=I32, device=DEV)
    w = api.linear_pack(torch.randn((256, 128), device=DEV), api.Linear.empty(256, 128, 128, DEV))
    x = torch.randn((2, 128), dtype=BF, device=DEV)
    big, y = torch.randn((2, 256), device=DEV), torch.randn((2, 256), device=DEV)
    return {
        "linear": lambda: api.linear_forward(x, w, stream=s),
        "kv_append": lambda: api.kv_append(q, q[:, :2], q[:, 2:], cache, table, pos, stream=s),
        "attn": lambda: api.attn_decode(q, cache, table, pos, stream=s),
        "norm": lambda: api.block_norm(big.clone(), y, stream=s),
    }[name]


@pytest.mark.parametrize("name", ["linear", "kv_append", "attn", "norm"])
def test_result_on_another_stream_does_not_take_memory_in_use(name):
    """2 x 256 bf16 of the current stream, freed while work on it is still to
    run: the call's result on the other stream must not be there."""
    s = torch.cuda.Stream()
    run = on_stream(name, s)
    slow = torch.ones(1 << 28, device=DEV)
    torch.cuda.synchronize()
    old = torch.full((2, 256), 7.0, dtype=BF, device=DEV)
    torch.cuda.synchronize()
    for _ in range(40):
        slow.mul_(1.0)
    kept = old.clone()
    del old
    out = run()
    torch.cuda.synchronize()
    assert out.numel() == 512 and (kept == 7.0).all()


def test_linear_of_the_most_tokens():
    """2^20 tokens, which every division of the work has to reach with its grid."""
    T = 1 << 20
    x = torch.randn((T, 128), device=DEV).to(BF)
    for group in (32, 128):
        w = api.linear_pack(torch.randn((16, 128), device=DEV), api.Linear.empty(16, 128, group, DEV))
        y = api.linear_forward(x, w)
        for t in (0, 12345, T - 20):
            assert torch.equal(y[t:t + 20], api.linear_forward(x[t:t + 20].contiguous(), w))


def test_norm_of_more_rows_than_a_grid_has():
    """A row of one value: h = x / |x|, x = x + y exact here."""
    T = (1 << 26) + 5
    x = (torch.arange(T, dtype=I32, device=DEV) % 31 - 15).to(F32)[:, None]
    y = torch.full((T, 1), 0.5, dtype=BF, device=DEV)
    want = x + 0.5
    h = api.block_norm(x, y, eps=0.0)
    assert torch.equal(x, want)
    assert torch.equal(h.float(), want.sign())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("max_len", [100, 5000])
def test_attention_over_its_queries(dtype, max_len):
    cache = cache_of(300, 16, 2, 128, dtype)
    table = torch.randperm(300, device=DEV).to(I32)[:300].view(3, 100)
    lengths = torch.tensor([1500, 40, 700], dtype=I32, device=DEV)
    q = torch.randn((3, 36, 128), device=DEV).to(dtype)
    want = api.attn_decode(q, cache, table, lengths, max_len=max_len)
    assert torch.equal(api.attn_decode(q, cache, table, lengths, max_len=max_len, out=q), want)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [7, 4096, 16384])
def test_norm_over_its_addend(d, dtype):
    x, y = torch.randn((300, d), device=DEV), torch.randn((300, d), device=DEV).to(dtype)
    w, x2 = torch.rand(d, device=DEV), x.clone()
    want = api.block_norm(x2, y, post_weight=w, pre_weight=w, h_dtype=dtype)
    h = api.block_norm(x, y, post_weight=w, pre_weight=w, h=y)
    assert torch.equal(x, x2) and torch.equal(h, want)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_of_one_head_over_many_parts(dtype):
    """A key head whose keys are divided over all workgroups, joined again, against
    the same keys as 40 sequences by their sums in binary64."""
    n, D = 40000, 64
    cache = cache_of(n // 16, 16, 1, D, dtype)
    table = torch.randperm(n // 16, device=DEV).to(I32)[None]
    q = torch.randn((1, 5, D), device=DEV).to(dtype)
    got = api.attn_decode(q, cache, table, torch.tensor([n - 3], dtype=I32, device=DEV))
    k, v = (t[table[0].long()].reshape(n, D)[:n - 3].double().cpu() for t in (cache.k, cache.v))
    s = (q[0].double().cpu() @ k.t()) * D ** -0.5
    p = torch.softmax(s, 1)
    want = p @ v
    # scores of 64 products in binary32: off by 64 2^-24 of the sum of |products|,
    # which is at most |q| |k|; a probability by twice that, a value sum by 2^-16 of
    # the sum of p |v| (two bf16 terms) and by 40000 2^-24 at most in binary32
    ds = 64 * 2.0 ** -24 * (q[0].double().cpu().norm(dim=1, keepdim=True) * k.norm(dim=1)).max() / 8
    mag = p @ v.abs()
    err = mag * (2 * ds + 2.0 ** -16 + n * 2.0 ** -24) + \
        want.abs() * torch.finfo(dtype).eps / 2 + 1e-30
    assert ((got[0].double().cpu() - want).abs() <= err).all()


def test_two_graphs_share_a_workspace():
    """Split calls captured over one workspace, replayed in turn with eager work
    between, follow their inputs: lengths, queries and the cache's new tokens."""
    B, H, D, page = 3, 2, 128, 16
    caches = [cache_of(B * 200, page, H, D) for _ in range(2)]
    table = torch.randperm(B * 200, device=DEV).to(I32).view(B, 200)
    qkv = torch.randn((B, 8 + 2 * H, D), device=DEV).to(BF)
    pos = torch.tensor([2500, 30, 1100], dtype=I32, device=DEV)
    lengths = pos + 1
    need = api.attn_decode_workspace(B, 8, caches[0], 3000)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    outs = [torch.empty((B, 8, D), dtype=BF, device=DEV) for _ in caches]

    def step(c, out, work):
        api.kv_append(None, qkv[:, 8:8 + H], qkv[:, 8 + H:], c, table, pos)
        api.attn_decode(qkv[:, :8], c, table, lengths, max_len=3000, out=out, workspace=work)

    graphs = []
    for c, out in zip(caches, outs):
        step(c, out, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(c, out, ws)
        graphs.append(g)
    for i in range(4):
        qkv.normal_()
        pos.copy_(torch.tensor([2600 + i, 31 * i, 1], dtype=I32))
        lengths.copy_(pos + 1)
        ws.fill_(255)
        for g, out in zip(graphs, outs):
            out.fill_(-7)
            g.replay()
        for c, out in zip(caches, outs):
            want = torch.empty_like(out)
            step(c, want, torch.empty_like(ws))
            torch.cuda.synchronize()
            assert torch.equal(out, want)
