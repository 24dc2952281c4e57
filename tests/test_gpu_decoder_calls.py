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
