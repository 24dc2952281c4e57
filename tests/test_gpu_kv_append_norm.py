"""New tokens into the paged cache with the norms of their query and key heads and
rotations of part of a head: every written row against binary64, every other row left
as it was."""
import numpy as np
import pytest
import torch

import decoder_ref as ref
import step_ref as step
from layer_cases import DEV
from paper_2504_15299_amd import api

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def gpu(a):
    return None if a is None else torch.from_numpy(a).to(DEV)


def f64(a):
    return None if a is None else a.astype(np.float64)


def angles(n_rot, half, rng):
    a = rng.uniform(-4, 4, (n_rot, half))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def run(N, seqs, H, Hq, D, rot, x_dtype=BF, dtype=BF, interleaved=False, page=5, norms="qk",
        in_place=False, order="pthd", eps=1e-6, size=1.0):
    rng = np.random.default_rng(N + D + rot)
    width = -(-N // (seqs * page)) + 2
    pool = seqs * width + 2
    shape = [{"p": pool, "t": page, "h": H, "d": D}[c] for c in order]
    cache = api.KVCache(*(torch.randn(shape, device=DEV).to(dtype)
                          .permute([order.index(c) for c in "pthd"]) for _ in range(2)))
    k0, v0 = cache.k.clone(), cache.v.clone()
    table = rng.permutation(pool)[:seqs * width].reshape(seqs, width).astype(np.int32)
    spots = rng.permutation(seqs * width * page)[:N]
    seq, pos = (spots // (width * page)).astype(np.int32), (spots % (width * page)).astype(np.int32)
    cos, sin = angles(width * page, rot // 2, rng) if rot else (None, None)
    qw, kw = ((1 + rng.standard_normal(D) * 0.3).astype(np.float32) if n in norms else None
              for n in "qk")
    qkv = ref.as_type(rng.standard_normal((N, Hq + 2 * H, D)) * size, x_dtype).to(DEV)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    if in_place:
        q = q.contiguous()
    q64, k64, v64 = ref.f64(q), ref.f64(k), ref.f64(v)
    out = api.kv_append_norm(q if Hq else None, k, v, cache, gpu(table), gpu(pos), gpu(seq),
                             q_weight=gpu(qw), k_weight=gpu(kw), eps=eps, cos=gpu(cos),
                             sin=gpu(sin), interleaved=interleaved, q_out=q if in_place else None)
    at = (torch.from_numpy(table[seq, pos // page].astype(np.int64)),
          torch.from_numpy((pos % page).astype(np.int64)))

    def want(x, w):
        return step.rotate(*step.head_norm(x, f64(w), eps), f64(cos), f64(sin), pos, interleaved)

    ref.close(cache.k[at], *want(k64, kw), dtype, "k")
    ref.close(cache.v[at], v64, np.zeros_like(v64), dtype, "v")
    if Hq:
        ref.close(out, *want(q64, qw), dtype, "q")
    else:
        assert out is None
    k0[at], v0[at] = cache.k[at], cache.v[at]
    assert torch.equal(cache.k, k0) and torch.equal(cache.v, v0)


@pytest.mark.parametrize("D,rot", [(8, 4), (8, 8), (8, 0), (16, 16), (24, 12), (24, 24), (40, 40),
                                   (64, 16), (72, 20), (80, 80), (80, 20), (96, 48), (128, 128),
                                   (128, 32), (128, 36), (136, 8), (192, 64), (248, 100),
                                   (256, 256), (256, 64), (256, 4), (256, 8)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("x_dtype,dtype", [(BF, BF), (F32, F32), (F32, BF), (BF, F32)])
def test_dims_rotations_and_types(D, rot, interleaved, x_dtype, dtype):
    run(N=9, seqs=3, H=2, Hq=6, D=D, rot=rot, x_dtype=x_dtype, dtype=dtype,
        interleaved=interleaved)


@pytest.mark.parametrize("norms", ["", "q", "k"])
@pytest.mark.parametrize("rot", [0, 32, 64])
def test_norms_of_either(norms, rot):
    run(N=7, seqs=2, H=2, Hq=3, D=64, rot=rot, norms=norms, x_dtype=F32, dtype=F32)


@pytest.mark.parametrize("H,Hq", [(1, 0), (1, 1), (1, 7), (8, 64), (5, 5)])
def test_heads(H, Hq):
    run(N=6, seqs=2, H=H, Hq=Hq, D=64, rot=64)
    run(N=6, seqs=2, H=H, Hq=Hq, D=128, rot=64, interleaved=True)


# rows that are stored past the caches, and more tokens than a grid has
@pytest.mark.parametrize("N,seqs,D,rot", [(300, 5, 8, 4), (300, 5, 80, 80), (300, 5, 128, 32),
                                          (65535 + 73, 64, 8, 8)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_tokens(N, seqs, D, rot, dtype):
    run(N=N, seqs=seqs, H=1, Hq=2, D=D, rot=rot, x_dtype=dtype, dtype=dtype, page=32)


# waves that keep some heads of 3 to 17 waves' worth over several tokens
@pytest.mark.parametrize("N,H,Hq,D,rot", [(5001, 3, 11, 128, 128), (1700, 3, 11, 80, 20),
                                          (9001, 2, 5, 64, 32)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_waves_that_stay(N, H, Hq, D, rot, dtype):
    run(N=N, seqs=4, H=H, Hq=Hq, D=D, rot=rot, x_dtype=dtype, dtype=dtype, page=32)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,rot,interleaved", [(64, 64, False), (64, 32, False), (80, 20, True),
                                               (256, 128, False), (256, 4, False)])
def test_in_place(dtype, D, rot, interleaved):
    run(N=40, seqs=3, H=2, Hq=5, D=D, rot=rot, x_dtype=dtype, dtype=dtype, interleaved=interleaved,
        in_place=True)


@pytest.mark.parametrize("order", ["phtd", "hptd"])
def test_orders(order):
    run(N=33, seqs=3, H=4, Hq=4, D=128, rot=128, order=order)


@pytest.mark.parametrize("size,eps", [(1e-8, 1e-6), (1e-15, 0.0), (1e15, 1e-6), (1.0, 100.0)])
def test_sizes_and_eps(size, eps):
    run(N=9, seqs=3, H=2, Hq=2, D=128, rot=128, x_dtype=F32, dtype=F32, size=size, eps=eps)


def test_without_norms_it_is_the_plain_append():
    """Half layout over the whole head, no weights: kv_append, to the last bit."""
    rng = np.random.default_rng(1)
    cos, sin = (gpu(a) for a in angles(12, 32, rng))
    qkv = torch.randn((4, 8, 64), device=DEV).to(BF)
    table = torch.tensor([[2, 0, 1], [5, 3, 4]], dtype=I32, device=DEV)
    pos, seq = (torch.tensor(a, dtype=I32, device=DEV) for a in ([11, 3, 0, 7], [0, 1, 1, 0]))
    res = []
    for fn in (api.kv_append, api.kv_append_norm):
        c = api.KVCache(torch.zeros((6, 4, 2, 64), dtype=BF, device=DEV),
                        torch.zeros((6, 4, 2, 64), dtype=BF, device=DEV))
        res.append((fn(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], c, table, pos, seq, cos=cos, sin=sin),
                    c.k, c.v))
    for a, b in zip(*res):
        assert torch.equal(a, b)


@pytest.mark.parametrize("rotary", [True, False])
def test_tokens_without_a_place_are_skipped(rotary):
    """Their query rows are normed, rotated where the rotation has their row."""
    D, H, page = 16, 2, 4
    cache = api.KVCache(*(torch.randn((6, page, H, D), device=DEV) for _ in range(2)))
    k0, v0 = cache.k.clone(), cache.v.clone()
    table = torch.tensor([[0, 7, -1], [6, 2, -2147483648]], dtype=I32, device=DEV)
    # beyond the row, negative, page 7 of 6, page -1, sequence outside, page 6 of 6, past
    # the rotation's rows, written
    pos = torch.tensor([12, -1, 5, 9, 0, 0, 0, 11, 6], dtype=I32, device=DEV)
    seq = torch.tensor([0, 0, 0, 0, 2, -1, 1, 1, 1], dtype=I32, device=DEV)
    rng = np.random.default_rng(0)
    cos, sin = angles(10, D // 2, rng) if rotary else (None, None)
    w = (1 + rng.standard_normal(D) * 0.3).astype(np.float32)
    x = rng.standard_normal((9, 3 * H, D)).astype(np.float32)
    xt = gpu(x)
    out = api.kv_append_norm(xt[:, :H], xt[:, H:2 * H], xt[:, 2 * H:], cache, table, pos, seq,
                             q_weight=gpu(w), k_weight=gpu(w), cos=gpu(cos), sin=gpu(sin))
    p = pos.cpu().numpy()
    n, err = step.head_norm(f64(x[:, :2 * H]), f64(w), 1e-6)
    r, rerr = step.rotate(n, err, f64(cos), f64(sin), np.clip(p, 0, 9), False)
    inside = ((p >= 0) & (p < 10))[:, None, None]
    ref.close(out, np.where(inside, r, n)[:, :H], np.where(inside, rerr, err)[:, :H], F32, "q")
    ref.close(cache.k[2, 2], r[8, H:], rerr[8, H:], F32, "k")
    assert torch.equal(cache.v[2, 2], xt[8, 2 * H:])
    k0[2, 2], v0[2, 2] = cache.k[2, 2], cache.v[2, 2]
    assert torch.equal(cache.k, k0) and torch.equal(cache.v, v0)


def test_another_stream():
    cache = api.KVCache.empty(4, 4, 1, 64, device=DEV)
    qkv = torch.randn((2, 3, 64), device=DEV).to(BF)
    table = torch.arange(4, dtype=I32, device=DEV).view(2, 2)
    pos, w = torch.tensor([3, 4], dtype=I32, device=DEV), torch.ones(64, device=DEV)
    a = (qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], cache, table, pos)
    want = api.kv_append_norm(*a, q_weight=w)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = api.kv_append_norm(*a, q_weight=w, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_pages_past_32_bit_offsets():
    """Pages behind the first 2^31 elements of the cache take what those of a small one do."""
    H, Hq, D, page = 2, 4, 128, 16
    n = (1 << 31) // (page * H * D) + 10
    torch.manual_seed(1)
    qkv = torch.randn((6, Hq + 2 * H, D), device=DEV).to(BF)
    w, table = torch.rand(D, device=DEV), torch.tensor([[3, 0], [5, 7]], dtype=I32, device=DEV)
    pos = torch.tensor([0, 15, 31, 3, 4, 20], dtype=I32, device=DEV)
    seq = torch.tensor([0, 0, 0, 1, 1, 1], dtype=I32, device=DEV)
    got = []
    for pages, off in ((n, n - 8), (8, 0)):
        c = api.KVCache(*(torch.zeros((pages, page, H, D), dtype=BF, device=DEV) for _ in range(2)))
        q = api.kv_append_norm(qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:], c, table + off, pos,
                               seq, q_weight=w, k_weight=w)
        got.append((q, c.k[off:].clone(), c.v[off:].clone(), c.k[:off].any().item()))
    for a, b in zip(got[0][:3], got[1][:3]):
        assert torch.equal(a, b)
    assert not got[0][3] and got[1][1].any()
