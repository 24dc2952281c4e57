"""The norms around a block against binary64 within the bounds of their
arithmetic, and against d2moe_residual_rmsnorm where the two are the same."""
import numpy as np
import pytest
import torch

import decoder_ref as ref
from layer_cases import DEV
from paper_2504_15299_amd import api

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def check(T, d, y_dtype, h_dtype, post, pre, gate, x_scale, y_scale, seed=0, eps=1e-5):
    rng = np.random.default_rng(seed)
    size = 10.0 ** rng.integers(-3, 3, (T, 1))
    x = (rng.standard_normal((T, d)) * size).astype(np.float32)
    y = ref.as_type(rng.standard_normal((T, d)) * size, y_dtype)
    wp, wq = ((1 + rng.standard_normal(d) * 0.2).astype(np.float32) for _ in range(2))
    dev = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    g = None
    if gate:
        g = ref.as_type(rng.standard_normal((T, d) if "token" in gate else (d,)),
                        BF if "bf16" in gate else F32).to(DEV)
        if "strided" in gate:
            wide = torch.full((T, d + 5), float("nan"), dtype=g.dtype, device=DEV)
            wide[:, :d] = g
            g = wide[:, :d]
    buf = torch.full((T + 2, d), -77.0, device=DEV)
    out = torch.full((T + 2, d), -77.0, dtype=h_dtype or F32, device=DEV)
    buf[1:T + 1] = dev(x)
    h = api.block_norm(buf[1:T + 1], y.to(DEV), eps, dev(wq) if pre else None,
                       dev(wp) if post else None, g, x_scale, y_scale,
                       h=None if h_dtype is None else out[1:T + 1], h_dtype=h_dtype)
    want, hw, err, herr = ref.block_norm(
        x.astype(np.float64), ref.f64(y), eps, wp.astype(np.float64) if post else None,
        None if g is None else ref.f64(g), wq.astype(np.float64) if pre else None,
        np.float64(np.float32(x_scale)), np.float64(np.float32(y_scale)))
    ref.close(buf[1:T + 1], want, err, F32, "x")
    assert (buf[0] == -77).all() and (buf[T + 1] == -77).all()
    if h_dtype is None:
        assert h is None
    else:
        ref.close(h, hw, herr, h_dtype, "h")
        assert (out[0] == -77).all() and (out[T + 1] == -77).all()


# widths of every kernel, whole, ragged and at their borders
@pytest.mark.parametrize("d", [1, 2, 3, 4, 7, 64, 255, 256, 257, 1000, 1024, 1025, 2048, 2050,
                               4095, 4096, 4097, 8192, 16383, 16384])
@pytest.mark.parametrize("y_dtype,h_dtype", [(BF, BF), (F32, F32)])
def test_widths(d, y_dtype, h_dtype):
    check(3, d, y_dtype, h_dtype, True, True, "row f32", 0.9, 0.5, seed=d)


@pytest.mark.parametrize("d", [2049, 4000, 4096, 4098, 8189])
def test_many_rows(d):
    """Row counts from which the wide rows take other workgroups."""
    for T in (256, 257):
        check(T, d, BF, BF, True, True, "token bf16", 0.9, 0.5, seed=T)


# rows that are stored past the caches, of every width's workgroups, whole and ragged
@pytest.mark.parametrize("T,d", [(17000, 256), (20001, 250), (4200, 1000), (2100, 2048), (2117, 2041),
                                 (1030, 4096), (1031, 4093), (520, 8192), (600, 8190), (257, 16384),
                                 (300, 16381)])
@pytest.mark.parametrize("y_dtype,h_dtype", [(BF, BF), (F32, F32)])
def test_rows_beyond_the_caches(T, d, y_dtype, h_dtype):
    assert T * d > 1 << 22
    check(T, d, y_dtype, h_dtype, True, True, "token bf16", 0.9, 0.5, seed=d)
    check(T, d, y_dtype, h_dtype, d % 2 == 0, False, None, 1.0, 1.0, seed=T)


@pytest.mark.parametrize("T", [1, 2, 65, 301])
@pytest.mark.parametrize("gate", [None, "row bf16", "token bf16", "token f32",
                                  "token strided bf16", "token strided f32"])
def test_gates(T, gate):
    check(T, 200, BF, F32, T % 2 == 0, False, gate, 1.0, 1.0, seed=T)


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("pre", [True, False])
@pytest.mark.parametrize("y_dtype,h_dtype", [(BF, F32), (F32, BF), (BF, None), (F32, None)])
def test_parts(post, pre, y_dtype, h_dtype):
    check(5, 513, y_dtype, h_dtype, post, pre, None, -0.3, 2.0)


def test_plain_sum_is_the_residual_norm():
    x = torch.randn((9, 4096), device=DEV)
    y = torch.randn((9, 4096), device=DEV, dtype=BF)
    a, b = x.clone(), x.clone()
    ha = api.residual_rmsnorm(a, y, h_dtype=F32)
    hb = api.block_norm(b, y, h_dtype=F32)
    assert torch.equal(a, b)
    # the two sum the squares in another order: 40 U at most
    assert ((ha - hb).abs() <= 48 * ref.U * ha.abs()).all()


def test_zero_rows_and_zero_eps():
    x, y = torch.zeros((2, 64), device=DEV), torch.zeros((2, 64), device=DEV)
    h = api.block_norm(x, y, 1e-5, post_weight=torch.ones(64, device=DEV), h_dtype=F32)
    assert (h == 0).all() and (x == 0).all()
    check(3, 64, F32, F32, True, True, None, 1.0, 1.0, eps=0.0)


def test_rows_that_are_not_finite_stay_alone():
    x = torch.randn((4, 300), device=DEV)
    y = torch.randn((4, 300), device=DEV)
    a, b = x.clone(), x.clone()
    want = api.block_norm(a, y, h_dtype=F32)
    y[2, 7] = float("inf")
    got = api.block_norm(b, y, h_dtype=F32)
    keep = [0, 1, 3]
    assert torch.equal(got[keep], want[keep]) and torch.equal(a[keep], b[keep])
    assert not torch.isfinite(b[2, 7])


def test_rejects_wrong_arguments():
    x, y = torch.zeros((2, 8), device=DEV), torch.zeros((2, 8), device=DEV)
    for bad in (dict(y=y[:1]), dict(x=x.double()), dict(gate=torch.zeros(7, device=DEV)),
                dict(pre_weight=torch.zeros(7, device=DEV)), dict(h=torch.zeros((2, 7), device=DEV)),
                dict(post_weight=torch.zeros(8, device=DEV, dtype=BF)), dict(x=x.cpu())):
        with pytest.raises(ValueError):
            api.block_norm(**{**dict(x=x, y=y), **bad})
    wide = torch.zeros((2, 16385), device=DEV)
    with pytest.raises(api.D2MoEError) as e:
        api.block_norm(wide, wide.clone())
    assert e.value.status == api.EINVAL
