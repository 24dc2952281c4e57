"""4-bit linear layers on the GPU: the packed layout and the quantization
exactly, the product against binary64 within the bound of its arithmetic."""
import numpy as np
import pytest
import torch

import decoder_ref as ref
from layer_cases import DEV
from paper_2504_15299_amd import api

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def weights(rows, cols, group, seed=0):
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 16, (rows, cols), dtype=np.uint8)
    scales = (rng.random((rows, cols // group)) * 0.01 + 1e-4).astype(np.float16)
    zeros = rng.integers(0, 16, (rows, cols // group), dtype=np.uint8)
    return codes, scales, zeros


def packed(codes, scales, zeros, group):
    t = [None if a is None else torch.from_numpy(a).to(DEV) for a in (codes, scales, zeros)]
    return api.linear_pack_codes(*t, api.Linear.empty(*codes.shape, group, device=DEV))


def buffers(w):
    return (w.codes.cpu().numpy().view(np.uint32), w.scales.cpu().numpy().view(np.float16),
            w.zeros.cpu().numpy())


@pytest.mark.parametrize("rows,cols,group", [(1, 32, 32), (16, 128, 128), (17, 96, 32),
                                             (100, 192, 64), (33, 640, 128)])
@pytest.mark.parametrize("given_zeros", [True, False])
def test_layout_of_given_codes(rows, cols, group, given_zeros):
    codes, scales, zeros = weights(rows, cols, group)
    if not given_zeros:
        zeros[:] = 8
    w = packed(codes, scales, zeros if given_zeros else None, group)
    for got, want in zip(buffers(w), ref.linear_layout(codes, scales, zeros, group)):
        assert np.array_equal(got, want)


@pytest.mark.parametrize("rows,cols,group", [(5, 32, 32), (31, 192, 64), (64, 512, 128)])
def test_quantization(rows, cols, group):
    rng = np.random.default_rng(rows)
    W = rng.standard_normal((rows, cols), dtype=np.float32) * 0.02
    W[0, :group] = 0.0                       # a group of zeros: scale 1
    W[1, :group] = np.abs(W[1, :group])      # one sign only
    W[2, :group] = -np.abs(W[2, :group])
    W[3, 3] = 1e30                           # the scale overflows: 1
    w = api.linear_pack(torch.from_numpy(W).to(DEV), api.Linear.empty(rows, cols, group, DEV))
    want = ref.linear_quantize(W, group)
    for got, exp in zip(buffers(w), ref.linear_layout(*want, group)):
        assert np.array_equal(got, exp)


def test_a_weight_that_is_not_a_number():
    W = np.random.default_rng(0).standard_normal((20, 192), dtype=np.float32)
    W[3, 7], W[4, 64:] = np.nan, np.nan
    w = api.linear_pack(torch.from_numpy(W).to(DEV), api.Linear.empty(20, 192, 64, DEV))
    codes, scales, zeros = ref.linear_quantize(np.where(np.isnan(W), 0, W), 64)
    codes[np.isnan(W)] = 0
    for got, exp in zip(buffers(w), ref.linear_layout(codes, scales, zeros, 64)):
        assert np.array_equal(got, exp)


def check(T, rows, cols, group, x_dtype, y_dtype, bias, seed=0, shift=0.0):
    rng = np.random.default_rng(seed)
    codes, scales, zeros = weights(rows, cols, group, seed)
    w = packed(codes, scales, zeros, group)
    x = ref.as_type(rng.standard_normal((T, cols)) + shift, x_dtype)
    b = rng.standard_normal(rows).astype(np.float32) if bias else None
    guard = torch.full((T + 2, rows), -77.0, dtype=y_dtype, device=DEV)
    y = api.linear_forward(x.to(DEV), w, None if b is None else torch.from_numpy(b).to(DEV),
                           y=guard[1:T + 1])
    want, err = ref.linear(ref.f64(x), codes, scales, zeros, group, b)
    ref.close(y, want, err, y_dtype, (T, rows, cols, group))
    assert (guard[0] == -77).all() and (guard[T + 1] == -77).all()


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 32, 33, 64, 65, 130])
@pytest.mark.parametrize("x_dtype", [BF, F32])
def test_tokens(T, x_dtype):
    check(T, 48, 384, 128, x_dtype, x_dtype, bias=T % 2 == 0, seed=T)


@pytest.mark.parametrize("rows", [1, 15, 16, 17, 100, 1003])
@pytest.mark.parametrize("cols,group", [(32, 32), (96, 32), (64, 64), (192, 64), (1984, 64),
                                        (128, 128), (1152, 128), (4096, 128)])
def test_shapes(rows, cols, group):
    check(3, rows, cols, group, BF, F32, bias=True, seed=rows + cols)
    check(19, rows, cols, group, F32, BF, bias=False, seed=rows + cols)


# row counts from which workgroups of more rows and tokens are taken
@pytest.mark.parametrize("T,rows", [(17, 24000), (33, 24590), (65, 12290), (100, 6150), (4, 8200),
                                    (7, 16500), (16, 33000), (130, 1040)])
@pytest.mark.parametrize("cols,group", [(160, 32), (192, 64), (384, 128)])
@pytest.mark.parametrize("x_dtype", [BF, F32])
def test_many_rows(T, rows, cols, group, x_dtype):
    check(T, rows, cols, group, x_dtype, x_dtype, bias=True, seed=T)


@pytest.mark.parametrize("T,rows,cols,group", [(1, 141, 128, 128), (3, 100, 192, 64), (9, 65, 96, 32),
                                               (20, 300, 640, 128), (40, 12300, 128, 64)])
def test_float_activations_keep_their_precision(T, rows, cols, group):
    """Activations of one binade: their first eight bits are multiples of 2^-7, the
    sums of those times 16 + n, and of those times 16 + z, of 2^13 at most, so both
    are exact, also where they cancel (most codes equal their zero point).  What is
    left, below 2^-16 here, has in a group two sums of 2 * group terms of 31 2^-16 at
    most, each addition off by 2 U of the sum so far."""
    rng = np.random.default_rng(cols)
    codes, scales, zeros = weights(rows, cols, group)
    same = rng.random((rows, cols)) < 0.95
    codes[same] = np.repeat(zeros, group, 1)[same]
    x = 1 + rng.integers(0, 128, (T, cols)) / 128 + rng.uniform(0, 2.0 ** -16, (T, cols))
    x = x.astype(np.float32)
    y = api.linear_forward(torch.from_numpy(x).to(DEV), packed(codes, scales, zeros, group))
    x = x.astype(np.float64)
    want, _ = ref.linear(x, codes, scales, zeros, group)
    s = scales.astype(np.float64)
    w = np.repeat(s, group, 1) * (codes.astype(np.float64) - np.repeat(zeros, group, 1))
    err = (2 * ref.U * 2 * group * 2.0 ** -16) * (62 * group * s.sum(1)) + \
        (cols // group + 20) * ref.U * (np.abs(x) @ np.abs(w).T)
    assert (np.abs(y.double().cpu().numpy() - want) <= err).all()


# workgroups of 64 rows by 32 tokens
@pytest.mark.parametrize("T,rows", [(50, 5003), (17, 16000)])
@pytest.mark.parametrize("cols,group", [(64, 64), (1984, 64), (128, 128), (1152, 128)])
def test_workgroups_of_64_rows(T, rows, cols, group):
    check(T, rows, cols, group, BF, F32, bias=True, seed=cols)
    check(T, rows, cols, group, BF, BF, bias=False, seed=cols + 1)


# workgroups of 256 rows, the last of them partly filled
@pytest.mark.parametrize("cols,group", [(160, 32), (192, 64), (384, 128), (1152, 128)])
@pytest.mark.parametrize("x_dtype", [BF, F32])
def test_widest_workgroups(cols, group, x_dtype):
    check(66, 20010, cols, group, x_dtype, F32, bias=True, seed=cols)
    check(66, 20010, cols, group, x_dtype, BF, bias=False, seed=cols + 1)



# every division of the work, by tokens and rows
@pytest.mark.parametrize("rows", [5, 40, 4100, 6150, 9001, 17000])
@pytest.mark.parametrize("tokens", [1, 4, 7, 16, 64, None])
@pytest.mark.parametrize("cols,group", [(160, 32), (192, 64), (320, 64), (384, 128)])
@pytest.mark.parametrize("x_dtype", [BF, F32])
def test_every_weight_and_every_bit(rows, tokens, cols, group, x_dtype):
    """Token t is 0 but at column t, where it has all the bits of its type: a result is
    one weight times that.  Its pieces' products with 16 + n, and the sum of the smaller
    two, have at most 21 bits, all exact, and what the zero point takes off leaves each
    part exact; their sum and its product with the scale are rounded, U each, and all
    other terms are 0.  (The pieces of a binary32 activation: without the third 2^-17,
    2^7 U, would be missing.)  `tokens` at a time, None: all of them."""
    codes, scales, zeros = weights(rows, cols, group, seed=rows)
    w = packed(codes, scales, zeros, group)
    v = ref.as_type(np.random.default_rng(cols).uniform(1, 2, cols) * (-1.0) ** np.arange(cols), x_dtype)
    x = torch.diag(v).to(DEV)
    step = tokens or cols
    y = torch.cat([api.linear_forward(x[t:t + step], w, y_dtype=F32) for t in range(0, cols, step)])
    s = torch.from_numpy(scales).double().repeat_interleave(group, 1)
    z = torch.from_numpy(zeros).double().repeat_interleave(group, 1)
    want = ((s * (torch.from_numpy(codes).double() - z)).t() * v.double()[:, None]).to(DEV)
    assert ((y.double() - want).abs() <= 2.5 * ref.U * want.abs()).all()


@pytest.mark.parametrize("T,rows,cols,group", [(1, 40, 4096, 128), (16, 6144, 4096, 128), (17, 700, 4096, 64),
                                               (64, 6150, 4032, 64), (64, 16384, 2048, 128),
                                               (33, 6150, 4064, 32), (128, 4096, 14336, 128),
                                               (300, 4096, 4096, 64)])
@pytest.mark.parametrize("x_dtype", [BF, F32])
def test_whole_numbers_are_exact(T, rows, cols, group, x_dtype):
    """Activations and scales that are small whole numbers and powers of two: every
    product and sum, of 31 * 4 * 128 within a group and 15 * 4 * 2 * 14336 at the
    end, in units of 1 / 2, has less than 24 bits."""
    rng = np.random.default_rng(cols)
    codes, _, zeros = weights(rows, cols, group)
    scales = (2.0 ** rng.integers(-1, 2, (rows, cols // group))).astype(np.float16)
    x = torch.from_numpy(rng.integers(-4, 5, (T, cols))).to(x_dtype).to(DEV)
    b = torch.from_numpy(rng.integers(-9, 10, rows)).float().to(DEV)
    y = api.linear_forward(x, packed(codes, scales, zeros, group), b, y_dtype=F32)
    s = torch.from_numpy(scales).double().repeat_interleave(group, 1)
    z = torch.from_numpy(zeros).double().repeat_interleave(group, 1)
    W = (s * (torch.from_numpy(codes).double() - z)).to(DEV)
    assert torch.equal(y.double(), x.double() @ W.t().contiguous() + b.double())


@pytest.mark.parametrize("T", [1, 3, 5, 20])
@pytest.mark.parametrize("x_dtype", [BF, F32])
def test_long_rows(T, x_dtype):
    check(T, 40, 14336, 128, x_dtype, x_dtype, bias=False, seed=T)
    check(T, 40, 8256, 64, x_dtype, x_dtype, bias=False, seed=T)


def test_activations_with_a_large_mean():
    check(16, 64, 512, 128, BF, BF, bias=False, shift=30.0)
    check(16, 64, 512, 128, F32, F32, bias=False, shift=30.0)


def test_small_and_large_activations():
    """Binary32 activations over the exponents that a product can have."""
    codes, scales, zeros = weights(20, 256, 128)
    w = packed(codes, scales, zeros, 128)
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((6, 256)) * 10.0 ** np.array([-25, -10, 0, 5, 15, 30])[:, None]
         ).astype(np.float32)
    y = api.linear_forward(torch.from_numpy(x).to(DEV), w)
    ref.close(y, *ref.linear(x.astype(np.float64), codes, scales, zeros, 128), F32)


# every division of the work, its last column block one to three quarters filled
@pytest.mark.parametrize("T,rows", [(1, 20), (5, 5000), (20, 20), (20, 9000), (40, 12300), (17, 16000),
                                    (66, 20010)])
@pytest.mark.parametrize("cols,group", [(32, 32), (96, 32), (64, 64), (192, 64)])
@pytest.mark.parametrize("x_dtype", [BF, F32])
def test_large_activations_in_a_last_block_not_filled(T, rows, cols, group, x_dtype):
    """Eight activations of 1e36 under codes of 15: the sums of their group are 2.5e38
    at most, within binary32, and nothing may repeat them beyond that."""
    codes, scales, zeros = weights(rows, cols, group)
    codes[:, -8:] = 15
    x = np.random.default_rng(0).standard_normal((T, cols))
    x[:, -8:] = 1e36
    x = ref.as_type(x, x_dtype)
    y = api.linear_forward(x.to(DEV), packed(codes, scales, zeros, group))
    ref.close(y, *ref.linear(ref.f64(x), codes, scales, zeros, group), x_dtype)


@pytest.mark.parametrize("x_dtype", [BF, F32])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_a_token_that_is_not_finite_stays_alone(x_dtype, value):
    codes, scales, zeros = weights(20, 192, 64)
    w = packed(codes, scales, zeros, 64)
    x = torch.randn((18, 192), generator=torch.Generator().manual_seed(0)).to(x_dtype)
    clean = api.linear_forward(x.to(DEV), w)
    x[17, 100] = value
    y = api.linear_forward(x.to(DEV), w)
    assert torch.equal(y[:17], clean[:17])
    assert not torch.isfinite(y[17]).any()


def test_no_tokens():
    w = packed(*weights(20, 64, 64), 64)
    assert api.linear_forward(torch.empty((0, 64), device=DEV), w).shape == (0, 20)


def test_rejects_wrong_arguments():
    w = packed(*weights(20, 64, 64), 64)
    x = torch.zeros((2, 64), device=DEV)
    for bad in (x[:, :32], x.t().contiguous().t(), x.cpu()):
        with pytest.raises(ValueError):
            api.linear_forward(bad, w)
    with pytest.raises(TypeError):
        api.linear_forward(x.half(), w)
    with pytest.raises(ValueError):
        api.linear_forward(x, w, bias=torch.zeros(19, device=DEV))
    with pytest.raises(ValueError):
        api.linear_forward(x, w, y=torch.zeros((2, 19), device=DEV))
    odd = torch.zeros(2 * 64 + 1, device=DEV)[1:].view(2, 64)      # not 16-byte aligned
    with pytest.raises(api.D2MoEError) as e:
        api.linear_forward(odd, w)
    assert e.value.status == api.EINVAL


def test_results_do_not_change_between_calls_and_streams():
    codes, scales, zeros = weights(300, 1024, 128)
    w = packed(codes, scales, zeros, 128)
    x = torch.randn((40, 1024), device=DEV, dtype=BF)
    torch.cuda.synchronize()
    a = api.linear_forward(x, w)
    s = torch.cuda.Stream()
    b = api.linear_forward(x, w, stream=s)
    c = api.linear_forward(x[:7].contiguous(), w)
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    assert torch.equal(a[:7], c)       # a token's result does not go by the batch
