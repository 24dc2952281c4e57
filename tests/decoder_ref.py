"""Plain binary64 forms of the decode operators around the MoE layer (numpy),
with the error bounds that follow from the kernels' binary32 arithmetic.

Roundings: a result of type t is off by half a step, HALF[t] relative to its
value; a binary32 operation by U = 2^-24."""
import numpy as np
import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def as_type(a, dtype):
    """A torch tensor of the type nearest to the numpy array."""
    return torch.from_numpy(np.asarray(a, np.float32)).to(dtype)


# ---- 4-bit linear layers -------------------------------------------------------

def linear_quantize(W, group):
    """Eq. 2 at four bits, binary32: codes [rows][cols], scales (float16)
    and zero points [rows][cols/group]."""
    rows, cols = W.shape
    w = np.asarray(W, np.float32).reshape(rows, cols // group, group)
    lo, hi = np.minimum(w.min(2), np.float32(0)), np.maximum(w.max(2), np.float32(0))
    with np.errstate(over="ignore"):
        s = ((hi - lo) / np.float32(15)).astype(np.float16)
    s = np.where((s > 0) & np.isfinite(s), s, np.float16(1))
    sf = s.astype(np.float32)
    z = np.clip(np.rint(-lo / sf), 0, 15).astype(np.float32)
    n = np.clip(np.rint(w / sf[..., None] + z[..., None]), 0, 15)
    return n.reshape(rows, cols).astype(np.uint8), s, z.astype(np.uint8)


def linear_layout(codes, scales, zeros, group):
    """The packed buffers, from the layout's definition."""
    rows, cols = codes.shape
    RB, KB, GB = -(-rows // 16), -(-cols // 128), 128 // group
    full = np.zeros((RB * 16, KB * 128), np.uint32)
    full[:rows, :cols] = codes
    s = np.zeros((RB * 16, KB * GB), np.float16)
    s[:rows, :cols // group] = scales
    z = np.full((RB * 16, KB * GB), 16, np.uint8)
    z[:rows, :cols // group] += zeros
    words = np.zeros((RB, KB, 64, 4), np.uint32)
    for lane in range(64):
        for j in range(4):
            for e in range(8):
                c = 32 * j + 8 * (lane // 16) + e
                n = full.reshape(RB, 16, KB, 128)[:, lane % 16, :, c]
                words[:, :, lane, j] |= n << np.uint32(4 * (e // 2 + 4 * (e % 2)))
    order = (0, 2, 3, 1)
    return (words.reshape(-1), s.reshape(RB, 16, KB, GB).transpose(order).reshape(-1),
            z.reshape(RB, 16, KB, GB).transpose(order).reshape(-1))


def linear(x, codes, scales, zeros, group, bias=None):
    """(y, bound on the error before the result's own rounding) for x [T][cols].

    A group's two sums have at most 3 * group terms (three pieces per binary32
    activation) of at most 31 |x|, each addition off by at most 2 U of the sum
    of magnitudes so far; then the groups and the waves' parts are added, and the bias."""
    rows, cols = codes.shape
    g = cols // group
    w = codes.astype(np.float64).reshape(rows, g, group) - zeros[..., None]
    w = (w * scales.astype(np.float64)[..., None]).reshape(rows, cols)
    y = x @ w.T
    ax = np.abs(x).reshape(len(x), g, group).sum(2)
    mag = ax @ (scales.astype(np.float64) * 62).T
    err = 2 * U * 3 * group * mag + (g + 20) * U * (np.abs(x) @ np.abs(w).T)
    if bias is not None:
        y = y + bias
        err = err + 2 * U * np.abs(bias)
    return y, err


# ---- paged cache -----------------------------------------------------------------

def kv_append(x, cos, sin, pos):
    """Rotated rows of x [N][heads][D] (cos None: x) and the error bound."""
    if cos is None:
        return x, np.zeros_like(x)
    half = x.shape[2] // 2
    a, b = x[..., :half], x[..., half:]
    c, s = cos[pos][:, None], sin[pos][:, None]
    err = 3 * U * np.concatenate([np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)], 2)
    return np.concatenate([a * c - b * s, b * c + a * s], 2), err


def attn(q, k, v, table, lengths, scale, window=0):
    """(out, bound on the error before the result's own rounding) for q
    [B][Hq][D], k, v [pages][page][H][D].

    A score is off by 2 U per product of its D terms, the exponent's argument
    by a few U of its size, a probability therefore relatively by twice that
    (it and the sum), and by 2 U per key of the sums.  (2^-15 is left on top.)"""
    B, Hq, D = q.shape
    n_pages, page, H, _ = k.shape
    out, err = np.zeros_like(q), np.zeros_like(q)
    for b in range(B):
        n = int(min(max(lengths[b], 0), table.shape[1] * page))
        j = np.arange(max(0, n - window) if window else 0, n)
        p = table[b][j // page] if len(j) else np.zeros(0, np.int64)
        ok = (p >= 0) & (p < n_pages)
        j, p = j[ok], p[ok].astype(np.int64)
        if not len(j):
            continue
        for h in range(Hq):
            kk, vv = k[p, j % page, h // (Hq // H)], v[p, j % page, h // (Hq // H)]
            s = kk @ q[b, h] * scale
            off = (np.abs(kk) @ np.abs(q[b, h])).max() * abs(scale) * 2 * U * (D + 2)
            off += 8 * U * np.abs(s).max()
            w = np.exp(s - s.max())
            w /= w.sum()
            out[b, h] = w @ vv
            rel = 2 * np.expm1(2 * off) + 2.0 ** -15 + 4 * U * (len(j) + 8)
            err[b, h] = rel * (w @ np.abs(vv))
    return out, err


# ---- norms -------------------------------------------------------------------------

def block_norm(x, y, eps, post=None, gate=None, pre=None, x_scale=1.0, y_scale=1.0):
    """(x, h, bound on x's error, relative bound on h's).  A sum of squares
    goes through at most 16 + 6 + 16 additions of its own term and the root halves its
    relative error; a handful of operations follow."""
    u, rel = y, 0.0
    if post is not None:
        u = u / np.sqrt((u * u).mean(1, keepdims=True) + eps) * post
        rel = 40 * U
    if gate is not None:
        u = u * gate
    new = x_scale * x + y_scale * u
    err = (rel + 8 * U) * np.abs(y_scale * u) + 4 * U * np.abs(x_scale * x)
    rms = np.sqrt((new * new).mean(1, keepdims=True) + eps)
    h = new / rms
    # x's error reaches h directly and through the root mean square
    herr = err / rms + np.abs(h) * (np.sqrt((err * err).mean(1, keepdims=True)) / rms + 40 * U)
    if pre is not None:
        h, herr = h * pre, herr * np.abs(pre)
    return new, h, err, herr


def close(got, want, err, dtype, what=""):
    """|got - want| within the bound and the result's own rounding."""
    got = f64(got) if isinstance(got, torch.Tensor) else got
    room = err + HALF[dtype] * (np.abs(want) + err) + 1e-37
    bad = ~(np.abs(got - want) <= room)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(),
                           float((np.abs(got - want) / room)[bad][0]))
