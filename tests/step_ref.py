"""Plain binary64 forms (numpy) of the head norms with their append, of routing by
scores, of sampling and of attention behind a shared prefix, with the error bounds
that follow from the kernels' binary32 arithmetic (decoder_ref.U, decoder_ref.close)."""
import numpy as np

from decoder_ref import U, attn


# ---- head norms and rotation ---------------------------------------------------------

def head_norm(x, weight, eps):
    """Rows of x [N][heads][D] normed (weight None: x) and the bound on the error.

    Every term of the sum of squares goes through at most 16 + 6 roundings, all terms
    are positive, and the root halves the sum's relative error; mean, eps, root,
    division and the products with the weight and the value follow."""
    if weight is None:
        return x, np.zeros_like(x)
    n = x / np.sqrt((x * x).mean(2, keepdims=True) + eps) * weight
    return n, (11 + 6) * U * np.abs(n)


def rotate(x, err, cos, sin, pos, interleaved):
    """The first 2 * cos.shape[1] values of every head of x [N][heads][D] rotated, and
    the bound on the error, err that of x."""
    if cos is None:
        return x, err
    half = cos.shape[1]
    x, err = x.copy(), err.copy()
    i, j = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else \
        (slice(0, half), slice(half, 2 * half))
    c, s = cos[pos][:, None], sin[pos][:, None]
    a, b, ea, eb = x[..., i], x[..., j], err[..., i], err[..., j]
    x[..., i], x[..., j], err[..., i], err[..., j] = (
        a * c - b * s, b * c + a * s,
        np.abs(ea * c) + np.abs(eb * s) + 3 * U * (np.abs(a * c) + np.abs(b * s)),
        np.abs(eb * c) + np.abs(ea * s) + 3 * U * (np.abs(b * c) + np.abs(a * s)))
    return x, err
