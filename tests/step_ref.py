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


# ---- routing by scores -----------------------------------------------------------------

def route_scored(logits, k, token_req, table, scoring, select_bias, groups, top_groups, renorm,
                 scale, b_min, b_max):
    """The routing's tensors by name, one token after the other in binary64."""
    T, E = logits.shape
    L = b_max - b_min + 1
    idx, w, bits = np.zeros((T, k), int), np.zeros((T, k)), np.zeros((T, k), int)
    flags = 0
    for t in range(T):
        x = logits[t].astype(np.float64)
        if scoring == "softmax":
            top = np.max(x)
            with np.errstate(invalid="ignore"):
                e = np.where(x == top, 1.0, np.exp(x - top)) if top > -np.inf else np.zeros(E)
            score = e / e.sum() if e.sum() > 0 else e
        else:
            with np.errstate(over="ignore"):
                score = 1 / (1 + np.exp(-x))
        by = score if select_bias is None else score + select_bias.astype(np.float64)
        size = E // groups
        value = [sum(sorted(by[g * size:(g + 1) * size])[-2:]) for g in range(groups)]
        on = sorted(range(groups), key=lambda g: (-value[g], g))[:top_groups]
        among = [e for e in range(E) if e // size in on]
        sel = sorted(among, key=lambda e: (-by[e], e))[:k]
        s = score[sel]
        if renorm:
            s = s / s.sum() if s.sum() > 0 else 0 * s
        idx[t], w[t] = sel, s * scale
        r = 0 if token_req is None else token_req[t]
        if r < 0 or r >= len(table):
            flags, r = flags | 2, min(max(r, 0), len(table) - 1)
        b = table[r][sel].astype(int)
        if ((b < b_min) | (b > b_max)).any():
            flags |= 1
        bits[t] = np.clip(b, b_min, b_max)
    key = (idx * L + bits - b_min).reshape(-1)
    hist = np.bincount(key, minlength=E * L).reshape(E, L)
    perm = np.argsort(key, kind="stable")
    slot = np.empty(T * k, int)
    slot[perm] = np.arange(T * k)
    most = [max([b_min + l for l in range(L) if hist[e, l]], default=0) for e in range(E)]
    return dict(topk_idx=idx, topk_w=w, topk_bits=bits, hist=hist,
                offsets=np.concatenate([[0], np.cumsum(hist.reshape(-1))]), perm=perm,
                slot_of=slot, expert_maxbit=np.array(most), flags=np.array([flags]))


# ---- sampling ------------------------------------------------------------------------------

def sample(l, u, t=1.0, k=0, p=1.0, m=0.0):
    """(token, share, room) of one row: room is the least distance, in parts of the sums
    concerned, of a choice to where it would turn."""
    live = l > -np.inf
    if not live.any():
        return -1, 0.0, 1.0
    order = np.argsort(np.where(live, -l.astype(np.float64), np.inf), kind="stable")[:live.sum()]
    if not t > 0 or k == 1:
        return int(order[0]), 1.0, 1.0
    d = l[order].astype(np.float64)
    with np.errstate(invalid="ignore"):
        w = np.where(d == d[0], 1.0, np.exp((d - d[0]) / t))
    w = np.where(w == w, w, 0.0)
    if k > 0:
        w = w[:k]
    n, room = len(w), 1.0
    if p < 1:
        run = np.cumsum(w)
        at = max(p, 0.0) * run[-1]
        n = 1 + int((run[:-1] < at).sum())
        room = min(room, np.abs(run - at).min() / run[-1]) if p > 0 else room
    if m > 0:
        n = min(n, int((w >= min(m, 1.0)).sum()))
        # (w itself is compared with m, not its units: off by 2^-42 of itself)
        room = min(room, np.abs(w[1:] / m - 1).min()) if len(w) > 1 and m < 1 else room
    run = np.cumsum(w[:n])
    at = min(max(u, 0.0), 1.0) * run[-1]
    i = min(int((run <= at).sum()), n - 1)
    if u > 0:
        room = min(room, np.abs(run - at).min() / run[-1])
    return int(order[i]), w[i] / run[-1], room


# ---- attention behind a shared prefix ----------------------------------------------------

def attn_prefix(q, k, v, table, lengths, prefix_table, prefix_lens, scale):
    """(out, bound on the error before the result's own rounding): decoder_ref.attn over
    the rows of pages that each sequence really has."""
    page, room = k.shape[1], len(prefix_table) * k.shape[1]
    width = max(len(prefix_table), table.shape[1])
    out, err = np.zeros_like(q), np.zeros_like(q)
    for b in range(len(q)):
        n = max(int(lengths[b]), 0)
        s = min(max(int(prefix_lens[b]), 0), n, room)
        n = max(min(n, table.shape[1] * page), s)
        if n == 0:
            continue
        # every token as a page of its own
        j = np.arange(n)
        own = np.full(width, -1, np.int64)
        own[:table.shape[1]] = table[b]
        pre = np.full(width, -1, np.int64)
        pre[:len(prefix_table)] = prefix_table
        p = np.where(j < s, pre[j // page], own[j // page])
        ok = (p >= 0) & (p < len(k))
        at = np.where(ok, p * page + j % page, -1)
        flat = lambda t: t.reshape(-1, 1, *t.shape[2:])  # noqa: E731
        o, e = attn(q[b:b + 1], flat(k), flat(v), at[None], [n], scale)
        out[b], err[b] = o[0], e[0]
    return out, err
