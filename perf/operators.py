"""The decode operators around the MoE layer: their performance cases and plain forms.

With ``own`` false, run() computes each operator from elementary torch
operations in binary32; with ``own`` true it calls the package's entry points
on the same inputs.  exact() gives the same outputs in binary64.

Operators (the case's "op"):
  linear  y = x W^T + bias with 4-bit weights W = s (n - z), one scale s and
          zero point z per row and group of columns
  attn    attention of one new token per sequence over a paged key-value cache
  append  rotary rotation of the new tokens' q and k, K and V into the pages
  norm    x <- a x + b gate * postnorm(y), h = prenorm(x)

Inputs are drawn on the GPU from the seed: Gaussian activations and cache
rows, weights of std 0.02 quantized per group, page tables that are a random
permutation of the pool's pages, ragged lengths.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases -------------------------------------------------------------------

def _linear(name, T, rows, cols, group=128, dtype="bf16", bias=False):
    return dict(name=name, op="linear", T=T, rows=rows, cols=cols, group=group, dtype=dtype,
                bias=bias)


def _attn(name, B, length, heads, kv_heads, dim, page=16, dtype="bf16", ragged=True, window=0):
    return dict(name=name, op="attn", B=B, length=length, heads=heads, kv_heads=kv_heads, dim=dim,
                page=page, dtype=dtype, ragged=ragged, window=window)


def _append(name, seqs, new, past, heads, kv_heads, dim, page=16, dtype="bf16", rotary=True):
    return dict(name=name, op="append", seqs=seqs, new=new, past=past, heads=heads,
                kv_heads=kv_heads, dim=dim, page=page, dtype=dtype, rotary=rotary)


def _norm(name, T, d, dtype="bf16", post=True, gate="row"):
    return dict(name=name, op="norm", T=T, d=d, dtype=dtype, post=post, gate=gate)


def listed():
    return [
        # one user's token through an output projection: latency
        _linear("linear_1", T=1, rows=4096, cols=4096),
        # the fused q, k, v projection of the serving batch
        _linear("linear_qkv_16", T=16, rows=6144, cols=4096, bias=True),
        # the head of a 64-sequence batch, the widest matrix of a decoder
        _linear("linear_head_64", T=64, rows=32000, cols=4096),
        # a small fp32 layer: rows that fill no tile, an odd number of groups
        _linear("linear_f32_odd", T=5, rows=1003, cols=1984, group=64, dtype="f32", bias=True),
        # one user, a short context: latency
        _attn("attn_1_short", B=1, length=333, heads=32, kv_heads=8, dim=128),
        # the serving batch, ragged contexts of up to 4096
        _attn("attn_16", B=16, length=4096, heads=32, kv_heads=8, dim=128, page=64),
        # the 64-sequence batch with long contexts, the cache at its largest
        _attn("attn_64_long", B=64, length=8192, heads=32, kv_heads=8, dim=128, ragged=False),
        # one key head per query head, narrow heads, a sliding window, fp32
        _attn("attn_f32_window", B=9, length=2500, heads=12, kv_heads=12, dim=64, dtype="f32",
              window=1000),
        # the new token of every sequence of the serving batch
        _append("append_16", seqs=16, new=1, past=4000, heads=32, kv_heads=8, dim=128),
        # prompts of four requests entering the cache
        _append("append_prompt", seqs=4, new=2048, past=100, heads=32, kv_heads=8, dim=128),
        # between two blocks of the serving batch: latency
        _norm("norm_16", T=16, d=4096),
        # the same in prefill, a gate per token
        _norm("norm_prefill", T=8192, d=4096, gate="token"),
    ]


def _logint(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng: random.Random):
    op = rng.choice(["linear", "linear", "attn", "attn", "attn", "append", "norm"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv_heads, per = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 4, 4, 7, 8])
    dim, page = rng.choice([64, 80, 96, 128, 128, 128, 256]), rng.choice([16, 16, 24, 32, 64, 128])
    if op == "linear":
        group = rng.choice([32, 64, 128, 128])
        rows, cols = _logint(rng, 16, 16384), group * max(1, _logint(rng, 64, 8192) // group)
        c = _linear("", T=_logint(rng, 1, 256), rows=rows, cols=cols, group=group, dtype=dtype,
                    bias=rng.random() < 0.5)
        while c["T"] * rows * cols > 64 * 32000 * 4096:
            c["T"] //= 2
    elif op == "attn":
        c = _attn("", B=_logint(rng, 1, 128), length=_logint(rng, 1, 32768), heads=kv_heads * per,
                  kv_heads=kv_heads, dim=dim, page=page, dtype=dtype, ragged=rng.random() < 0.75,
                  window=rng.choice([0, 0, 0, _logint(rng, 1, 4096)]))
        while c["B"] * c["length"] * kv_heads * dim > 64 * 8192 * 8 * 128 // 4:
            if c["B"] > 1:
                c["B"] //= 2
            else:
                c["length"] //= 2
    elif op == "append":
        c = _append("", seqs=_logint(rng, 1, 64), new=_logint(rng, 1, 2048),
                    past=_logint(rng, 1, 4096), heads=kv_heads * per, kv_heads=kv_heads, dim=dim,
                    page=page, dtype=dtype, rotary=rng.random() < 0.75)
        while c["seqs"] * c["new"] * kv_heads * per * dim > 8192 * 32 * 128:
            c["new"] = c["new"] // 2 or 1
            if c["new"] == 1:
                break
    else:
        c = _norm("", T=_logint(rng, 1, 8192), d=_logint(rng, 64, 8192), dtype=dtype,
                  post=rng.random() < 0.5, gate=rng.choice(["none", "row", "token"]))
        while c["T"] * c["d"] > 8192 * 4096:
            c["T"] //= 2
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------

def _randn(g, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=dtype) * std)


def _pool(c, g, lengths, longest):
    """A pool of pages that holds every sequence at its longest, and a table
    that permutes them: the entries past a sequence's last page are -1."""
    need = -(-lengths // c["page"])
    width = -(-longest // c["page"])
    used = torch.arange(width)[None] < need[:, None]
    n = len(lengths) * width
    table = torch.full(used.shape, -1, dtype=torch.int32)
    table[used] = torch.randperm(n, generator=g, device=DEV)[:int(need.sum())].cpu().int()
    shape = (n, c["page"], c["kv_heads"], c["dim"])
    dt = DTYPES[c["dtype"]]
    return _randn(g, *shape, dtype=dt), _randn(g, *shape, dtype=dt), table.to(DEV)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(DEV)
    g.manual_seed(1_000_003 * (seed % (1 << 40)) + 17)
    h = torch.Generator()
    h.manual_seed(seed % (1 << 40) + 5)
    dt = DTYPES[c["dtype"]]
    s = {"case": c}
    if c["op"] == "linear":
        rows, cols, group = c["rows"], c["cols"], c["group"]
        w = _randn(g, rows, cols // group, group, std=0.02)
        lo, hi = w.amin(2).clamp(max=0), w.amax(2).clamp(min=0)
        s["scales"] = ((hi - lo) / 15).half()
        sf = s["scales"].float()
        s["zeros"] = torch.round(-lo / sf).clamp(0, 15).to(torch.uint8)
        s["codes"] = torch.round(w / sf[..., None] + s["zeros"].float()[..., None]) \
            .clamp(0, 15).to(torch.uint8).reshape(rows, cols)
        s["bias"] = _randn(g, rows, std=0.1) if c["bias"] else None
        s["x"] = _randn(g, c["T"], cols, dtype=dt)
        if own:
            from paper_2504_15299_amd import api
            s["w"] = api.linear_pack_codes(s["codes"], s["scales"], s["zeros"],
                                           api.Linear.empty(rows, cols, group, device=DEV))
    elif c["op"] == "attn":
        lengths = torch.full((c["B"],), c["length"])
        if c["ragged"]:
            # from an eighth of the longest up, the first one the longest
            lengths[1:] = torch.randint(-(-c["length"] // 8), c["length"] + 1, (c["B"] - 1,),
                                        generator=h)
        s["k"], s["v"], s["table"] = _pool(c, g, lengths, c["length"])
        s["lengths"] = lengths.to(torch.int32).to(DEV)
        s["q"] = _randn(g, c["B"], c["heads"], c["dim"], dtype=dt)
        if own:
            from paper_2504_15299_amd import api
            s["cache"] = api.KVCache(s["k"], s["v"])
            s["ws"] = torch.empty(api.attn_decode_workspace(c["B"], c["heads"], s["cache"],
                                                            c["length"]),
                                  dtype=torch.uint8, device=DEV)
    elif c["op"] == "append":
        past = torch.randint(-(-c["past"] // 2), c["past"] + 1, (c["seqs"],), generator=h)
        s["k"], s["v"], s["table"] = _pool(c, g, past + c["new"], c["past"] + c["new"])
        n = c["seqs"] * c["new"]
        s["seq"] = torch.arange(c["seqs"], dtype=torch.int32).repeat_interleave(c["new"]).to(DEV)
        s["pos"] = (past[:, None] + torch.arange(c["new"])).reshape(n).to(torch.int32).to(DEV)
        # q, k and v as the fused projection leaves them, one row per token
        s["qkv"] = _randn(g, n, c["heads"] + 2 * c["kv_heads"], c["dim"], dtype=dt)
        if c["rotary"]:
            f = 1e4 ** (-torch.arange(c["dim"] // 2, dtype=torch.float64) * 2 / c["dim"])
            a = torch.arange(c["past"] + c["new"], dtype=torch.float64)[:, None] * f
            s["cos"], s["sin"] = a.cos().float().to(DEV), a.sin().float().to(DEV)
        else:
            s["cos"] = s["sin"] = None
        if own:
            from paper_2504_15299_amd import api
            s["cache"] = api.KVCache(s["k"], s["v"])
    else:
        T, d = c["T"], c["d"]
        s["x"] = _randn(g, T, d)
        s["y"] = _randn(g, T, d, dtype=dt)
        s["pre"] = 1 + _randn(g, d, std=0.1)
        s["post"] = 1 + _randn(g, d, std=0.1) if c["post"] else None
        s["gate"] = {"none": None, "row": _randn(g, d, std=0.5),
                     "token": _randn(g, T, d, dtype=dt, std=0.5) if c["gate"] == "token" else None
                     }[c["gate"]]
    return s


X_SCALE, Y_SCALE, EPS = 0.9, 0.5, 1e-5


# ---- the package's calls -----------------------------------------------------

def _run_own(s):
    from paper_2504_15299_amd import api
    c = s["case"]
    if c["op"] == "linear":
        return api.linear_forward(s["x"], s["w"], bias=s["bias"])
    if c["op"] == "attn":
        return api.attn_decode(s["q"], s["cache"], s["table"], s["lengths"], window=c["window"],
                               max_len=c["length"], workspace=s["ws"])
    if c["op"] == "append":
        H, K = c["heads"], c["kv_heads"]
        q, k, v = s["qkv"][:, :H], s["qkv"][:, H:H + K], s["qkv"][:, H + K:]
        out = api.kv_append(q, k, v, s["cache"], s["table"], s["pos"], token_seq=s["seq"],
                            cos=s["cos"], sin=s["sin"])
        return out, s["k"], s["v"]
    out = api.block_norm(s["x"], s["y"], EPS, pre_weight=s["pre"], post_weight=s["post"],
                         gate=s["gate"], x_scale=X_SCALE, y_scale=Y_SCALE,
                         h_dtype=DTYPES[c["dtype"]])
    return s["x"], out


# ---- the plain forms, in binary32 ----------------------------------------------

def _plain_linear(s):
    c = s["case"]
    rows, cols, group = c["rows"], c["cols"], c["group"]
    w = s["codes"].float().reshape(rows, cols // group, group) - s["zeros"].float()[..., None]
    w = (w * s["scales"].float()[..., None]).reshape(rows, cols)
    y = torch.matmul(s["x"].float(), w.t())
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["x"].dtype)


def _plain_attn(s):
    c = s["case"]
    B, K, D, G = c["B"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"]
    pages = s["table"].long().clamp(min=0)
    k = s["k"][pages].float().reshape(B, -1, K, D).permute(0, 2, 3, 1)
    v = s["v"][pages].float().reshape(B, -1, K, D).permute(0, 2, 1, 3)
    j = torch.arange(k.shape[3], device=DEV)
    n = s["lengths"].long()[:, None]
    seen = j < n
    if c["window"]:
        seen = seen & (j >= n - c["window"])
    x = torch.matmul(s["q"].float().reshape(B, K, G, D), k) / math.sqrt(D)
    x = torch.where(seen[:, None, None], x, -math.inf)
    m = x.amax(3, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    o = torch.matmul(p, v) / p.sum(3, keepdim=True).clamp(min=1e-30)
    return o.reshape(B, c["heads"], D).to(s["q"].dtype)


def _plain_rotate(x, cos, sin):
    if cos is None:
        return x
    a, b = x.float().chunk(2, dim=2)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), dim=2).to(x.dtype)


def _plain_append(s):
    c = s["case"]
    H, K = c["heads"], c["kv_heads"]
    q, k, v = s["qkv"][:, :H], s["qkv"][:, H:H + K], s["qkv"][:, H + K:]
    pos = s["pos"].long()
    cos = sin = None
    if c["rotary"]:
        cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    page = s["table"][s["seq"].long(), pos // c["page"]].long()
    s["k"][page, pos % c["page"]] = _plain_rotate(k, cos, sin)
    s["v"][page, pos % c["page"]] = v
    return _plain_rotate(q, cos, sin), s["k"], s["v"]


def _plain_norm(s):
    c = s["case"]
    u = s["y"].float()
    if s["post"] is not None:
        u = u / torch.sqrt((u * u).mean(1, keepdim=True) + EPS) * s["post"]
    if s["gate"] is not None:
        u = u * s["gate"].float()
    s["x"] = X_SCALE * s["x"] + Y_SCALE * u
    h = s["x"] / torch.sqrt((s["x"] * s["x"]).mean(1, keepdim=True) + EPS) * s["pre"]
    return s["x"], h.to(DTYPES[c["dtype"]])


def run(state):
    if own:
        return _run_own(state)
    return {"linear": _plain_linear, "attn": _plain_attn, "append": _plain_append,
            "norm": _plain_norm}[state["case"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------

def work(case):
    c = case
    size = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "linear":
        n = c["rows"] * c["cols"]
        return {"bytes": n / 2 + 3 * n / c["group"] + size * c["T"] * (c["cols"] + c["rows"])
                + (4 * c["rows"] if c["bias"] else 0), "flops": 2 * c["T"] * n}
    if c["op"] == "attn":
        # ragged lengths are spread evenly from an eighth of the longest up
        keys, at = 0.0, 64
        for i in range(at):
            n = c["length"] * (1 / 8 + 7 / 8 * (i + 0.5) / at) if c["ragged"] else c["length"]
            keys += min(n, c["window"] or n) / at
        if c["B"] == 1:
            keys = min(c["length"], c["window"] or c["length"])
        else:
            keys = (keys * (c["B"] - 1) + min(c["length"], c["window"] or c["length"])) / c["B"]
        keys *= c["B"]
        return {"bytes": 2 * size * keys * c["kv_heads"] * c["dim"]
                + 2 * size * c["B"] * c["heads"] * c["dim"] + 4 * keys / c["page"],
                "flops": 4 * keys * c["heads"] * c["dim"]}
    if c["op"] == "append":
        n = c["seqs"] * c["new"]
        row = (c["heads"] + 2 * c["kv_heads"]) * c["dim"]
        table = min(n, c["past"] + c["new"]) * c["dim"] * 4 if c["rotary"] else 0
        return {"bytes": 2 * size * n * row + table + 12 * n,
                "flops": 3 * n * (c["heads"] + c["kv_heads"]) * c["dim"] if c["rotary"] else 0}
    n = c["T"] * c["d"]
    return {"bytes": n * (8 + 2 * size + (size if c["gate"] == "token" else 0)) + 12 * c["d"],
            "flops": 10 * n}


# ---- binary64 --------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["op"] == "linear":
        # group by group: s * (n . x - z * sum x)
        x = s["x"].double()
        y = torch.zeros((c["T"], c["rows"]), dtype=torch.float64, device=DEV)
        for i in range(c["cols"] // c["group"]):
            xs = x[:, i * c["group"]:(i + 1) * c["group"]]
            n = s["codes"][:, i * c["group"]:(i + 1) * c["group"]].double()
            y += s["scales"][:, i].double() * (xs @ n.t() - xs.sum(1, keepdim=True)
                                               * s["zeros"][:, i].double())
        return y if s["bias"] is None else y + s["bias"].double()
    if c["op"] == "attn":
        out = []
        G = c["heads"] // c["kv_heads"]
        for b, n in enumerate(s["lengths"].tolist()):
            first = max(0, n - c["window"]) if c["window"] else 0
            at = torch.arange(first, n, device=DEV)
            page, slot = s["table"][b].long()[at // c["page"]], at % c["page"]
            heads = []
            for h in range(c["kv_heads"]):
                k, v = s["k"][page, slot, h].double(), s["v"][page, slot, h].double()
                q = s["q"][b, h * G:(h + 1) * G].double()
                heads.append(torch.softmax(q @ k.t() * c["dim"] ** -0.5, 1) @ v)
            out.append(torch.cat(heads))
        return torch.stack(out)
    if c["op"] == "append":
        H, K, half = c["heads"], c["kv_heads"], c["dim"] // 2
        x = s["qkv"].double()
        pos, seq = s["pos"].long(), s["seq"].long()
        if c["rotary"]:
            w = torch.complex(s["cos"].double(), s["sin"].double())[pos][:, None]
            z = torch.complex(x[:, :H + K, :half], x[:, :H + K, half:]) * w
            x = torch.cat((torch.cat((z.real, z.imag), 2), x[:, H + K:]), 1)
        kc, vc = s["k"].double(), s["v"].double()
        flat = s["table"].long()[seq, pos // c["page"]] * c["page"] + pos % c["page"]
        kc.view(-1, K, c["dim"]).index_copy_(0, flat, x[:, H:H + K].contiguous())
        vc.view(-1, K, c["dim"]).index_copy_(0, flat, x[:, H + K:].contiguous())
        return x[:, :H].contiguous(), kc, vc
    u = s["y"].double()
    if s["post"] is not None:
        u = u * s["post"].double() * (u.square().mean(1, keepdim=True) + EPS).rsqrt()
    if s["gate"] is not None:
        u = u * s["gate"].double()
    x = X_SCALE * s["x"].double() + Y_SCALE * u
    return x, x * s["pre"].double() * (x.square().mean(1, keepdim=True) + EPS).rsqrt()
