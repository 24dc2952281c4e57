"""What a decode iteration needs beside perf/operators.py's operators: their
performance cases and plain forms.

With ``own`` false, run() computes each operator from elementary torch
operations, in binary32 (the choices of experts and tokens, which a last bit
could turn, in binary64); with ``own`` true it calls the package's entry points
on the same inputs.  exact() gives the same outputs in binary64.

Operators (the case's "op"):
  prefix  attention of one new token per sequence, the keys of a shared prefix
          read once for the whole batch
  append  RMS norms of the query and key heads, rotary rotation of all or part
          of a head, K and V into the pages
  route   experts by softmax or sigmoid scores with a balance bias and groups,
          weights, counts and permutation
  sample  tokens from logits by temperature, top-k, top-p and min-p

Inputs are drawn on the GPU from the seed: Gaussian activations, cache rows and
logits, page tables that are a random permutation of the pool's pages, ragged
lengths.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
B_MIN, B_MAX = 2, 8     # bit-widths of the experts
EPS = 1e-6


# ---- cases -------------------------------------------------------------------

def _prefix(name, B, prefix, rest, heads, kv_heads, dim, page=16, dtype="bf16", mixed=False):
    """``rest``: the most tokens of a sequence past its prefix; ``mixed``: every
    fourth sequence shares a part of the prefix only, or nothing."""
    return dict(name=name, op="prefix", B=B, prefix=prefix, rest=rest, heads=heads,
                kv_heads=kv_heads, dim=dim, page=page, dtype=dtype, mixed=mixed)


def _append(name, seqs, new, past, heads, kv_heads, dim, rot, page=16, dtype="bf16",
            interleaved=False):
    return dict(name=name, op="append", seqs=seqs, new=new, past=past, heads=heads,
                kv_heads=kv_heads, dim=dim, rot=rot, page=page, dtype=dtype,
                interleaved=interleaved)


def _route(name, T, E, k, scoring="softmax", bias=False, groups=1, top_groups=1, renorm=True,
           scale=1.0):
    return dict(name=name, op="route", T=T, E=E, k=k, scoring=scoring, bias=bias, groups=groups,
                top_groups=top_groups, renorm=renorm, scale=scale)


def _sample(name, B, V, dtype="f32", top_k=True, top_p=True, min_p=True):
    return dict(name=name, op="sample", B=B, V=V, dtype=dtype, top_k=top_k, top_p=top_p,
                min_p=min_p)


def listed():
    return [
        # two answers to one short prompt: latency
        _prefix("prefix_2_short", B=2, prefix=501, rest=40, heads=32, kv_heads=8, dim=128),
        # the serving batch behind a system prompt that ends inside a page
        _prefix("prefix_16", B=16, prefix=2000, rest=512, heads=32, kv_heads=8, dim=128, page=64,
                mixed=True),
        # the 64-sequence batch over a long document, the most work
        _prefix("prefix_64_long", B=64, prefix=8192, rest=512, heads=32, kv_heads=8, dim=128),
        # one key head per query head, narrow heads, fp32
        _prefix("prefix_f32", B=9, prefix=1500, rest=300, heads=12, kv_heads=12, dim=64,
                dtype="f32"),
        # the new token of every sequence of the serving batch
        _append("append_16", seqs=16, new=1, past=4000, heads=32, kv_heads=8, dim=128, rot=128),
        # prompts of four requests entering the cache
        _append("append_prompt", seqs=4, new=2048, past=100, heads=32, kv_heads=8, dim=128,
                rot=128),
        # pairs side by side over a quarter of narrow heads, fp32
        _append("append_part", seqs=3, new=101, past=700, heads=7, kv_heads=1, dim=80, rot=20,
                dtype="f32", interleaved=True),
        # the serving batch to two of eight experts: latency
        _route("route_16", T=16, E=8, k=2),
        # many tokens to fine-grained experts, in groups, with a bias for balance
        _route("route_groups", T=8192, E=64, k=6, scoring="sigmoid", bias=True, groups=8,
               top_groups=4, scale=2.5),
        # one user's next token from all of the vocabulary that top-p leaves: latency
        _sample("sample_1", B=1, V=32000, top_k=False, min_p=False),
        # the 64-sequence batch, each request with its own settings
        _sample("sample_64", B=64, V=32000),
        # a large batch over a large vocabulary, bf16
        _sample("sample_wide", B=256, V=131072, dtype="bf16"),
    ]


def _logint(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng: random.Random):
    op = rng.choice(["prefix", "prefix", "prefix", "append", "append", "route", "sample",
                     "sample"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kv_heads, per = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 4, 4, 7, 8])
    dim, page = rng.choice([64, 80, 96, 128, 128, 128, 256]), rng.choice([16, 16, 24, 32, 64, 128])
    if op == "prefix":
        c = _prefix("", B=_logint(rng, 1, 128), prefix=_logint(rng, 1, 16384),
                    rest=_logint(rng, 1, 1024), heads=kv_heads * per, kv_heads=kv_heads, dim=dim,
                    page=page, dtype=dtype, mixed=rng.random() < 0.4)
        # (fp32 products take eight times as long)
        most = 64 * (8192 + 256) * 32 * 128 // (8 if dtype == "f32" else 1)
        while c["B"] * (c["prefix"] + c["rest"]) * c["heads"] * dim > most or \
                c["B"] * c["rest"] * kv_heads * dim > 64 * 512 * 8 * 128:
            if c["B"] > 1:
                c["B"] //= 2
            else:
                c["prefix"] = c["prefix"] // 2 or 1
                c["rest"] = c["rest"] // 2 or 1
    elif op == "append":
        rot = rng.choice([dim, dim, dim // 2, dim // 4])
        c = _append("", seqs=_logint(rng, 1, 64), new=_logint(rng, 1, 2048),
                    past=_logint(rng, 1, 4096), heads=kv_heads * per, kv_heads=kv_heads, dim=dim,
                    rot=rot, page=page, dtype=dtype, interleaved=rng.random() < 0.4)
        while c["seqs"] * c["new"] * kv_heads * (per + 2) * dim > 8192 * 48 * 128:
            c["new"] = c["new"] // 2 or 1
            if c["new"] == 1:
                break
    elif op == "route":
        E = rng.choice([8, 8, 16, 32, 48, 60, 64, 64])
        groups = rng.choice([1, 1, 2, 4]) if E % 8 == 0 or E == 60 else 1
        top = rng.randint(1, groups)
        c = _route("", T=_logint(rng, 1, 8192), E=E, k=rng.randint(1, min(8, E // groups * top)),
                   scoring=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.5,
                   groups=groups, top_groups=top, renorm=rng.random() < 0.7,
                   scale=rng.choice([1.0, 1.0, 2.5]))
    else:
        c = _sample("", B=_logint(rng, 1, 256), V=_logint(rng, 1000, 131072), dtype=dtype,
                    top_k=rng.random() < 0.6, top_p=rng.random() < 0.6, min_p=rng.random() < 0.4)
        while c["B"] * c["V"] > 256 * 131072 // (4 if dtype == "f32" else 1):
            c["B"] //= 2
    del c["name"]
    return c


# ---- inputs ------------------------------------------------------------------

def _randn(g, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=dtype) * std)


def _own_lengths(c, h):
    """Tokens of each sequence in its own pages, the first one's the most."""
    n = torch.randint(1, c["rest"] + 1, (c["B"],), generator=h)
    n[0] = c["rest"]
    return n


def _shared(c, h):
    """Tokens of the prefix that each sequence shares."""
    p = torch.full((c["B"],), c["prefix"])
    if c["mixed"]:
        p[1::4] = torch.randint(0, c["prefix"] + 1, (len(p[1::4]),), generator=h)
    return p


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(DEV)
    g.manual_seed(1_000_033 * (seed % (1 << 40)) + 29)
    h = torch.Generator()
    h.manual_seed(seed % (1 << 40) + 7)
    s = {"case": c}
    i32 = torch.int32
    if c["op"] == "prefix":
        dt, page = DTYPES[c["dtype"]], c["page"]
        shared = _shared(c, h)
        lengths = shared + _own_lengths(c, h)
        head = -(-c["prefix"] // page)
        # a row's first pages are the prefix's as far as it is shared whole pages, its
        # own after that; entries past its last page are -1
        whole, need = shared // page, -(-lengths // page)
        width = int(need.max())
        at = torch.arange(width)[None]
        mine = (at >= whole[:, None]) & (at < need[:, None])
        n_pages = head + int(mine.sum())
        order = torch.randperm(n_pages, generator=g, device=DEV).cpu().to(i32)
        table = torch.full((c["B"], width), -1, dtype=i32)
        n = min(head, width)
        table[:, :n] = torch.where(at[:, :n] < whole[:, None], order[None, :n], table[:, :n])
        table[mine] = order[head:]
        shape = (n_pages, page, c["kv_heads"], c["dim"])
        s["k"], s["v"] = _randn(g, *shape, dtype=dt), _randn(g, *shape, dtype=dt)
        s["table"], s["lengths"] = table.to(DEV), lengths.to(i32).to(DEV)
        s["prefix_table"], s["shared"] = order[:head].to(DEV), shared.to(i32).to(DEV)
        # the most tokens past a prefix, which the server knows from its own lists
        s["max_rest"] = c["rest"]
        s["q"] = _randn(g, c["B"], c["heads"], c["dim"], dtype=dt)
        if own:
            from paper_2504_15299_amd import api
            s["cache"] = api.KVCache(s["k"], s["v"])
            s["ws"] = torch.empty(api.attn_prefix_workspace(c["B"], c["heads"], s["cache"],
                                                            c["prefix"], c["rest"]),
                                  dtype=torch.uint8, device=DEV)
    elif c["op"] == "append":
        dt = DTYPES[c["dtype"]]
        past = torch.randint(-(-c["past"] // 2), c["past"] + 1, (c["seqs"],), generator=h)
        longest = c["past"] + c["new"]
        need, width = -(-(past + c["new"]) // c["page"]), -(-longest // c["page"])
        used = torch.arange(width)[None] < need[:, None]
        pool = c["seqs"] * width
        table = torch.full(used.shape, -1, dtype=i32)
        table[used] = torch.randperm(pool, generator=g, device=DEV)[:int(need.sum())].cpu().to(i32)
        shape = (pool, c["page"], c["kv_heads"], c["dim"])
        s["k"], s["v"], s["table"] = (_randn(g, *shape, dtype=dt), _randn(g, *shape, dtype=dt),
                                      table.to(DEV))
        n = c["seqs"] * c["new"]
        s["seq"] = torch.arange(c["seqs"], dtype=i32).repeat_interleave(c["new"]).to(DEV)
        s["pos"] = (past[:, None] + torch.arange(c["new"])).reshape(n).to(i32).to(DEV)
        # q, k and v as the fused projection leaves them, one row per token
        s["qkv"] = _randn(g, n, c["heads"] + 2 * c["kv_heads"], c["dim"], dtype=dt)
        s["qw"], s["kw"] = (1 + _randn(g, c["dim"], std=0.1) for _ in range(2))
        f = 1e4 ** (-torch.arange(c["rot"] // 2, dtype=torch.float64) * 2 / c["rot"])
        a = torch.arange(longest, dtype=torch.float64)[:, None] * f
        s["cos"], s["sin"] = a.cos().float().to(DEV), a.sin().float().to(DEV)
        if own:
            from paper_2504_15299_amd import api
            s["cache"] = api.KVCache(s["k"], s["v"])
    elif c["op"] == "route":
        s["logits"] = _randn(g, c["T"], c["E"], std=1.5)
        s["bias"] = _randn(g, c["E"], std=0.1) if c["bias"] else None
        s["req"] = (torch.arange(c["T"]) % 16).to(i32).to(DEV)
        s["bits"] = torch.tensor([2, 3, 4, 8], dtype=torch.uint8)[
            torch.randint(0, 4, (16, c["E"]), generator=h)].to(DEV)
        if own:
            from paper_2504_15299_amd import api
            s["out"] = api.Routing.empty(c["T"], c["E"], c["k"], B_MIN, B_MAX, device=DEV)
    else:
        B = c["B"]
        s["logits"] = _randn(g, B, c["V"], std=3.0).to(DTYPES[c["dtype"]])
        s["u"] = torch.rand(B, generator=g, device=DEV)
        s["temperature"] = 0.5 + torch.rand(B, generator=g, device=DEV)
        s["temperature"][5::8] = 0.0        # some requests want the likeliest token
        s["top_k"] = torch.randint(1, 200, (B,), generator=h).to(i32) if c["top_k"] else None
        if c["top_k"]:
            s["top_k"][3::4] = 0             # some no bound
            s["top_k"] = s["top_k"].to(DEV)
        s["top_p"] = 0.5 + 0.5 * torch.rand(B, generator=g, device=DEV) if c["top_p"] else None
        s["min_p"] = 0.1 * torch.rand(B, generator=g, device=DEV) if c["min_p"] else None
    return s


# ---- the package's calls -----------------------------------------------------

def _run_own(s):
    from paper_2504_15299_amd import api
    c = s["case"]
    if c["op"] == "prefix":
        return api.attn_prefix(s["q"], s["cache"], s["table"], s["lengths"], s["prefix_table"],
                               s["shared"], max_prefix=c["prefix"], max_rest=s["max_rest"],
                               workspace=s["ws"])
    if c["op"] == "append":
        H, K = c["heads"], c["kv_heads"]
        q, k, v = s["qkv"][:, :H], s["qkv"][:, H:H + K], s["qkv"][:, H + K:]
        out = api.kv_append_norm(q, k, v, s["cache"], s["table"], s["pos"], token_seq=s["seq"],
                                 q_weight=s["qw"], k_weight=s["kw"], eps=EPS, cos=s["cos"],
                                 sin=s["sin"], interleaved=c["interleaved"])
        return out, s["k"], s["v"]
    if c["op"] == "route":
        r = api.route_scored(s["logits"], c["k"], s["req"], s["bits"], scoring=c["scoring"],
                             select_bias=s["bias"], groups=c["groups"], top_groups=c["top_groups"],
                             renorm=c["renorm"], scale=c["scale"], b_min=B_MIN, b_max=B_MAX,
                             out=s["out"])
        return (r.topk_idx, r.topk_w, r.topk_bits, r.hist, r.offsets, r.perm, r.slot_of,
                r.expert_maxbit)
    return api.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"],
                      top_p=s["top_p"], min_p=s["min_p"])


# ---- the plain forms -----------------------------------------------------------

def _plain_prefix(s):
    c = s["case"]
    B, K, D, G, page = c["B"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"], c["page"]
    P = s["prefix_table"].shape[0] * page
    q = s["q"].float().reshape(B, K, G, D) / math.sqrt(D)
    # the prefix's keys for all queries of a key head together
    pages = s["prefix_table"].long()
    k = s["k"][pages].float().reshape(P, K, D).permute(1, 2, 0).contiguous()
    v = s["v"][pages].float().reshape(P, K, D).permute(1, 0, 2).contiguous()
    qh = q.permute(1, 0, 2, 3).reshape(K, B * G, D).contiguous()
    x0 = torch.matmul(qh, k).reshape(K, B, G, P).permute(1, 0, 2, 3)
    seen = torch.arange(P, device=DEV) < s["shared"].long()[:, None]
    x0 = torch.where(seen[:, None, None], x0, -math.inf)
    # each sequence's own keys
    j = s["shared"].long()[:, None] + torch.arange(c["rest"], device=DEV)
    real = j < s["lengths"].long()[:, None]
    j = torch.where(real, j, s["shared"].long()[:, None])
    mine = s["table"].long().gather(1, j // page).clamp(min=0)
    k1 = s["k"][mine, j % page].float().permute(0, 2, 3, 1).contiguous()
    v1 = s["v"][mine, j % page].float().permute(0, 2, 1, 3).contiguous()
    x1 = torch.where(real[:, None, None], torch.matmul(q, k1), -math.inf)
    m = torch.maximum(x0.amax(3, keepdim=True), x1.amax(3, keepdim=True))
    p0, p1 = torch.exp(x0 - m), torch.exp(x1 - m)
    o = torch.matmul(p0.permute(1, 0, 2, 3).reshape(K, B * G, P), v)
    o = o.reshape(K, B, G, D).permute(1, 0, 2, 3) + torch.matmul(p1, v1)
    o = o / (p0.sum(3, keepdim=True) + p1.sum(3, keepdim=True))
    return o.reshape(B, c["heads"], D).to(s["q"].dtype)


def _plain_norm_rotate(x, w, cos, sin, interleaved):
    x = x.float()
    x = x / torch.sqrt((x * x).mean(2, keepdim=True) + EPS) * w
    R = 2 * cos.shape[2]
    r, rest = x[..., :R], x[..., R:]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=3).flatten(2)
    else:
        a, b = r.chunk(2, dim=2)
        r = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=2)
    return torch.cat((r, rest), dim=2)


def _plain_append(s):
    c = s["case"]
    H, K = c["heads"], c["kv_heads"]
    q, k, v = s["qkv"][:, :H], s["qkv"][:, H:H + K], s["qkv"][:, H + K:]
    pos = s["pos"].long()
    cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
    page = s["table"][s["seq"].long(), pos // c["page"]].long()
    s["k"][page, pos % c["page"]] = _plain_norm_rotate(k, s["kw"], cos, sin,
                                                       c["interleaved"]).to(k.dtype)
    s["v"][page, pos % c["page"]] = v
    out = _plain_norm_rotate(q, s["qw"], cos, sin, c["interleaved"]).to(q.dtype)
    return out, s["k"], s["v"]


def _plain_route(s):
    c = s["case"]
    T, E, k, n = c["T"], c["E"], c["k"], c["groups"]
    x = s["logits"].double()
    if c["scoring"] == "softmax":
        e = torch.exp(x - x.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    else:
        score = 1 / (1 + torch.exp(-x))
    by = score if s["bias"] is None else score + s["bias"].double()
    if n > 1:
        best = by.reshape(T, n, E // n).sort(dim=2, descending=True).values[..., :2].sum(2)
        top = best.sort(dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        on = torch.zeros((T, n), dtype=torch.bool, device=DEV).scatter_(1, top, True)
        by = torch.where(on.repeat_interleave(E // n, 1), by, -math.inf)
    idx = by.sort(dim=1, descending=True, stable=True).indices[:, :k]
    w = score.gather(1, idx)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    bits = s["bits"][s["req"].long()[:, None], idx]
    L = B_MAX - B_MIN + 1
    key = (idx * L + bits.long() - B_MIN).reshape(-1)
    hist = torch.zeros(E * L, dtype=torch.int64, device=DEV).scatter_add_(0, key,
                                                                          torch.ones_like(key))
    offsets = torch.cat((torch.zeros(1, dtype=torch.int64, device=DEV), hist.cumsum(0)))
    perm = key.sort(dim=0, stable=True).indices
    slot = torch.empty_like(perm)
    slot[perm] = torch.arange(T * k, device=DEV)
    used = (hist.reshape(E, L) > 0) * torch.arange(B_MIN, B_MAX + 1, device=DEV)
    i32 = torch.int32
    return (idx.to(i32), (w * c["scale"]).float(), bits, hist.reshape(E, L).to(i32),
            offsets.to(i32), perm.to(i32), slot.to(i32), used.amax(1).to(torch.uint8))


def _plain_sample(s):
    x = s["logits"].double()
    B, V = x.shape
    order = x.sort(dim=1, descending=True, stable=True)
    t = s["temperature"].double()[:, None]
    w = torch.exp((order.values - order.values[:, :1]) / torch.where(t > 0, t, 1.0))
    keep = torch.ones((B, V), dtype=torch.bool, device=DEV)
    if s["top_k"] is not None:
        n = s["top_k"].long()[:, None]
        keep = (torch.arange(V, device=DEV)[None] < n) | (n <= 0)
    if s["top_p"] is not None:
        run = torch.where(keep, w, 0.0)
        keep = keep & (run.cumsum(1) - run < s["top_p"].double()[:, None] * run.sum(1, keepdim=True))
    if s["min_p"] is not None:
        keep = keep & (w >= s["min_p"].double()[:, None])
    keep[:, 1:] &= t > 0
    run = torch.where(keep, w, 0.0).cumsum(1)
    total = run[:, -1:]
    at = (run <= s["u"].double()[:, None] * total).sum(1, keepdim=True)
    token = order.indices.gather(1, at)[:, 0]
    return token.to(torch.int32), (w.gather(1, at) / total)[:, 0].float()


def run(state):
    if own:
        return _run_own(state)
    return {"prefix": _plain_prefix, "append": _plain_append, "route": _plain_route,
            "sample": _plain_sample}[state["case"]["op"]](state)


# ---- what a pass cannot do without ------------------------------------------------

def work(case):
    c = case
    if c["op"] == "route":
        n = c["T"] * c["k"]
        return {"bytes": 4 * c["T"] * (c["E"] + 1) + 17 * n + 8 * c["E"] * (B_MAX - B_MIN + 1),
                "flops": 10 * c["T"] * c["E"]}
    size = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "sample":
        return {"bytes": size * c["B"] * c["V"] + 28 * c["B"], "flops": 10 * c["B"] * c["V"]}
    if c["op"] == "prefix":
        # shares and lengths are spread evenly, every fourth sequence's share where mixed
        part = (c["B"] + 2) // 4 if c["mixed"] else 0
        pairs = c["prefix"] * (c["B"] - part / 2)
        rest = c["rest"] + (c["B"] - 1) * (c["rest"] + 1) / 2
        row = 2 * size * c["kv_heads"] * c["dim"]
        read = c["prefix"] if part < c["B"] else c["prefix"] / 2
        return {"bytes": row * (read + rest) + 2 * size * c["B"] * c["heads"] * c["dim"],
                "flops": 4 * (pairs + rest) * c["heads"] * c["dim"]}
    n = c["seqs"] * c["new"]
    row = (c["heads"] + 2 * c["kv_heads"]) * c["dim"]
    return {"bytes": 2 * size * n * row + min(n, c["past"] + c["new"]) * c["rot"] * 4 + 12 * n
            + 8 * c["dim"], "flops": 7 * n * (c["heads"] + c["kv_heads"]) * c["dim"]}


# ---- binary64 --------------------------------------------------------------------

def _exact_prefix(s):
    c = s["case"]
    K, G = c["kv_heads"], c["heads"] // c["kv_heads"]
    out = []
    for b, (n, p) in enumerate(zip(s["lengths"].tolist(), s["shared"].tolist())):
        j = torch.arange(n, device=DEV)
        cols = j // c["page"]
        page = s["table"][b].long()[cols]
        page[:p] = s["prefix_table"].long()[cols[:p]]
        heads = []
        for h in range(K):
            k, v = s["k"][page, j % c["page"], h].double(), s["v"][page, j % c["page"], h].double()
            q = s["q"][b, h * G:(h + 1) * G].double()
            heads.append(torch.softmax(q @ k.t() * c["dim"] ** -0.5, 1) @ v)
        out.append(torch.cat(heads))
    return torch.stack(out)


def _exact_append(s):
    c = s["case"]
    H, K, R = c["heads"], c["kv_heads"], c["rot"]
    x = s["qkv"].double()
    pos = s["pos"].long()
    heads = x[:, :H + K] * (x[:, :H + K].square().mean(2, keepdim=True) + EPS).rsqrt()
    heads = heads * torch.cat((s["qw"].double().expand(H, -1), s["kw"].double().expand(K, -1)))
    turn = torch.complex(s["cos"].double(), s["sin"].double())[pos][:, None]
    if c["interleaved"]:
        z = torch.view_as_complex(heads[..., :R].reshape(*heads.shape[:2], R // 2, 2).contiguous())
        r = torch.view_as_real(z * turn).flatten(2)
    else:
        z = torch.complex(heads[..., :R // 2], heads[..., R // 2:R]) * turn
        r = torch.cat((z.real, z.imag), 2)
    heads = torch.cat((r, heads[..., R:]), 2)
    kc, vc = s["k"].double(), s["v"].double()
    at = s["table"].long()[s["seq"].long(), pos // c["page"]] * c["page"] + pos % c["page"]
    kc.view(-1, K, c["dim"]).index_copy_(0, at, heads[:, H:].contiguous())
    vc.view(-1, K, c["dim"]).index_copy_(0, at, x[:, H + K:].contiguous())
    return heads[:, :H].contiguous(), kc, vc


def _exact_route(s):
    c = s["case"]
    E, k, n = c["E"], c["k"], c["groups"]
    x = s["logits"].cpu().numpy().astype(np.float64)
    if c["scoring"] == "softmax":
        score = np.exp(x - x.max(1, keepdims=True))
        score /= score.sum(1, keepdims=True)
    else:
        score = 1 / (1 + np.exp(-x))
    by = score + (0 if s["bias"] is None else s["bias"].cpu().numpy().astype(np.float64))
    if n > 1:
        best = np.sort(by.reshape(len(x), n, E // n), 2)
        best = best[..., -1] + (best[..., -2] if E // n > 1 else 0)
        # groups that fewer than top_groups others come before
        at = np.arange(n)
        ahead = (best[:, None, :] > best[:, :, None]) | \
            ((best[:, None, :] == best[:, :, None]) & (at[None, :] < at[:, None])[None])
        out = np.repeat(ahead.sum(2) >= c["top_groups"], E // n, 1)
        by = np.where(out, -np.inf, by)
    idx = np.argsort(-by, 1, kind="stable")[:, :k]
    w = np.take_along_axis(score, idx, 1)
    if c["renorm"]:
        w = w / w.sum(1, keepdims=True)
    bits = s["bits"].cpu().numpy()[s["req"].cpu().numpy()[:, None], idx]
    L = B_MAX - B_MIN + 1
    key = (idx * L + bits.astype(np.int64) - B_MIN).reshape(-1)
    hist = np.bincount(key, minlength=E * L)
    perm = np.argsort(key, kind="stable")
    slot = np.argsort(perm)
    most = np.array([max([b + B_MIN for b in range(L) if row[b]], default=0)
                     for row in hist.reshape(E, L)])
    return [torch.from_numpy(np.ascontiguousarray(a)).to(DEV) for a in
            (idx, w * c["scale"], bits.astype(np.int64), hist.reshape(E, L),
             np.concatenate(([0], np.cumsum(hist))), perm, slot, most)]


def _exact_sample(s):
    x = s["logits"].float().cpu().numpy()
    conf = {n: None if s[n] is None else s[n].cpu().numpy().astype(np.float64)
            for n in ("u", "temperature", "top_k", "top_p", "min_p")}
    tokens, probs = [], []
    for b, row in enumerate(x):
        at = np.argsort(-row, kind="stable")
        t = conf["temperature"][b]
        if t <= 0:
            tokens.append(int(at[0]))
            probs.append(1.0)
            continue
        if conf["top_k"] is not None and conf["top_k"][b] > 0:
            at = at[:int(conf["top_k"][b])]
        d = row[at].astype(np.float64)
        w = np.exp((d - d[0]) / t)
        n = len(w)
        if conf["top_p"] is not None:
            before = np.concatenate(([0.0], np.cumsum(w)[:-1]))
            n = int(np.searchsorted(before, conf["top_p"][b] * w.sum(), side="left"))
        if conf["min_p"] is not None:
            n = min(n, int((w >= conf["min_p"][b]).sum()))
        run = np.cumsum(w[:n])
        i = int(np.searchsorted(run, conf["u"][b] * run[-1], side="right"))
        tokens.append(int(at[i]))
        probs.append(w[i] / run[-1])
    return (torch.tensor(tokens, device=DEV), torch.tensor(probs, dtype=torch.float64, device=DEV))


def exact(case, seed):
    c = case
    if c["op"] == "sample" and c["B"] * c["V"] > 1 << 25:
        return None     # sorting these rows on the host takes too long
    s = prepare(c, seed)
    return {"prefix": _exact_prefix, "append": _exact_append, "route": _exact_route,
            "sample": _exact_sample}[c["op"]](s)
