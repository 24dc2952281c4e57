"""The decode step of a small decoder as a serving loop runs it: norm, q / k / v
projection, append to the paged cache with rotation, attention, output
projection, norm, routing, experts, norm.  Two layers, ragged sequences, three
steps that feed themselves, against the oracle and the plain binary64 forms with
bf16 where the device has bf16; and the same step captured in a graph."""
import numpy as np
import pytest
import torch

import decoder_ref as ref
from layer_cases import DEV, FWD_TOL, ambiguous_tokens, logit_error_bound, row_max_abs_rel
from oracle import oracle as O
from paper_2504_15299_amd import api
from paper_2504_15299_amd import workloads as wl

pytestmark = pytest.mark.gpu

LAYERS, STEPS, EPS, GROUP, PAGE = 2, 3, 1e-5, 64, 4
HQ, H, D = 4, 2, 64
PAST = [0, 1, 5, 11, 3, 8, 30, 2]


class Decoder:
    def __init__(self):
        self.spec = s = wl.scaled(wl.mixtral_stack(), d=256, f=256, T=len(PAST),
                                  n_requests=len(PAST))
        rng = np.random.default_rng(3)
        self.req, self.table = wl.token_requests(s), wl.bit_table(s)
        width = -(-(max(PAST) + STEPS) // PAGE)
        self.pages = rng.permutation(s.T * width + 1)[:s.T * width].reshape(s.T, width) \
            .astype(np.int32)
        ang = np.arange(width * PAGE)[:, None] / 1e4 ** (np.arange(D // 2) * 2 / D)
        self.cos, self.sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
        self.layers = []
        for l in range(LAYERS):
            Wg, _ = wl.gate(s, l)
            w = {"Wg": Wg,
                 "W13": np.stack([wl.expert_w13(s, e, l) for e in range(s.E)]),
                 "W2": np.stack([wl.expert_w2(s, e, l) for e in range(s.E)])}
            for name, rows, cols in (("qkv", (HQ + 2 * H) * D, s.d), ("o", s.d, HQ * D)):
                w[name] = ref.linear_quantize(
                    (rng.standard_normal((rows, cols)) * cols ** -0.5).astype(np.float32), GROUP)
            w["n1"], w["n2"] = ((1 + rng.standard_normal(s.d) * 0.1).astype(np.float32)
                                for _ in range(2))
            shape = (s.T * width + 1, PAGE, H, D)
            w["k"], w["v"] = (wl.round_to_bf16(rng.standard_normal(shape, dtype=np.float32))
                              for _ in range(2))
            self.layers.append(w)
        self.x0 = rng.standard_normal((s.T, s.d)).astype(np.float32)

    def upload(self):
        s = self.spec
        dev = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
        self.dev = []
        for w in self.layers:
            w13 = api.MWQ.empty(s.E, 2 * s.f, s.d, s.group, device=DEV)
            w2 = api.MWQ.empty(s.E, s.d, s.f, s.group, device=DEV)
            api.pack_mwq(dev(w["W13"]), w13)
            api.pack_mwq(dev(w["W2"]), w2)
            lin = {n: api.linear_pack_codes(*map(dev, w[n]),
                                            api.Linear.empty(*w[n][0].shape, GROUP, device=DEV))
                   for n in ("qkv", "o")}
            self.dev.append({"w13": w13, "w2": w2, "Wg": dev(w["Wg"]), "n1": dev(w["n1"]),
                             "n2": dev(w["n2"]), **lin, "cache": api.KVCache(
                                 dev(w["k"]).bfloat16(), dev(w["v"]).bfloat16())})
        self.x, self.pos = dev(self.x0), dev(np.array(PAST, np.int32))
        self.t = [dev(a) for a in (self.req, self.table, self.pages, self.cos, self.sin)]
        self.h = api.block_norm(self.x, torch.zeros_like(self.x), EPS, self.dev[0]["n1"])
        return self

    def step(self):
        req, table, pages, cos, sin = self.t
        x, h, s = self.x, self.h, self.spec
        lengths = self.pos + 1
        for l, w in enumerate(self.dev):
            qkv = api.linear_forward(h, w["qkv"]).view(s.T, HQ + 2 * H, D)
            q = api.kv_append(qkv[:, :HQ], qkv[:, HQ:HQ + H], qkv[:, HQ + H:], w["cache"], pages,
                              self.pos, cos=cos, sin=sin)
            a = api.attn_decode(q, w["cache"], pages, lengths)
            y = api.linear_forward(a.view(s.T, HQ * D), w["o"])
            h = api.block_norm(x, y, EPS, pre_weight=w["n2"], y_scale=0.7)
            r = api.route(h, w["Wg"], None, s.k, req, table)
            y = api.moe_forward(h, w["w13"], w["w2"], r, s.k)
            h = api.block_norm(x, y, EPS, pre_weight=self.dev[(l + 1) % LAYERS]["n1"], y_scale=0.7,
                               h=self.h)
        self.pos += 1

    def reference(self):
        """The residual stream after every step, and the tokens whose experts
        the device may choose otherwise."""
        s = self.spec
        bf = lambda a: O.round_bf16(a.astype(np.float32)).reshape(a.shape).astype(float)  # noqa: E731
        f = [{k: v.astype(np.float64) if k in ("n1", "n2", "k", "v") else v for k, v in w.items()}
             for w in self.layers]
        c13 = [[O.mwq_quantize(m, s.group) for m in w["W13"]] for w in self.layers]
        c2 = [[O.mwq_quantize(m, s.group) for m in w["W2"]] for w in self.layers]
        x, pos = self.x0.astype(np.float64), np.array(PAST)
        _, h, _, _ = ref.block_norm(x, 0 * x, EPS, pre=f[0]["n1"])
        amb, out = np.zeros(s.T, bool), []
        for _ in range(STEPS):
            for l, w in enumerate(f):
                qkv = bf(ref.linear(bf(h), *w["qkv"], GROUP)[0]).reshape(s.T, HQ + 2 * H, D)
                rot = bf(ref.kv_append(qkv[:, :HQ + H], self.cos.astype(float),
                                       self.sin.astype(float), pos)[0])
                at = self.pages[np.arange(s.T), pos // PAGE], pos % PAGE
                w["k"][at], w["v"][at] = rot[:, HQ:], qkv[:, HQ + H:]
                a = bf(ref.attn(rot[:, :HQ], w["k"], w["v"], self.pages, pos + 1, D ** -0.5)[0])
                y = bf(ref.linear(a.reshape(s.T, HQ * D), *w["o"], GROUP)[0])
                x, h, _, _ = ref.block_norm(x, y, EPS, pre=w["n2"], y_scale=0.7)
                hb = bf(h).astype(np.float32)
                logits = O.gate_logits(hb, w["Wg"])
                amb |= ambiguous_tokens(logits, s.k, 8 * logit_error_bound(
                    np.ones((s.T, s.d), np.float32) * np.abs(hb).max(1, keepdims=True), w["Wg"],
                    None))
                route = O.route_from_logits(logits, s.k, self.req, self.table)
                y = bf(O.moe_layer(hb, route, c13[l], c2[l]))
                x, h, _, _ = ref.block_norm(x, y, EPS, pre=f[(l + 1) % LAYERS]["n1"], y_scale=0.7)
            out.append(x)
            pos = pos + 1
        return out, amb


def test_decode_steps_against_the_oracle():
    d = Decoder()
    want, amb = d.reference()
    assert amb.sum() <= 2
    d.upload()
    for x in want:
        d.step()
        torch.cuda.synchronize()
        err = row_max_abs_rel(d.x.cpu().numpy()[~amb], x[~amb])
        print(f"worst row {err.max():.3e}, near-tied tokens {int(amb.sum())}")
        assert err.max() <= FWD_TOL
    assert d.pos.tolist() == [p + STEPS for p in PAST]


def test_captured_step_replays_like_the_eager_one():
    a, b = Decoder().upload(), Decoder().upload()
    x0, h0 = b.x.clone(), b.h.clone()
    caches = [(w["cache"].k.clone(), w["cache"].v.clone()) for w in b.dev]
    b.step()                                    # warm-up, undone below
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.step()
    b.x.copy_(x0)
    b.h.copy_(h0)
    b.pos.copy_(torch.tensor(PAST, dtype=torch.int32))
    for w, (k, v) in zip(b.dev, caches):
        w["cache"].k.copy_(k)
        w["cache"].v.copy_(v)
    for _ in range(STEPS):
        a.step()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.x, b.x) and torch.equal(a.h, b.h)
        for u, w in zip(a.dev, b.dev):
            assert torch.equal(u["cache"].k, w["cache"].k)
            assert torch.equal(u["cache"].v, w["cache"].v)
