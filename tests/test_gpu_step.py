"""One decode iteration after the other with the operators of a serving loop whose
sequences share a prompt: q / k / v projection, append with head norms and a rotation of
part of a head, attention behind the shared prefix, output projection, norm, experts by
sigmoid scores, norm, and after the last layer the vocabulary's logits and a sampled
token, which the next iteration starts from.  Against the oracle and the plain binary64
forms with bf16 where the device has bf16, and captured in a graph.  And the calls that
only their surroundings make hard."""
import numpy as np
import pytest
import torch

import decoder_ref as ref
import step_ref as step
from layer_cases import DEV, FWD_TOL, ambiguous_tokens, logit_error_bound, row_max_abs_rel
from oracle import oracle as O
from paper_2504_15299_amd import api
from paper_2504_15299_amd import workloads as wl
from test_gpu_decoder_step import D, EPS, GROUP, H, HQ, LAYERS, PAGE, PAST, STEPS, Decoder

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
V, ROT, SCALE = 512, 32, 1.5
SHARED = [0, 0, 0, 8, 0, 8, 6, 0]  # tokens of the prompt that a sequence starts with
PROMPT = 10


class Server(Decoder):
    def __init__(self):
        super().__init__()
        s, rng = self.spec, np.random.default_rng(8)
        for w in self.layers:
            w["qw"], w["kw"] = ((1 + rng.standard_normal(D) * 0.2).astype(np.float32)
                                for _ in range(2))
            # the prompt's pages come behind the sequences' own
            for n in "kv":
                more = wl.round_to_bf16(rng.standard_normal((3, PAGE, H, D), dtype=np.float32))
                w[n] = np.concatenate([w[n], more])
        n_own = len(self.layers[0]["k"]) - 3
        self.prompt = np.array([n_own + 2, n_own, n_own + 1], np.int32)
        for b, n in enumerate(SHARED):
            self.pages[b, :n // PAGE] = -1
        self.cos, self.sin = (a[:, ::2][:, :ROT // 2].copy() for a in (self.cos, self.sin))
        self.head = ref.linear_quantize(
            (rng.standard_normal((V, s.d)) * 3 * s.d ** -0.5).astype(np.float32), GROUP)
        self.emb = rng.standard_normal((V, s.d)).astype(np.float32)
        self.u = rng.random((STEPS, s.T)).astype(np.float32)
        self.settings = (rng.choice([0.0, 0.7, 1.0], s.T).astype(np.float32),
                         rng.integers(0, 40, s.T).astype(np.int32),
                         rng.choice([0.8, 0.95, 1.0], s.T).astype(np.float32),
                         rng.choice([0.0, 0.05], s.T).astype(np.float32))

    def upload(self):
        super().upload()
        dev = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
        for w, l in zip(self.dev, self.layers):
            w["qw"], w["kw"] = dev(l["qw"]), dev(l["kw"])
        self.dprompt, self.dshared = dev(self.prompt), dev(np.array(SHARED, np.int32))
        self.dhead = api.linear_pack_codes(*map(dev, self.head),
                                           api.Linear.empty(V, self.spec.d, GROUP, device=DEV))
        self.demb, self.du = dev(self.emb), dev(self.u)
        self.dset = [dev(a) for a in self.settings]
        self.ui = torch.zeros(self.spec.T, device=DEV)
        self.tokens = torch.arange(self.spec.T, dtype=I32, device=DEV)
        self.probs = torch.zeros(self.spec.T, device=DEV)
        return self

    def step(self):
        req, table, pages, cos, sin = self.t
        s, n = self.spec, self.spec.T
        torch.index_select(self.demb, 0, self.tokens, out=self.x)
        h = api.block_norm(self.x, torch.zeros_like(self.x), EPS, self.dev[0]["n1"])
        lengths = self.pos + 1
        for l, w in enumerate(self.dev):
            qkv = api.linear_forward(h, w["qkv"]).view(n, HQ + 2 * H, D)
            q = api.kv_append_norm(qkv[:, :HQ], qkv[:, HQ:HQ + H], qkv[:, HQ + H:], w["cache"],
                                   pages, self.pos, q_weight=w["qw"], k_weight=w["kw"], eps=EPS,
                                   cos=cos, sin=sin)
            a = api.attn_prefix(q, w["cache"], pages, lengths, self.dprompt, self.dshared,
                                max_prefix=PROMPT)
            y = api.linear_forward(a.view(n, HQ * D), w["o"])
            h = api.block_norm(self.x, y, EPS, pre_weight=w["n2"], y_scale=0.7)
            r = api.route_scored(None, s.k, req, table, "sigmoid", scale=SCALE, x=h, Wg=w["Wg"])
            y = api.moe_forward(h, w["w13"], w["w2"], r, s.k)
            h = api.block_norm(self.x, y, EPS, y_scale=0.7,
                               pre_weight=self.dev[(l + 1) % LAYERS]["n1"])
        self.logits = api.linear_forward(h, self.dhead)
        api.sample(self.logits, self.ui, *self.dset, tokens=self.tokens, probs=self.probs)
        self.pos += 1

    def reference(self):
        """A generator: the tokens that a step starts from, to (residual stream, rows whose
        experts the device may choose otherwise)."""
        s = self.spec
        bf = lambda a: O.round_bf16(a.astype(np.float32)).reshape(a.shape).astype(float)  # noqa: E731
        f = [{k: v.astype(np.float64) if k in ("n1", "n2", "k", "v", "qw", "kw") else v
              for k, v in w.items()} for w in self.layers]
        c13 = [[O.mwq_quantize(m, s.group) for m in w["W13"]] for w in self.layers]
        c2 = [[O.mwq_quantize(m, s.group) for m in w["W2"]] for w in self.layers]
        cos, sin = self.cos.astype(float), self.sin.astype(float)
        pos, amb, x = np.array(PAST), np.zeros(s.T, bool), None
        while True:
            tokens = yield x, amb
            x = self.emb[tokens].astype(np.float64)
            _, h, _, _ = ref.block_norm(x, 0 * x, EPS, pre=f[0]["n1"])
            for l, w in enumerate(f):
                qkv = bf(ref.linear(bf(h), *w["qkv"], GROUP)[0]).reshape(s.T, HQ + 2 * H, D)
                q, k = (bf(step.rotate(*step.head_norm(t, w[n], EPS), cos, sin, pos, False)[0])
                        for t, n in ((qkv[:, :HQ], "qw"), (qkv[:, HQ:HQ + H], "kw")))
                at = self.pages[np.arange(s.T), pos // PAGE], pos % PAGE
                w["k"][at], w["v"][at] = k, qkv[:, HQ + H:]
                a = bf(step.attn_prefix(q, w["k"], w["v"], self.pages, pos + 1, self.prompt,
                                        SHARED, D ** -0.5)[0])
                y = bf(ref.linear(a.reshape(s.T, HQ * D), *w["o"], GROUP)[0])
                x, h, _, _ = ref.block_norm(x, y, EPS, pre=w["n2"], y_scale=0.7)
                hb = bf(h).astype(np.float32)
                logits = O.gate_logits(hb, w["Wg"])
                amb = amb | ambiguous_tokens(logits, s.k, 8 * logit_error_bound(
                    np.ones((s.T, s.d), np.float32) * np.abs(hb).max(1, keepdims=True), w["Wg"],
                    None))
                route = step.route_scored(logits, s.k, self.req, self.table, "sigmoid", None, 1, 1,
                                          True, SCALE, 2, 8)
                y = bf(O.moe_layer(hb, route, c13[l], c2[l]))
                x, h, _, _ = ref.block_norm(x, y, EPS, pre=f[(l + 1) % LAYERS]["n1"], y_scale=0.7)
            pos = pos + 1


def test_iterations_against_the_oracle():
    d = Server().upload()
    want = d.reference()
    next(want)
    for i in range(STEPS):
        start = d.tokens.cpu().numpy()
        d.ui.copy_(d.du[i])
        d.step()
        torch.cuda.synchronize()
        x, amb = want.send(start)
        assert amb.sum() <= 2
        err = row_max_abs_rel(d.x.cpu().numpy()[~amb], x[~amb])
        print(f"worst row {err.max():.3e}, near-tied tokens {int(amb.sum())}")
        assert err.max() <= FWD_TOL
        logits, tokens = d.logits.float().cpu().numpy(), d.tokens.tolist()
        for b, t in enumerate(tokens):
            token, share, room = step.sample(logits[b], float(d.u[i, b]),
                                             *(float(a[b]) for a in d.settings[:1]),
                                             int(d.settings[1][b]), float(d.settings[2][b]),
                                             float(d.settings[3][b]))
            assert room > 1e-9 and t == token
            # 512 weights, each within 2^-42 of the largest, and the rounding to binary32
            assert abs(float(d.probs[b]) - share) <= 2.0 ** -24 * share + 2.0 ** -32
    assert d.pos.tolist() == [p + STEPS for p in PAST]


def test_captured_iteration_replays_like_the_eager_one():
    a, b = Server().upload(), Server().upload()
    caches = [(w["cache"].k.clone(), w["cache"].v.clone()) for w in b.dev]
    first = b.tokens.clone()
    b.step()                                    # warm-up, undone below
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.step()
    b.tokens.copy_(first)
    b.pos.copy_(torch.tensor(PAST, dtype=I32))
    for w, (k, v) in zip(b.dev, caches):
        w["cache"].k.copy_(k)
        w["cache"].v.copy_(v)
    for i in range(STEPS):
        for d in (a, b):
            d.ui.copy_(d.du[i])
        a.step()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.tokens, b.tokens) and torch.equal(a.probs, b.probs)
        assert torch.equal(a.x, b.x)
        for u, w in zip(a.dev, b.dev):
            assert torch.equal(u["cache"].k, w["cache"].k)
            assert torch.equal(u["cache"].v, w["cache"].v)


def on_stream(name, s):
    """One call of the operator on stream s with a result of 512 bf16, 256 ints or floats
    of its own."""
    cache = api.KVCache.empty(8, 16, 2, 64, BF, DEV)
    cache.k.normal_()
    cache.v.normal_()
    table = torch.arange(8, dtype=I32, device=DEV).view(2, 4)
    q = torch.randn((2, 4, 64), dtype=BF, device=DEV)
    pos = torch.tensor([3, 60], dtype=I32, device=DEV)
    logits, u = torch.randn((256, 100), device=DEV), torch.rand(256, device=DEV)
    scores = torch.randn((128, 8), device=DEV)
    bits = torch.full((1, 8), 4, dtype=torch.uint8, device=DEV)
    return {
        "kv_append_norm": lambda: api.kv_append_norm(q, q[:, :2], q[:, 2:], cache, table, pos,
                                                     stream=s),
        "attn_prefix": lambda: api.attn_prefix(q, cache, table, pos, table[0], pos, stream=s),
        "sample": lambda: api.sample(logits, u, stream=s),
        "route_scored": lambda: api.route_scored(scores, 2, None, bits, stream=s),
    }[name]


@pytest.mark.parametrize("name", ["kv_append_norm", "attn_prefix", "sample", "route_scored"])
def test_result_on_another_stream_does_not_take_memory_in_use(name):
    """Memory of the current stream, freed while work on it is still to run: the call's
    results on the other stream must not be there."""
    s = torch.cuda.Stream()
    run = on_stream(name, s)
    slow = torch.ones(1 << 28, device=DEV)
    torch.cuda.synchronize()
    old = [torch.full((512,), 7.0, dtype=BF, device=DEV) for _ in range(12)]
    torch.cuda.synchronize()
    for _ in range(40):
        slow.mul_(1.0)
    kept = [t.clone() for t in old]
    del old
    out = run()
    torch.cuda.synchronize()
    assert out is not None and all((t == 7.0).all() for t in kept)


def test_threads_on_their_own_streams():
    """Calls of four threads at once, each on a stream of its own, like one after the
    other."""
    import threading
    sets = []
    for i in range(4):
        torch.manual_seed(i)
        cache = api.KVCache.empty(600, 16, 2, 128, BF, DEV)
        cache.k.normal_()
        cache.v.normal_()
        table = torch.randperm(600, device=DEV).to(I32)
        sets.append(dict(
            cache=cache, prompt=table[:200].clone(), own=table[200:].view(5, 80).clone(),
            q=torch.randn((5, 16, 128), device=DEV).to(BF),
            lengths=torch.tensor([3000 + i, 3200, 2999, 4000, 77], dtype=I32, device=DEV),
            shared=torch.tensor([3000, 3000, 1000, 2990 + i, 100], dtype=I32, device=DEV),
            scores=torch.randn((700 + i, 16), device=DEV),
            bits=torch.randint(2, 9, (1, 16), device=DEV).to(torch.uint8),
            logits=torch.randn((6, 40000), device=DEV) * 3, u=torch.rand(6, device=DEV),
            top_p=torch.full((6,), 0.9, device=DEV), stream=torch.cuda.Stream()))

    def calls(c, stream):
        a = api.attn_prefix(c["q"], c["cache"], c["own"], c["lengths"], c["prompt"], c["shared"],
                            stream=stream)
        r = api.route_scored(c["scores"], 3, None, c["bits"], "sigmoid", stream=stream)
        t, p = api.sample(c["logits"], c["u"], top_p=c["top_p"], stream=stream)
        return a, r.topk_idx, r.topk_w, r.perm, r.slot_of, r.hist, t, p

    want = [calls(c, None) for c in sets]
    torch.cuda.synchronize()
    got = [[] for _ in sets]

    def work(i):
        for _ in range(10):
            got[i].append(calls(sets[i], sets[i]["stream"]))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for w, runs in zip(want, got):
        assert len(runs) == 10
        for g in runs:
            assert all(torch.equal(a, b) for a, b in zip(w, g))
