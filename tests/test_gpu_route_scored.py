"""Routing by softmax or sigmoid scores with a balance bias and groups: choices, counts
and permutation equal to the plain form's, weights within their rounding."""
import numpy as np
import pytest
import torch

import step_ref as step
from layer_cases import DEV
from oracle import oracle as O
from paper_2504_15299_amd import api
from paper_2504_15299_amd import workloads as wl

pytestmark = pytest.mark.gpu

F32, I32 = torch.float32, torch.int32


def gpu(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def check(r, want):
    for name, w in want.items():
        got = getattr(r, name).cpu().numpy()
        if name == "topk_w":
            # binary64 up to one rounding (the sums' order may turn it)
            assert (np.abs(got - w) <= 2.0 ** -24 * (1 + 1e-6) * np.abs(w) + 1e-45).all()
        else:
            assert np.array_equal(got.astype(int), w), name


def run(T, E, k, scoring="softmax", bias=False, groups=1, top_groups=1, renorm=True, scale=1.0,
        b_min=2, b_max=8, R=5, seed=0, logits=None, req=True):
    rng = np.random.default_rng(seed + T)
    if logits is None:
        logits = (rng.standard_normal((T, E)) * 1.5).astype(np.float32)
    sb = (rng.standard_normal(E) * 0.1).astype(np.float32) if bias else None
    table = rng.integers(b_min, b_max + 1, (R, E)).astype(np.uint8)
    token_req = rng.integers(0, R, T).astype(np.int32) if req else None
    a = (token_req, table, scoring, sb, groups, top_groups, renorm, scale, b_min, b_max)
    want = step.route_scored(logits, k, *a)
    before = gpu(logits)
    r = api.route_scored(before, k, gpu(token_req), gpu(table), scoring, gpu(sb), groups,
                         top_groups, renorm, scale, b_min=b_min, b_max=b_max)
    check(r, want)
    assert r.logits is before and np.array_equal(before.cpu().numpy(), logits, equal_nan=True)
    return r


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("renorm,scale", [(True, 1.0), (False, 2.5)])
@pytest.mark.parametrize("T", [1, 16, 64, 65, 400])
def test_scores_and_weights(T, scoring, bias, renorm, scale):
    run(T, 8, 2, scoring, bias, renorm=renorm, scale=scale)
    run(T, 64, 6, scoring, bias, renorm=renorm, scale=scale)


@pytest.mark.parametrize("E,groups,top,k", [(64, 8, 4, 8), (64, 8, 1, 8), (64, 64, 7, 7),
                                            (64, 2, 1, 32), (60, 4, 3, 6), (60, 2, 1, 5),
                                            (33, 11, 4, 12), (63, 3, 2, 1), (6, 6, 6, 6),
                                            (10, 5, 2, 3), (1, 1, 1, 1), (2, 2, 1, 1)])
@pytest.mark.parametrize("T", [7, 90])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_groups(E, groups, top, k, T, scoring):
    run(T, E, k, scoring, True, groups, top, seed=E)


# one workgroup, a wave a token, and blocks of slots, at their borders: n = T k of
# 2047, 2048, 2049, whole and part blocks, the last one nearly twice as long
@pytest.mark.parametrize("T,k", [(0, 2), (1, 64), (31, 64), (32, 64), (64, 32), (63, 32), (64, 31),
                                 (89, 23), (2047, 1), (2048, 1), (2049, 1), (3071, 1), (683, 3),
                                 (1024, 7), (8191, 2), (70000, 1)])
def test_sizes(T, k):
    run(T, 64, k, "sigmoid", seed=k)


@pytest.mark.parametrize("b_min,b_max", [(1, 8), (2, 2), (8, 8), (1, 1), (3, 6)])
@pytest.mark.parametrize("T", [20, 900])
def test_ladders(T, b_min, b_max):
    run(T, 64, 4, b_min=b_min, b_max=b_max)
    run(T, 5, 4, b_min=b_min, b_max=b_max, R=1, req=False)


@pytest.mark.parametrize("T", [40, 3000])
@pytest.mark.parametrize("groups,top", [(1, 1), (4, 2)])
@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
def test_ties_and_infinities(T, groups, top, scoring):
    """Few distinct logits, some masked, rows with nothing but masked ones: ties go to
    the lower index, of groups too."""
    rng = np.random.default_rng(T)
    x = rng.integers(-1, 2, (T, 16)).astype(np.float32)
    x[rng.random((T, 16)) < 0.3] = -np.inf
    x[3], x[T - 1] = -np.inf, -np.inf
    x[5, 9] = x[5, 2] = np.inf
    run(T, 16, 4, scoring, groups=groups, top_groups=top, logits=x)


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("T", [3, 100])
def test_nan_is_chosen_last(scoring, T):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((T, 8)).astype(np.float32)
    x[1, 3] = np.nan
    x[2] = np.nan
    table = np.full((1, 8), 4, np.uint8)
    r = api.route_scored(gpu(x), 3, None, gpu(table), scoring)
    idx, w = r.topk_idx.cpu().numpy(), r.topk_w.cpu().numpy()
    rest = np.delete(x, 3, 1)
    want = step.route_scored(rest[1:2], 3, None, table[:, :7], scoring, None, 1, 1, True, 1.0, 2, 8)
    at = want["topk_idx"][0]
    assert (idx[1] == at + (at >= 3)).all()
    assert np.allclose(w[1], want["topk_w"][0], rtol=2.0 ** -23)
    assert (idx[2] == [0, 1, 2]).all()
    x[1, 3] = -50.0
    want = step.route_scored(x[:1], 3, None, table, scoring, None, 1, 1, True, 1.0, 2, 8)
    assert (idx[0] == want["topk_idx"][0]).all()
    assert sorted(r.perm.cpu().tolist()) == list(range(3 * T))


@pytest.mark.parametrize("T", [10, 100, 3000])
def test_flags(T):
    rng = np.random.default_rng(0)
    x = rng.standard_normal((T, 8)).astype(np.float32)
    for bad_req, bad_bits in ((True, False), (False, True), (True, True)):
        table = rng.integers(2, 9, (3, 8)).astype(np.uint8)
        req = rng.integers(0, 3, T).astype(np.int32)
        if bad_req:
            req[T - 1], req[0] = 3, -7
        if bad_bits:
            table[1], table[2, 1] = 9, 1
        a = (req, table, "sigmoid", None, 1, 1, True, 1.0, 2, 8)
        check(api.route_scored(gpu(x), 4, gpu(req), gpu(table), "sigmoid"),
              step.route_scored(x, 4, *a))


@pytest.mark.parametrize("dtype", [torch.bfloat16, F32])
@pytest.mark.parametrize("T", [4, 130])
def test_logits_from_activations(dtype, T):
    """The logits are d2moe_route's, to the last bit, the rest follows from them; and a
    softmax over everything, renormalised, chooses and weighs like a softmax over the
    chosen."""
    x = torch.randn((T, 256), device=DEV).to(dtype)
    Wg, bias = torch.randn((8, 256), device=DEV) * 0.1, torch.randn(8, device=DEV)
    table = torch.randint(2, 9, (1, 8), device=DEV).to(torch.uint8)
    a = api.route(x, Wg, bias, 2, None, table)
    b = api.route_scored(None, 2, None, table, x=x, Wg=Wg, bias=bias)
    for f in ("logits", "topk_idx", "topk_bits", "hist", "offsets", "perm", "slot_of",
              "expert_maxbit", "flags"):
        assert torch.equal(getattr(a, f), getattr(b, f)), f
    # binary32 there: two exponentials, a sum and a division
    assert ((a.topk_w - b.topk_w).abs() <= 16 * 2.0 ** -24 * b.topk_w).all()


def test_result_given_and_graph():
    """Into a result kept by the caller, captured and replayed over other logits."""
    T, E, k = 500, 32, 5
    out = api.Routing.empty(T, E, k, device=DEV)
    x = torch.randn((T, E), device=DEV)
    table = torch.randint(2, 9, (1, E), device=DEV).to(torch.uint8)
    kept = out.logits.fill_(3.0)

    def step_():
        return api.route_scored(x, k, None, table, "sigmoid", groups=4, top_groups=2, out=out)

    step_()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r = step_()
    assert r.topk_idx is out.topk_idx and r.logits is x and (kept == 3.0).all()
    for _ in range(3):
        x.normal_()
        g.replay()
        got = [t.clone() for t in (r.topk_idx, r.topk_w, r.hist, r.perm, r.slot_of)]
        e = api.route_scored(x, k, None, table, "sigmoid", groups=4, top_groups=2)
        torch.cuda.synchronize()
        for a, b in zip(got, (e.topk_idx, e.topk_w, e.hist, e.perm, e.slot_of)):
            assert torch.equal(a, b)


def test_layer_on_its_routing():
    """The MoE layer takes this routing like any other."""
    spec = wl.scaled(wl.tiny(seed=0), T=16)
    x, table = wl.activations(spec), wl.bit_table(spec)
    Wg, _ = wl.gate(spec)
    W13 = np.stack([wl.expert_w13(spec, e) for e in range(spec.E)])
    W2 = np.stack([wl.expert_w2(spec, e) for e in range(spec.E)])
    w13 = api.pack_mwq(gpu(W13), api.MWQ.empty(spec.E, 2 * spec.f, spec.d, spec.group, device=DEV))
    w2 = api.pack_mwq(gpu(W2), api.MWQ.empty(spec.E, spec.d, spec.f, spec.group, device=DEV))
    r = api.route_scored(None, spec.k, None, gpu(table), "sigmoid", groups=4, top_groups=2,
                         scale=1.5, x=gpu(x), Wg=gpu(Wg))
    got = api.moe_forward(gpu(x), w13, w2, r, spec.k).float().cpu().numpy()
    want = step.route_scored(r.logits.cpu().numpy(), spec.k, None, table, "sigmoid", None, 4, 2,
                             True, 1.5, 2, 8)
    check(r, want)
    ref = O.moe_layer(x, want | {"topk_w": want["topk_w"].astype(np.float32)},
                      [O.mwq_quantize(m, spec.group) for m in W13],
                      [O.mwq_quantize(m, spec.group) for m in W2])
    assert (np.abs(got - ref).max(1) / np.abs(ref).max(1)).max() <= 2e-2
