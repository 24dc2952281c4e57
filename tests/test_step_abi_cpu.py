"""Refusals of the normed append, scored routing, sampling and shared-prefix attention,
on the host: nothing is launched (the pointers are fake and would fault if used)."""
import ctypes

import pytest
import torch

from paper_2504_15299_amd import api
from test_decoder_abi_cpu import BAD_CACHES, FAKE, ODD, cache, refuses


def append_norm(**kw):
    d = dict(q=FAKE, qs=512, h=8, k=FAKE, v=FAKE, ks=256, t=1, N=3, c=cache(), bt=FAKE, ns=2, mp=3,
             p=FAKE, sq=None, qw=FAKE, kw=FAKE, eps=1e-6, co=FAKE, si=FAKE, nr=100, rd=64, il=0,
             qo=2 * FAKE, s=None)
    d.update(kw)
    return d


def test_kv_append_norm_refusals():
    ok = append_norm()
    refuses("d2moe_kv_append_norm", ok, [dict(c=cache(**b)) for b in BAD_CACHES])
    refuses("d2moe_kv_append_norm", ok, [
        dict(N=-1), dict(N=(1 << 30) + 1), dict(ns=-1), dict(mp=-1), dict(k=None), dict(v=None),
        dict(p=None), dict(bt=None), dict(qo=None), dict(co=None), dict(si=None), dict(nr=-1),
        dict(h=0), dict(h=70000), dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(qo=2 * FAKE + 8),
        dict(co=FAKE + 4), dict(si=FAKE + 4), dict(qw=ODD), dict(kw=ODD), dict(qs=504),
        dict(qs=516), dict(ks=248), dict(ks=260), dict(eps=-1.0), dict(eps=float("nan")),
        dict(rd=0), dict(rd=2), dict(rd=66), dict(rd=68), dict(rd=-4), dict(il=2), dict(il=-1),
        dict(qo=FAKE, qs=1024),                       # in place, rows not packed
        dict(qo=FAKE, t=0), dict(qo=FAKE, c=cache(dtype=0))])
    refuses("d2moe_kv_append_norm", ok, [dict(t=2), dict(t=-1)], api.EUNSUPPORTED)
    # no tokens: nothing is done
    refuses("d2moe_kv_append_norm", ok, [dict(N=0), dict(N=0, co=None, si=None, rd=0)], api.OK)


def test_kv_append_norm_binding_refusals():
    c = api.KVCache.empty(2, 4, 1, 8, dtype=torch.float32, device="cpu")
    x, one = torch.zeros((1, 1, 8)), torch.zeros(1, dtype=torch.int32)
    t = torch.zeros((3, 4))
    for kw in (dict(cos=t[:0], sin=t[:0]), dict(cos=t, sin=t[:2]), dict(cos=t, sin=t[:, :2]),
               dict(q_weight=torch.ones(4)), dict(k_weight=torch.ones(8).bfloat16()), dict(sin=t),
               dict(cos=t, sin=t)):                   # (the last: tensors on the host)
        with pytest.raises(ValueError):
            api.kv_append_norm(x, x, x, c, one[None], one, **kw)


def routing():
    return api._Routing(*([FAKE] * 10))


def test_route_scored_refusals():
    ok = dict(x=FAKE, xt=1, T=5, d=64, w=FAKE, b=None, E=16, k=4, sc=1, sb=None, g=4, tg=2, rn=1,
              s=1.0, rq=None, bt=FAKE, R=2, lo=2, hi=8, o=routing(), st=None)
    nan, inf = float("nan"), float("inf")
    refuses("d2moe_route_scored", ok, [
        dict(T=-1), dict(E=0), dict(E=65), dict(k=0), dict(k=17), dict(k=9), dict(sc=2),
        dict(sc=-1), dict(g=0), dict(g=3), dict(g=-4), dict(g=32), dict(tg=0), dict(tg=5),
        dict(rn=2), dict(s=nan), dict(s=inf), dict(R=0), dict(lo=0), dict(hi=9), dict(lo=5, hi=4),
        dict(d=0), dict(w=None), dict(bt=None), dict(o=None), dict(T=1 << 29)])
    for f, _ in api._Routing._fields_:
        r = routing()
        setattr(r, f, None)
        refuses("d2moe_route_scored", ok, [dict(o=r), dict(o=r, x=None)])
    refuses("d2moe_route_scored", ok, [dict(xt=2), dict(xt=-1)], api.EUNSUPPORTED)


def test_route_scored_binding_refusals():
    x, table = torch.zeros((3, 8)), torch.full((1, 8), 4, dtype=torch.uint8)
    for kw in (dict(scoring="relu"), dict(x=x), dict(Wg=x), dict(select_bias=torch.zeros(7)),
               dict(token_req=torch.zeros(3)), dict(out=api.Routing.empty(4, 8, 2, device="cpu")),
               dict(logits=x.double()), dict(logits=None), dict(logits=None, x=x), dict(b_min=9),
               dict(bit_table=table.int()), dict(bit_table=table[:, :7]), {}):
        a = {**dict(logits=x, k=2, token_req=None, bit_table=table), **kw}
        with pytest.raises(ValueError):       # (the last: tensors on the host)
            api.route_scored(**a)


def test_sample_refusals():
    ok = dict(x=FAKE, xt=0, s=100, B=3, V=100, u=FAKE, t=None, k=None, p=None, m=None, o=FAKE,
              pr=None, st=None)
    refuses("d2moe_sample", ok, [dict(x=None), dict(u=None), dict(o=None), dict(B=-1),
                                 dict(B=(1 << 24) + 1), dict(V=0), dict(V=-1), dict(s=99),
                                 dict(V=(1 << 24) + 1, s=1 << 25), dict(x=FAKE + 2),
                                 dict(x=FAKE + 1, xt=1)])
    refuses("d2moe_sample", ok, [dict(xt=2), dict(xt=-1)], api.EUNSUPPORTED)
    refuses("d2moe_sample", ok, [dict(B=0), dict(B=0, x=None, u=None, o=None)], api.OK)


def test_sample_binding_refusals():
    x, u = torch.zeros((3, 8)), torch.zeros(3)
    for kw in (dict(u=u[:2]), dict(u=u.double()), dict(top_k=u), dict(top_p=u.half()),
               dict(temperature=u[None]), dict(logits=x.t().contiguous().t()),
               dict(tokens=u), dict(probs=u.int()), {}):
        with pytest.raises(ValueError):       # (the last: tensors on the host)
            api.sample(**{**dict(logits=x, u=u), **kw})
    with pytest.raises(TypeError):
        api.sample(x.half(), u)


def test_attn_prefix_refusals():
    ok = dict(q=FAKE, qs=512, B=3, h=8, c=cache(), bt=FAKE, mp=300, ln=FAKE, pt=FAKE, pp=200,
              pl=FAKE, mx=3200, mr=1600, sc=0.125, o=FAKE, ws=FAKE, n=1 << 40, s=None)
    refuses("d2moe_attn_prefix", ok, [dict(c=cache(**b)) for b in BAD_CACHES])
    refuses("d2moe_attn_prefix", ok, [
        dict(q=None), dict(o=None), dict(ln=None), dict(bt=None), dict(pt=None), dict(pl=None),
        dict(q=ODD), dict(o=ODD), dict(qs=504), dict(qs=516), dict(B=-1), dict(B=65536),
        dict(B=65535, h=128, qs=8192), dict(h=0), dict(h=6), dict(h=3), dict(h=65536),
        dict(mp=-1), dict(mp=(1 << 26) + 1), dict(pp=-1), dict(pp=(1 << 26) + 1), dict(mx=-1),
        dict(mr=-1), dict(mx=(1 << 30) + 1), dict(mr=(1 << 30) + 1), dict(sc=float("nan")),
        dict(sc=float("inf")), dict(sc=2.5e38)])
    refuses("d2moe_attn_prefix", ok, [dict(ws=None), dict(ws=ODD), dict(n=16)], api.EWORKSPACE)
    refuses("d2moe_attn_prefix", ok, [dict(B=0)], api.OK)


def test_attn_prefix_workspace():
    """Grows with either length expected."""
    n = ctypes.c_size_t()

    def need(*a):
        assert api.lib().d2moe_attn_prefix_workspace(*a, ctypes.byref(n)) == 0
        return n.value

    assert need(0, 8, 8, 64, 10 ** 6, 10 ** 6) == 0 < need(1, 1, 1, 8, 0, 0)
    for B, hq, h, d in ((1, 8, 2, 64), (16, 32, 8, 128), (64, 32, 8, 128), (9, 12, 12, 256)):
        last = 0
        for length in list(range(0, 20000, 37)) + [1 << 30]:
            assert need(B, hq, h, d, length, length // 3) >= last
            last = need(B, hq, h, d, length, length // 3)
    for args in ((-1, 8, 8, 64, 1, 1), (1, 7, 2, 64, 1, 1), (1, 8, 8, 60, 1, 1),
                 (1, 8, 8, 64, -1, 1), (1, 8, 8, 64, 1, -1)):
        assert api.lib().d2moe_attn_prefix_workspace(*args, ctypes.byref(n)) == api.EINVAL
    assert api.lib().d2moe_attn_prefix_workspace(1, 8, 8, 64, 1, 1, None) == api.EINVAL
