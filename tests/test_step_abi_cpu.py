"""Refusals of the entry points for head norms with the append, on the host: nothing
is launched (the pointers are fake and would fault if used)."""
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
