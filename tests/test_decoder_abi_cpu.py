"""Host-side checks of the decode operators' entry points that need no GPU:
sizes follow the packed format, and invalid arguments are refused before
anything is launched (the pointers are fake and would fault if used)."""
import ctypes

import pytest
import torch

from paper_2504_15299_amd import api

FAKE = 1 << 20
ODD = FAKE + 8          # not a multiple of 16


def refuses(name, args, bad, status=api.EINVAL):
    """The call with each change of `bad` applied to the valid arguments."""
    fn = getattr(api.lib(), name)
    for change in bad:
        a = {**args, **change}
        a = [ctypes.byref(v) if isinstance(v, ctypes.Structure) else v for v in a.values()]
        assert fn(*a) == status, (name, change)


def linear(**kw):
    d = dict(rows=48, cols=256, group=64, codes=FAKE, scales=FAKE, zeros=FAKE)
    d.update(kw)
    return api._Linear(**d)


BAD_LINEARS = [dict(rows=0), dict(rows=(1 << 27) + 1), dict(rows=-16), dict(cols=0), dict(cols=-256), dict(cols=200),
               dict(cols=32), dict(group=16), dict(group=0), dict(group=256), dict(codes=0),
               dict(scales=0), dict(zeros=0), dict(codes=ODD), dict(cols=(1 << 22) + 64)]


@pytest.mark.parametrize("rows,cols,group", [(1, 32, 32), (16, 128, 128), (17, 160, 32),
                                             (1003, 1984, 64), (32000, 4096, 128)])
def test_linear_size(rows, cols, group):
    blocks = -(-rows // 16) * -(-cols // 128)
    assert api.linear_size(rows, cols, group) == (
        blocks * 1024, blocks * 16 * (128 // group) * 2, blocks * 16 * (128 // group))


def test_linear_refusals():
    with pytest.raises(api.D2MoEError):
        api.linear_size(16, 100, 64)
    bad = [dict(w=linear(**b)) for b in BAD_LINEARS]
    refuses("d2moe_linear_pack", dict(W=FAKE, t=0, w=linear(), s=None), bad + [dict(W=None)])
    refuses("d2moe_linear_pack", dict(W=FAKE, t=0, w=linear(), s=None), [dict(t=1), dict(t=7)],
            api.EUNSUPPORTED)
    refuses("d2moe_linear_pack_codes", dict(c=FAKE, sc=FAKE, z=None, w=linear(), s=None),
            bad + [dict(c=None), dict(sc=None)])
    ok = dict(x=FAKE, xt=1, T=4, w=linear(), b=None, y=FAKE, yt=1, s=None)
    refuses("d2moe_linear_forward", ok, bad + [dict(x=None), dict(y=None), dict(x=ODD),
                                               dict(T=-1), dict(T=(1 << 20) + 1)])
    refuses("d2moe_linear_forward", ok, [dict(xt=2), dict(yt=-1)], api.EUNSUPPORTED)
    assert api.lib().d2moe_linear_forward(None, 1, 0, ctypes.byref(linear()), None, None, 1,
                                          None) == api.OK


def cache(**kw):
    d = dict(n_pages=10, page_size=16, n_heads=4, head_dim=64, dtype=1, page_stride=4096,
             token_stride=256, head_stride=64, k=FAKE, v=FAKE)
    d.update(kw)
    return api._KVCache(**d)


BAD_CACHES = [dict(n_pages=0), dict(page_size=0), dict(n_heads=0), dict(head_dim=0),
              dict(head_dim=60), dict(head_dim=264), dict(dtype=2), dict(k=0), dict(v=0),
              dict(k=ODD), dict(v=ODD), dict(page_stride=0), dict(page_stride=-4096),
              dict(token_stride=252), dict(head_stride=32),       # rows would overlap
              dict(page_stride=4095), dict(page_stride=4100),     # not multiples of 16 bytes
              dict(page_stride=3840), dict(page_stride=1 << 62)]


def test_cache_strides():
    """Any order of the dimensions whose rows do not overlap, unused strides
    whatever they are."""
    ok = dict(q=None, qs=0, h=0, k=FAKE, v=FAKE, ks=256, t=1, N=0, c=cache(), bt=FAKE, ns=2, mp=3,
              p=FAKE, sq=None, co=None, si=None, nr=0, qo=None, s=None)
    for good in (cache(), cache(token_stride=64, head_stride=1024),
                 cache(page_stride=64, token_stride=2560, head_stride=640),
                 cache(page_stride=8192), cache(n_pages=1, page_stride=1),
                 cache(n_heads=1, head_stride=-3, token_stride=64),
                 cache(dtype=0, token_stride=260, page_stride=4160)):
        refuses("d2moe_kv_append", ok, [dict(c=good)], api.OK)       # no tokens: nothing is done


def test_kv_append_refusals():
    ok = dict(q=FAKE, qs=512, h=8, k=FAKE, v=FAKE, ks=256, t=1, N=3, c=cache(), bt=FAKE, ns=2, mp=3,
              p=FAKE, sq=None, co=FAKE, si=FAKE, nr=100, qo=2 * FAKE, s=None)
    refuses("d2moe_kv_append", ok, [dict(c=cache(**b)) for b in BAD_CACHES])
    refuses("d2moe_kv_append", ok, [
        dict(N=-1), dict(N=(1 << 30) + 1), dict(ns=-1), dict(mp=-1), dict(k=None), dict(v=None),
        dict(p=None), dict(bt=None), dict(qo=None), dict(co=None), dict(si=None), dict(nr=-1), dict(h=0),
        dict(h=70000), dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(qo=2 * FAKE + 8),
        dict(co=FAKE + 4), dict(si=FAKE + 4), dict(qs=504), dict(qs=516), dict(ks=248),
        dict(ks=260),
        dict(qo=FAKE, qs=1024),                       # in place, rows not packed
        dict(qo=FAKE, t=0), dict(qo=FAKE, c=cache(dtype=0))])
    refuses("d2moe_kv_append", ok, [dict(t=2), dict(t=-1)], api.EUNSUPPORTED)


def test_kv_append_with_an_empty_rotation():
    """Tokens past the rotation's rows are not written; without any rows they must not be
    written unrotated."""
    c = api.KVCache.empty(2, 4, 1, 8, dtype=torch.float32, device="cpu")
    x, one = torch.zeros((1, 1, 8)), torch.zeros(1, dtype=torch.int32)
    none = torch.empty((0, 4))
    with pytest.raises(ValueError, match="a row"):
        api.kv_append(x, x, x, c, one[None], one, cos=none, sin=none)


def test_attn_decode_refusals():
    ok = dict(q=FAKE, qs=512, B=3, h=8, c=cache(), bt=FAKE, mp=300, ln=FAKE, ml=4800, w=0, sc=0.125,
              o=FAKE, ws=FAKE, n=1 << 30, s=None)
    refuses("d2moe_attn_decode", ok, [dict(c=cache(**b)) for b in BAD_CACHES])
    refuses("d2moe_attn_decode", ok, [
        dict(q=None), dict(o=None), dict(ln=None), dict(bt=None), dict(q=ODD), dict(o=ODD),
        dict(qs=504), dict(qs=516), dict(B=-1), dict(B=65536),
        dict(B=65535, h=128, qs=8192), dict(h=0), dict(h=6), dict(h=3),
        dict(h=65536), dict(mp=-1), dict(mp=(1 << 26) + 1), dict(ml=-1), dict(w=-1), dict(sc=float("nan")),
        dict(sc=float("inf"))])
    refuses("d2moe_attn_decode", ok, [dict(ws=None), dict(ws=ODD), dict(n=16)], api.EWORKSPACE)
    refuses("d2moe_attn_decode", ok, [dict(B=0)], api.OK)


def test_attn_decode_scale_that_overflows():
    """Scores are scaled in units of log2, where the largest scales have no number: 0
    times infinity would take the place of a score of 0."""
    ok = dict(q=FAKE, qs=512, B=3, h=8, c=cache(), bt=FAKE, mp=300, ln=FAKE, ml=4800, w=0, sc=0.125,
              o=FAKE, ws=None, n=0, s=None)
    refuses("d2moe_attn_decode", ok, [dict(sc=2.5e38), dict(sc=-2.5e38), dict(sc=3.4e38)])
    refuses("d2moe_attn_decode", ok, [dict(sc=2e38), dict(sc=-2e38), dict(sc=0.0)], api.EWORKSPACE)


def test_attn_decode_over_queries_that_are_not_packed():
    """A result over strided queries would overwrite rows that are still to be read."""
    bad = dict(q=FAKE, qs=1024, B=2, h=8, c=cache(), bt=FAKE, mp=300, ln=FAKE, ml=4800, w=0, sc=0.125,
               o=FAKE, ws=None, n=0, s=None)
    refuses("d2moe_attn_decode", bad, [dict(), dict(B=64), dict(qs=520), dict(ws=FAKE, n=1 << 30)])
    # one sequence, packed rows, another result: the workspace is what is missing then
    refuses("d2moe_attn_decode", bad, [dict(B=1), dict(qs=512), dict(o=2 * FAKE)], api.EWORKSPACE)


def test_attn_decode_workspace():
    """Grows with the length expected, so that one made for the longest serves
    them all; a call that does not divide its keys needs none."""
    n = ctypes.c_size_t()

    def need(B, hq, h, d, length):
        assert api.lib().d2moe_attn_decode_workspace(B, hq, h, d, length, ctypes.byref(n)) == 0
        return n.value

    assert need(1, 8, 8, 64, 0) == need(1, 8, 8, 64, 128) == need(0, 8, 8, 64, 10 ** 6) == 0
    assert need(4096, 32, 8, 128, 10 ** 6) == 0 < need(64, 32, 8, 128, 4096)
    last = 0
    for length in range(0, 40000, 37):
        assert need(2, 8, 2, 64, length) >= last
        last = need(2, 8, 2, 64, length)
    for args in ((-1, 8, 8, 64, 1), (1, 7, 2, 64, 1), (1, 8, 8, 60, 1), (1, 8, 8, 64, -1)):
        assert api.lib().d2moe_attn_decode_workspace(*args, ctypes.byref(n)) == api.EINVAL
    assert api.lib().d2moe_attn_decode_workspace(1, 8, 8, 64, 1, None) == api.EINVAL


def test_block_norm_refusals():
    ok = dict(x=FAKE, xs=1.0, y=FAKE, yt=1, ys=1.0, pw=None, g=FAKE, gt=0, gs=0, qw=None, T=3, d=64,
              eps=1e-5, h=FAKE, ht=1, s=None)
    refuses("d2moe_block_norm", ok, [
        dict(x=None), dict(y=None), dict(T=-1), dict(d=0), dict(d=16385), dict(eps=-1.0),
        dict(eps=float("nan")), dict(yt=2), dict(gt=2), dict(ht=-1), dict(gs=63), dict(gs=-64)])
    refuses("d2moe_block_norm", ok, [dict(T=0)], api.OK)


def test_block_norm_over_its_inputs():
    """h over y of another type would overwrite rows that are still to be read, h over
    x the residual."""
    bad = dict(x=FAKE, xs=1.0, y=2 * FAKE, yt=1, ys=1.0, pw=None, g=None, gt=0, gs=0, qw=None, T=3, d=64,
               eps=1e-5, h=2 * FAKE, ht=1, s=None)
    refuses("d2moe_block_norm", bad, [dict(yt=0), dict(ht=0), dict(h=FAKE), dict(h=FAKE, ht=0)])


def test_host_tensors_are_refused():
    x = torch.zeros((2, 8))
    with pytest.raises(ValueError):
        api.block_norm(x, x.clone())
    c = api.KVCache.empty(2, 4, 1, 8, device="cpu")
    with pytest.raises(ValueError):
        api.attn_decode(torch.zeros((1, 1, 8), dtype=torch.bfloat16), c,
                        torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
