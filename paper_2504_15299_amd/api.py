"""Python binding of libd2moe (ctypes).  Argument marshalling only: every step
of the MoE layer runs in the HIP library; torch provides device memory and the
current stream.  The names mirror the C ABI in include/d2moe.h.

The library is loaded from this package directory (or from the path in the
D2MOE_LIB environment variable); if it is missing the call fails loudly (run
``paper_2504_15299_amd.build.build()`` first).
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("D2MOE_LIB") or os.path.join(_HERE, "libd2moe.so")

D2MOE_F32, D2MOE_BF16 = 0, 1
OK, EINVAL, EUNSUPPORTED, EHIP, EWORKSPACE, ESCRATCH = 0, -1, -2, -3, -4, -5
NOALLOC_SCRATCH_BYTES = 32 << 20   # D2MOE_NOALLOC_SCRATCH_BYTES

_P = ctypes.c_void_p
_I = ctypes.c_int32


class _Mwq(ctypes.Structure):
    _fields_ = [("n_experts", _I), ("rows", _I), ("cols", _I), ("group", _I), ("b_min", _I),
                ("b_max", _I), ("planes", _P), ("scales", _P), ("zeros", _P)]


class _Unit(ctypes.Structure):
    _fields_ = [("expert", _I), ("bits", _I), ("load_from", _I), ("load_to", _I), ("count", _I)]


class _BudgetAction(ctypes.Structure):
    _fields_ = [("action", _I), ("layer", _I), ("expert", _I), ("level", _I)]


class _Linear(ctypes.Structure):
    _fields_ = [("rows", _I), ("cols", _I), ("group", _I), ("codes", _P), ("scales", _P),
                ("zeros", _P)]


class _KVCache(ctypes.Structure):
    _fields_ = [("n_pages", _I), ("page_size", _I), ("n_heads", _I), ("head_dim", _I),
                ("dtype", _I), ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64), ("k", _P), ("v", _P)]


class _Routing(ctypes.Structure):
    _fields_ = [("logits", _P), ("topk_idx", _P), ("topk_w", _P), ("topk_bits", _P),
                ("hist", _P), ("offsets", _P), ("perm", _P), ("slot_of", _P),
                ("expert_maxbit", _P), ("flags", _P)]


_lib = None


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"HIP library not built: {LIB_PATH} is missing "
                               "(call paper_2504_15299_amd.build.build())")
        L = ctypes.CDLL(LIB_PATH)
        sz = ctypes.POINTER(ctypes.c_size_t)
        L.d2moe_status_string.argtypes = [_I]
        L.d2moe_status_string.restype = ctypes.c_char_p
        L.d2moe_mwq_size.argtypes = [_I, _I, _I, _I, _I, _I, sz, sz, sz]
        L.d2moe_pack_mwq.argtypes = [_P, _I, ctypes.POINTER(_Mwq), _P]
        L.d2moe_debug_unpack.argtypes = [ctypes.POINTER(_Mwq), _I, _I, _P, _P, _P]
        L.d2moe_mwq_calib_factor_workspace.argtypes = [_I, sz]
        L.d2moe_mwq_calib_factor.argtypes = [_P, _I, _I, ctypes.c_double, _P, _P, _P,
                                             ctypes.c_size_t, _P]
        L.d2moe_pack_mwq_calibrated_workspace.argtypes = [_I, _I, _I, sz]
        L.d2moe_pack_mwq_calibrated.argtypes = [_P, _I, _P, _I, ctypes.POINTER(_Mwq), _P,
                                                ctypes.c_size_t, _P]
        L.d2moe_route.argtypes = [_P, _I, _I, _I, _P, _P, _I, _I, _P, _P, _I, _I, _I,
                                  ctypes.POINTER(_Routing), _P]
        L.d2moe_route_learned.argtypes = [_P, _I, _I, _I, _P, _P, _I, _I, _P, _P, _I, _I, _P,
                                          ctypes.POINTER(_Routing), _P]
        L.d2moe_route_scored.argtypes = [_P, _I, _I, _I, _P, _P, _I, _I, _I, _P, _I, _I, _I,
                                         ctypes.c_float, _P, _P, _I, _I, _I,
                                         ctypes.POINTER(_Routing), _P]
        L.d2moe_moe_forward_workspace.argtypes = [_I, _I, _I, _I, _I, _I, sz]
        L.d2moe_moe_forward.argtypes = [_P, _I, _I, _I, _I, _I, _I, ctypes.POINTER(_Mwq),
                                        ctypes.POINTER(_Mwq), ctypes.POINTER(_Routing),
                                        ctypes.POINTER(_Mwq), ctypes.POINTER(_Mwq), _I, _I, _P,
                                        _P, ctypes.c_size_t, _P]
        L.d2moe_moe_forward_profiled.argtypes = L.d2moe_moe_forward.argtypes + [_P]
        L.d2moe_moe_forward_noalloc.argtypes = [_P, _I, _I, _I, _I, _I, _I,
                                                ctypes.POINTER(_Mwq), ctypes.POINTER(_Mwq),
                                                ctypes.POINTER(_Routing), ctypes.POINTER(_Mwq),
                                                ctypes.POINTER(_Mwq), _I, _I, _P, _P]
        L.d2moe_stream_read.argtypes = [_P, ctypes.c_size_t, _P, _I, _P]
        L.d2moe_hebf_order.argtypes = [_P, _I, _I, _I, _P, _P, _P]
        L.d2moe_budget_plan.argtypes = [_P, _I, _I, _P, _I, ctypes.c_int64, _P, _P, _I, _P]
        L.d2moe_moe_forward_streamed.argtypes = [
            _P, _I, _I, _I, _I, _I, _I, ctypes.POINTER(_Mwq), ctypes.POINTER(_Mwq),
            ctypes.POINTER(_Mwq), ctypes.POINTER(_Mwq), _P, ctypes.POINTER(_Routing), _P, _P, _I,
            _P, _P, ctypes.c_size_t, _P, _P, _P]
        L.d2moe_residual_rmsnorm.argtypes = [_P, _P, _I, _I, _I, ctypes.c_float, _P, _I, _P]
        i64, f32, size = ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        lin, kvc = ctypes.POINTER(_Linear), ctypes.POINTER(_KVCache)
        L.d2moe_linear_size.argtypes = [_I, _I, _I, sz, sz, sz]
        L.d2moe_linear_pack.argtypes = [_P, _I, lin, _P]
        L.d2moe_linear_pack_codes.argtypes = [_P, _P, _P, lin, _P]
        L.d2moe_linear_forward.argtypes = [_P, _I, _I, lin, _P, _P, _I, _P]
        L.d2moe_kv_append.argtypes = [_P, i64, _I, _P, _P, i64, _I, _I, kvc, _P, _I, _I, _P, _P,
                                      _P, _P, _I, _P, _P]
        L.d2moe_kv_append_norm.argtypes = [_P, i64, _I, _P, _P, i64, _I, _I, kvc, _P, _I, _I, _P,
                                           _P, _P, _P, f32, _P, _P, _I, _I, _I, _P, _P]
        L.d2moe_attn_decode_workspace.argtypes = [_I, _I, _I, _I, _I, sz]
        L.d2moe_attn_decode.argtypes = [_P, i64, _I, _I, kvc, _P, _I, _P, _I, _I, f32, _P, _P,
                                        size, _P]
        L.d2moe_attn_prefix_workspace.argtypes = [_I, _I, _I, _I, _I, _I, sz]
        L.d2moe_attn_prefix.argtypes = [_P, i64, _I, _I, kvc, _P, _I, _P, _P, _I, _P, _I, _I, f32,
                                        _P, _P, size, _P]
        L.d2moe_block_norm.argtypes = [_P, f32, _P, _I, f32, _P, _P, _I, i64, _P, _I, _I, f32, _P,
                                       _I, _P]
        L.d2moe_sample.argtypes = [_P, _I, i64, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P]
        for name in ("d2moe_linear_size", "d2moe_linear_pack", "d2moe_linear_pack_codes",
                     "d2moe_linear_forward", "d2moe_kv_append", "d2moe_kv_append_norm",
                     "d2moe_attn_decode_workspace", "d2moe_attn_decode",
                     "d2moe_attn_prefix_workspace", "d2moe_attn_prefix", "d2moe_block_norm",
                     "d2moe_sample",
                     "d2moe_mwq_size", "d2moe_pack_mwq", "d2moe_debug_unpack", "d2moe_route",
                     "d2moe_mwq_calib_factor_workspace", "d2moe_mwq_calib_factor",
                     "d2moe_pack_mwq_calibrated_workspace", "d2moe_pack_mwq_calibrated",
                     "d2moe_route_learned", "d2moe_route_scored",
                     "d2moe_moe_forward_workspace", "d2moe_moe_forward",
                     "d2moe_moe_forward_profiled", "d2moe_moe_forward_noalloc",
                     "d2moe_residual_rmsnorm", "d2moe_stream_read", "d2moe_hebf_order",
                     "d2moe_budget_plan", "d2moe_moe_forward_streamed"):
            getattr(L, name).restype = _I
        _lib = L
    return _lib


class D2MoEError(RuntimeError):
    def __init__(self, fn, status):
        super().__init__(f"{fn} failed: {status} ({status_string(status)})")
        self.status = status


def status_string(s: int) -> str:
    return lib().d2moe_status_string(int(s)).decode()


def _check(fn, rc):
    if rc != OK:
        raise D2MoEError(fn, rc)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return D2MOE_F32
    if t.dtype == torch.bfloat16:
        return D2MOE_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


# ---- packed weights ---------------------------------------------------------

def mwq_size(n_experts, rows, cols, group, b_min=2, b_max=8):
    a, b, c = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check("d2moe_mwq_size", lib().d2moe_mwq_size(n_experts, rows, cols, group, b_min, b_max,
                                                  ctypes.byref(a), ctypes.byref(b),
                                                  ctypes.byref(c)))
    return a.value, b.value, c.value


@dataclass
class MWQ:
    """Device buffers of packed MWQ weights (canonical tiled bit-plane layout)."""
    n_experts: int
    rows: int
    cols: int
    group: int
    b_min: int
    b_max: int
    planes: torch.Tensor   # uint32 words, stored as int32
    scales: torch.Tensor   # binary16 bit patterns, stored as int16
    zeros: torch.Tensor    # uint8

    @staticmethod
    def empty(n_experts, rows, cols, group, b_min=2, b_max=8, device="cuda"):
        pb, sb, zb = mwq_size(n_experts, rows, cols, group, b_min, b_max)
        return MWQ(n_experts, rows, cols, group, b_min, b_max,
                   torch.empty(pb // 4, dtype=torch.int32, device=device),
                   torch.empty(sb // 2, dtype=torch.int16, device=device),
                   torch.empty(zb, dtype=torch.uint8, device=device))

    def _c(self) -> _Mwq:
        return _Mwq(self.n_experts, self.rows, self.cols, self.group, self.b_min, self.b_max,
                    self.planes.data_ptr(), self.scales.data_ptr(), self.zeros.data_ptr())

    def nbytes(self):
        return self.planes.numel() * 4 + self.scales.numel() * 2 + self.zeros.numel()

    def expert(self, e: int) -> "MWQ":
        """View of expert e as a one-expert MWQ (experts are outermost)."""
        np_, ns, nz = (t.numel() // self.n_experts for t in (self.planes, self.scales, self.zeros))
        return MWQ(1, self.rows, self.cols, self.group, self.b_min, self.b_max,
                   self.planes.narrow(0, e * np_, np_), self.scales.narrow(0, e * ns, ns),
                   self.zeros.narrow(0, e * nz, nz))


def pack_mwq(W: torch.Tensor, out: MWQ, stream=None) -> MWQ:
    """Quantize + pack W [n_experts][rows][cols] (fp32, device) into ``out``."""
    assert W.is_cuda and W.is_contiguous()
    c = out._c()
    _check("d2moe_pack_mwq", lib().d2moe_pack_mwq(_ptr(W), _dtype_code(W), ctypes.byref(c),
                                                  _stream(stream)))
    return out


def mwq_calib_factor(X: torch.Tensor, lam: float, stream=None):
    """``d2moe_mwq_calib_factor``: X [tokens][h] float (device) ->
    (U [h][h] float, info int32 tensor of one element)."""
    T, h = X.shape
    n = ctypes.c_size_t()
    _check("d2moe_mwq_calib_factor_workspace",
           lib().d2moe_mwq_calib_factor_workspace(h, ctypes.byref(n)))
    ws = torch.empty(n.value, dtype=torch.uint8, device=X.device)
    U = torch.empty((h, h), dtype=torch.float32, device=X.device)
    info = torch.empty(1, dtype=torch.int32, device=X.device)
    _check("d2moe_mwq_calib_factor",
           lib().d2moe_mwq_calib_factor(_ptr(X), T, h, float(lam), _ptr(U), _ptr(info), _ptr(ws),
                                        n.value, _stream(stream)))
    return U, info


def pack_mwq_calibrated(W: torch.Tensor, U: torch.Tensor, gamma: int, out: MWQ,
                        stream=None) -> MWQ:
    """``d2moe_pack_mwq_calibrated``: W [n_experts][rows][cols] float and the
    factor U [cols][cols] float, both on the device."""
    assert W.is_cuda and W.is_contiguous() and U.is_contiguous()
    n = ctypes.c_size_t()
    _check("d2moe_pack_mwq_calibrated_workspace",
           lib().d2moe_pack_mwq_calibrated_workspace(out.rows, out.cols, gamma, ctypes.byref(n)))
    ws = torch.empty(n.value, dtype=torch.uint8, device=W.device)
    c = out._c()
    _check("d2moe_pack_mwq_calibrated",
           lib().d2moe_pack_mwq_calibrated(_ptr(W), _dtype_code(W), _ptr(U), gamma,
                                           ctypes.byref(c), _ptr(ws), n.value, _stream(stream)))
    return out


def debug_unpack(w: MWQ, expert: int, bits: int, stream=None):
    """(q1 [rows][cols] uint8, signs [bits-b_min][rows][cols] int8 or None)."""
    dev = w.planes.device
    q1 = torch.empty((w.rows, w.cols), dtype=torch.uint8, device=dev)
    signs = (torch.empty((bits - w.b_min, w.rows, w.cols), dtype=torch.int8, device=dev)
             if bits > w.b_min else None)
    c = w._c()
    _check("d2moe_debug_unpack", lib().d2moe_debug_unpack(ctypes.byref(c), expert, bits,
                                                          _ptr(q1), _ptr(signs),
                                                          _stream(stream)))
    return q1, signs


# ---- routing ----------------------------------------------------------------

@dataclass
class Routing:
    logits: torch.Tensor
    topk_idx: torch.Tensor
    topk_w: torch.Tensor
    topk_bits: torch.Tensor
    hist: torch.Tensor
    offsets: torch.Tensor
    perm: torch.Tensor
    slot_of: torch.Tensor
    expert_maxbit: torch.Tensor
    flags: torch.Tensor

    @staticmethod
    def empty(T, E, k, b_min=2, b_max=8, device="cuda"):
        L = b_max - b_min + 1
        i32, dev = torch.int32, device
        return Routing(torch.empty((T, E), dtype=torch.float32, device=dev),
                       torch.empty((T, k), dtype=i32, device=dev),
                       torch.empty((T, k), dtype=torch.float32, device=dev),
                       torch.empty((T, k), dtype=torch.uint8, device=dev),
                       torch.empty((E, L), dtype=i32, device=dev),
                       torch.empty(E * L + 1, dtype=i32, device=dev),
                       torch.empty(T * k, dtype=i32, device=dev),
                       torch.empty(T * k, dtype=i32, device=dev),
                       torch.empty(E, dtype=torch.uint8, device=dev),
                       torch.empty(1, dtype=i32, device=dev))

    def _c(self) -> _Routing:
        return _Routing(*[getattr(self, f).data_ptr() for f, _ in _Routing._fields_])


def route(x: torch.Tensor, Wg: torch.Tensor, bias, k: int, token_req, bit_table: torch.Tensor,
          b_min=2, b_max=8, out: Routing | None = None, stream=None) -> Routing:
    T, d = x.shape
    E = Wg.shape[0]
    if out is None:
        out = Routing.empty(T, E, k, b_min, b_max, device=x.device)
    c = out._c()
    _check("d2moe_route", lib().d2moe_route(_ptr(x), _dtype_code(x), T, d, _ptr(Wg), _ptr(bias),
                                            E, k, _ptr(token_req), _ptr(bit_table),
                                            bit_table.shape[0], b_min, b_max, ctypes.byref(c),
                                            _stream(stream)))
    return out


def route_learned(x: torch.Tensor, Wg: torch.Tensor, bias, k: int, Wr: torch.Tensor, br,
                  b_min=2, b_max=8, out: Routing | None = None,
                  bit_logits: torch.Tensor | None = None, stream=None):
    """Dual routing with learned bit-width routers (``d2moe_route_learned``):
    Wr [E][L][d] float, br [E][L] float or None, L = b_max - b_min + 1.
    Returns (routing, bit_logits [T][E][L])."""
    T, d = x.shape
    E = Wg.shape[0]
    L_ = b_max - b_min + 1
    if tuple(Wr.shape) != (E, L_, d):
        raise ValueError(f"Wr must be [E][L][d] = {(E, L_, d)}, got {tuple(Wr.shape)}")
    if out is None:
        out = Routing.empty(T, E, k, b_min, b_max, device=x.device)
    if bit_logits is None:
        bit_logits = torch.empty((T, E, L_), dtype=torch.float32, device=x.device)
    c = out._c()
    _check("d2moe_route_learned",
           lib().d2moe_route_learned(_ptr(x), _dtype_code(x), T, d, _ptr(Wg), _ptr(bias), E, k,
                                     _ptr(Wr), _ptr(br), b_min, b_max, _ptr(bit_logits),
                                     ctypes.byref(c), _stream(stream)))
    return out, bit_logits


_SCORING = {"softmax": 0, "sigmoid": 1}


def route_scored(logits, k: int, token_req, bit_table: torch.Tensor, scoring: str = "softmax",
                 select_bias: torch.Tensor | None = None, groups: int = 1, top_groups: int = 1,
                 renorm: bool = True, scale: float = 1.0, x: torch.Tensor | None = None,
                 Wg: torch.Tensor | None = None, bias=None, b_min=2, b_max=8,
                 out: Routing | None = None, stream=None) -> Routing:
    """``d2moe_route_scored``: experts by scores of ``logits`` [T][E] float32, or, with
    ``logits`` None, of x [T][d] Wg [E][d]^T + bias.  ``scoring`` is "softmax" or
    "sigmoid", select_bias [E] float32 or None, token_req [T] int32 or None, bit_table
    [R][E] uint8.  The routing's ``logits`` are the ones given (those of ``out`` are left
    alone), or the ones computed."""
    if scoring not in _SCORING:
        raise ValueError(f'scoring must be "softmax" or "sigmoid", got {scoring!r}')
    f32, dev = torch.float32, bit_table.get_device()
    px, pw, pb, code, d = None, None, None, D2MOE_F32, 0
    if logits is not None:
        if x is not None or Wg is not None or bias is not None:
            raise ValueError("logits, or x and Wg with their bias, not both")
        T, E = logits.shape
        pl = _arg(logits, (T, E), f32, dev, "logits")
    else:
        if x is None or Wg is None:
            raise ValueError("logits, or x and Wg, must be given")
        (T, d), E = x.shape, Wg.shape[0]
        if x.dtype not in _CODES:
            raise TypeError(f"unsupported dtype {x.dtype}")
        px, code = _arg(x, (T, d), x.dtype, dev, "x"), _CODES[x.dtype]
        pw = _arg(Wg, (E, d), f32, dev, "Wg")
        pb = None if bias is None else _arg(bias, (E,), f32, dev, "bias")
    R, L, slots = bit_table.shape[0], b_max - b_min + 1, T * k
    i32, u8 = torch.int32, torch.uint8
    if out is None:
        if b_min > b_max or k < 1:
            raise ValueError("b_min <= b_max and k >= 1 are needed")
        shapes = [((T, k), i32), ((T, k), f32), ((T, k), u8), ((E, L), i32),
                  ((E * L + 1,), i32), ((slots,), i32), ((slots,), i32), ((E,), u8), ((1,), i32)]
        out = Routing(_new(bit_table, (T, E), f32, stream) if logits is None else logits,
                      *[_new(bit_table, s, t, stream) for s, t in shapes])
    if logits is None:
        pl = _arg(out.logits, (T, E), f32, dev, "logits")
    elif out.logits is not logits:
        out = Routing(logits, out.topk_idx, out.topk_w, out.topk_bits, out.hist, out.offsets,
                      out.perm, out.slot_of, out.expert_maxbit, out.flags)
    c = _Routing(pl, _arg(out.topk_idx, (T, k), i32, dev, "topk_idx"),
                 _arg(out.topk_w, (T, k), f32, dev, "topk_w"),
                 _arg(out.topk_bits, (T, k), u8, dev, "topk_bits"),
                 _arg(out.hist, (E, L), i32, dev, "hist"),
                 _arg(out.offsets, (E * L + 1,), i32, dev, "offsets"),
                 _arg(out.perm, (slots,), i32, dev, "perm"),
                 _arg(out.slot_of, (slots,), i32, dev, "slot_of"),
                 _arg(out.expert_maxbit, (E,), u8, dev, "expert_maxbit"),
                 _arg(out.flags, (1,), i32, dev, "flags"))
    _run("d2moe_route_scored", dev, stream, px, code, T, d, pw, pb, E, k, _SCORING[scoring],
         None if select_bias is None else _arg(select_bias, (E,), f32, dev, "select_bias"), groups,
         top_groups, int(renorm), scale,
         None if token_req is None else _arg(token_req, (T,), i32, dev, "token_req"),
         _arg(bit_table, (R, E), u8, dev, "bit_table"), R, b_min, b_max, ctypes.byref(c))
    return out


# ---- forward ----------------------------------------------------------------

def moe_forward_workspace(T, d, d_ff, E, k, shared_d_ff=0) -> int:
    n = ctypes.c_size_t()
    _check("d2moe_moe_forward_workspace",
           lib().d2moe_moe_forward_workspace(T, d, d_ff, E, k, shared_d_ff, ctypes.byref(n)))
    return n.value


def moe_forward(x: torch.Tensor, w13: MWQ, w2: MWQ, r: Routing, k: int, shared=None,
                out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                stream=None, events=None) -> torch.Tensor:
    """``shared`` is None or (shared_w13: MWQ, shared_w2: MWQ, shared_bits).
    ``events``: optional 4 torch.cuda.Event (created with enable_timing) that
    are recorded around the W1/W3 and the W2 expert kernels."""
    T, d = x.shape
    E = w13.n_experts
    d_ff = w2.cols
    sw13 = sw2 = None
    sbits = sff = 0
    if shared is not None:
        sw13, sw2, sbits = shared
        sff = sw2.cols
    if out is None:
        out = torch.empty_like(x)
    need = moe_forward_workspace(T, d, d_ff, E, k, sff)
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=x.device)
    c13, c2, cr = w13._c(), w2._c(), r._c()
    cs13 = ctypes.byref(sw13._c()) if sw13 is not None else None
    cs2 = ctypes.byref(sw2._c()) if sw2 is not None else None
    args = (_ptr(x), _dtype_code(x), T, d, d_ff, E, k, ctypes.byref(c13), ctypes.byref(c2),
            ctypes.byref(cr), cs13, cs2, sbits, sff, _ptr(out), _ptr(workspace),
            workspace.numel(), _stream(stream))
    if events is None:
        _check("d2moe_moe_forward", lib().d2moe_moe_forward(*args))
    else:
        arr = (ctypes.c_void_p * 4)(*[ev.cuda_event for ev in events])
        _check("d2moe_moe_forward_profiled", lib().d2moe_moe_forward_profiled(*args, arr))
    return out


def moe_forward_noalloc(x: torch.Tensor, w13: MWQ, w2: MWQ, r: Routing, k: int, shared=None,
                        out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """``d2moe_moe_forward_noalloc``: the forward with the library's fixed
    per-GPU scratch array as workspace (nothing is allocated by the call;
    ``out`` is allocated here only when not given)."""
    T, d = x.shape
    sw13 = sw2 = None
    sbits = sff = 0
    if shared is not None:
        sw13, sw2, sbits = shared
        sff = sw2.cols
    if out is None:
        out = torch.empty_like(x)
    c13, c2, cr = w13._c(), w2._c(), r._c()
    cs13 = ctypes.byref(sw13._c()) if sw13 is not None else None
    cs2 = ctypes.byref(sw2._c()) if sw2 is not None else None
    _check("d2moe_moe_forward_noalloc",
           lib().d2moe_moe_forward_noalloc(_ptr(x), _dtype_code(x), T, d, w2.cols,
                                           w13.n_experts, k, ctypes.byref(c13),
                                           ctypes.byref(c2), ctypes.byref(cr), cs13, cs2, sbits,
                                           sff, _ptr(out), _stream(stream)))
    return out


def residual_rmsnorm(x: torch.Tensor, y: torch.Tensor | None, eps: float = 1e-5,
                     h: torch.Tensor | None = None, h_dtype=torch.bfloat16,
                     stream=None) -> torch.Tensor:
    """x [T][d] float32 (updated in place: x += y); returns h = x / rms(x)
    (h_dtype).  y is None or [T][d] bfloat16 / float32."""
    T, d = x.shape
    if x.dtype != torch.float32 or not x.is_contiguous():
        raise ValueError("x must be a contiguous float32 tensor")
    if y is not None and (y.shape != x.shape or not y.is_contiguous()):
        raise ValueError("y must match x")
    if h is None:
        h = torch.empty((T, d), dtype=h_dtype, device=x.device)
    _check("d2moe_residual_rmsnorm",
           lib().d2moe_residual_rmsnorm(_ptr(x), _ptr(y) if y is not None else None,
                                        _dtype_code(y) if y is not None else D2MOE_F32, T, d,
                                        float(eps), _ptr(h), _dtype_code(h), _stream(stream)))
    return h


# ---- the rest of a decoder block: 4-bit linear layers, paged cache, norms ------

# Tensors' devices are compared by their index (-1 for the CPU), which costs half
# of what comparing device objects does.

def _arg(t, shape, dtype, dev, what):
    """Pointer of a contiguous tensor of this shape and type."""
    if t.dtype != dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor of shape {shape} on GPU {dev}")
    return t.data_ptr()


def _new(like, shape, dtype, stream):
    """A contiguous tensor for a call on ``stream`` (None: the current one): memory that
    the current stream has freed may still be in use there, so it is taken from
    ``stream``'s own, and kept until the current one is past its uses."""
    if stream is None:
        if like.shape == shape:  # the same, sooner
            return torch.empty_like(like, dtype=dtype, memory_format=torch.contiguous_format)
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(stream):
        t = like.new_empty(shape, dtype=dtype)
    t.record_stream(torch.cuda.current_stream(like.device))
    return t


_CODES = {torch.float32: D2MOE_F32, torch.bfloat16: D2MOE_BF16}
_entry = {}     # entry points by name


def _run(name, dev, stream, *args):
    """The entry point on ``stream`` (None: the current one of the tensors'
    device, number ``dev``), with that device current."""
    fn = _entry.get(name)
    if fn is None:
        fn = _entry[name] = getattr(lib(), name)
    if dev < 0:
        raise ValueError(f"{name}: tensors must be on a GPU")
    raw = torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream
    if dev == torch._C._cuda_getDevice():
        rc = fn(*args, raw)
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, raw)
    if rc != OK:
        raise D2MoEError(name, rc)


def linear_size(rows, cols, group=128):
    a, b, c = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check("d2moe_linear_size", lib().d2moe_linear_size(rows, cols, group, ctypes.byref(a),
                                                        ctypes.byref(b), ctypes.byref(c)))
    return a.value, b.value, c.value


class Linear:
    """Device buffers of a linear layer's 4-bit weights (``d2moe_linear``)."""

    def __init__(self, rows, cols, group, codes, scales, zeros):
        sizes = linear_size(rows, cols, group)
        for t, n in zip((codes, scales, zeros), sizes):
            if t.numel() * t.element_size() != n or not t.is_contiguous() or \
                    t.device != codes.device:
                raise ValueError(f"buffers of {sizes} bytes on one device are needed")
        self.rows, self.cols, self.group = rows, cols, group
        self.codes, self.scales, self.zeros, self.index = codes, scales, zeros, codes.get_device()
        self._c = _Linear(rows, cols, group, codes.data_ptr(), scales.data_ptr(),
                          zeros.data_ptr())
        self._ref = ctypes.byref(self._c)

    @staticmethod
    def empty(rows, cols, group=128, device="cuda"):
        cb, sb, zb = linear_size(rows, cols, group)
        return Linear(rows, cols, group, torch.empty(cb // 4, dtype=torch.int32, device=device),
                      torch.empty(sb // 2, dtype=torch.int16, device=device),
                      torch.empty(zb, dtype=torch.uint8, device=device))

    def nbytes(self):
        return self.codes.numel() * 4 + self.scales.numel() * 2 + self.zeros.numel()


def linear_pack(W: torch.Tensor, out: Linear, stream=None) -> Linear:
    """``d2moe_linear_pack``: quantize + pack W [rows][cols] (fp32, device)."""
    dev = out.index
    _run("d2moe_linear_pack", dev, stream,
         _arg(W, (out.rows, out.cols), torch.float32, dev, "W"), D2MOE_F32, out._ref)
    return out


def linear_pack_codes(codes: torch.Tensor, scales: torch.Tensor, zeros, out: Linear,
                      stream=None) -> Linear:
    """``d2moe_linear_pack_codes``: codes [rows][cols] uint8 (0..15), scales
    [rows][cols/group] float16, zeros [rows][cols/group] uint8 or None (8)."""
    dev, g = out.index, (out.rows, out.cols // out.group)
    _run("d2moe_linear_pack_codes", dev, stream,
         _arg(codes, (out.rows, out.cols), torch.uint8, dev, "codes"),
         _arg(scales, g, torch.float16, dev, "scales"),
         None if zeros is None else _arg(zeros, g, torch.uint8, dev, "zeros"), out._ref)
    return out


def linear_forward(x: torch.Tensor, w: Linear, bias: torch.Tensor | None = None,
                   y: torch.Tensor | None = None, y_dtype=None, stream=None) -> torch.Tensor:
    """``d2moe_linear_forward``: x [T][cols] -> [T][rows] (y_dtype, x's type
    when not given); bias [rows] float32 or None."""
    T, dev, dtype = x.shape[0], w.index, x.dtype
    px = _arg(x, (T, w.cols), dtype, dev, "x")
    if y is None:
        y = _new(x, (T, w.rows), y_dtype or dtype, stream)
        py = y.data_ptr()
    else:
        py = _arg(y, (T, w.rows), y.dtype, dev, "y")
    if dtype not in _CODES or y.dtype not in _CODES:
        raise TypeError(f"unsupported dtypes {dtype}, {y.dtype}")
    _run("d2moe_linear_forward", dev, stream, px, _CODES[dtype], T, w._ref,
         None if bias is None else _arg(bias, (w.rows,), torch.float32, dev, "bias"), py,
         _CODES[y.dtype])
    return y


class KVCache:
    """A paged key-value cache over two tensors [page][token][head][dim] of
    one shape and one set of strides (``d2moe_kv_cache``); views of another
    order or of a joint buffer will do."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or \
                k.dtype != v.dtype or k.device != v.device or k.stride(3) != 1:
            raise ValueError("k and v must be [page][token][head][dim] tensors of one type, shape "
                             "and stride, dim contiguous")
        self.k, self.v = k, v
        self.n_pages, self.page_size, self.n_heads, self.head_dim = k.shape
        self.index = k.get_device()
        self._c = _KVCache(*k.shape, _dtype_code(k), *k.stride()[:3], k.data_ptr(), v.data_ptr())
        self._ref = ctypes.byref(self._c)

    @staticmethod
    def empty(n_pages, page_size, n_heads, head_dim, dtype=torch.bfloat16, device="cuda"):
        shape = (n_pages, page_size, n_heads, head_dim)
        return KVCache(torch.empty(shape, dtype=dtype, device=device),
                       torch.empty(shape, dtype=dtype, device=device))


def _rows(t, shape, dtype, dev, what):
    """Pointer and token stride of a [token][head][dim] tensor whose heads are
    packed."""
    if t.shape != shape or t.dtype != dtype or t.get_device() != dev:
        raise ValueError(f"{what} must be a {dtype} tensor of shape {shape} on GPU {dev}")
    n, heads, dim = shape
    row, head, one = t.stride()
    if one != 1 or (heads > 1 and head != dim):
        raise ValueError(f"{what} must have its heads packed")
    return t.data_ptr(), row if n > 1 else heads * dim


def _append_args(q, k, v, cache, q_out, stream):
    """(q, its stride and heads, k, v, their stride, type code, tokens), q_out and its
    pointer, of a call that appends."""
    dev, dtype, N, D = cache.index, k.dtype, k.shape[0], cache.head_dim
    shape = (N, cache.n_heads, D)
    pk, ks = _rows(k, shape, dtype, dev, "k")
    pv, vs = _rows(v, shape, dtype, dev, "v")
    if vs != ks:
        raise ValueError("k and v must have the same token stride")
    if dtype not in _CODES:
        raise TypeError(f"unsupported dtype {dtype}")
    pq, qs, heads, po = None, 0, 0, None
    if q is not None:
        heads = q.shape[1]
        pq, qs = _rows(q, (N, heads, D), dtype, dev, "q")
        if q_out is None:
            q_out = _new(q, (N, heads, D), cache.k.dtype, stream)
            po = q_out.data_ptr()
        else:
            po = _arg(q_out, (N, heads, D), cache.k.dtype, dev, "q_out")
    return (pq, qs, heads, pk, pv, ks, _CODES[dtype], N), q_out, po


def _place_args(N, cache, block_table, positions, token_seq):
    """The table with its sizes, positions and sequences of a call that appends."""
    n_seqs, pages = block_table.shape
    dev, i32 = cache.index, torch.int32
    return (_arg(block_table, (n_seqs, pages), i32, dev, "block_table"), n_seqs, pages,
            _arg(positions, (N,), i32, dev, "positions"),
            None if token_seq is None else _arg(token_seq, (N,), i32, dev, "token_seq"))


def _turn_args(cos, sin, half, dev):
    """cos, sin and their rows; half the rotated values: columns, when given."""
    if cos is None and sin is None:
        return None, None, 0
    n_rot = 0 if cos is None else cos.shape[0]
    if cos is not None and n_rot == 0:  # (an empty tensor has no address, which is no rotation)
        raise ValueError("cos and sin must have a row")
    return (None if cos is None else _arg(cos, (n_rot, half), torch.float32, dev, "cos"),
            None if sin is None else _arg(sin, (n_rot, half), torch.float32, dev, "sin"), n_rot)


def kv_append(q, k: torch.Tensor, v: torch.Tensor, cache: KVCache, block_table: torch.Tensor,
              positions: torch.Tensor, token_seq: torch.Tensor | None = None, cos=None, sin=None,
              q_out: torch.Tensor | None = None, stream=None):
    """``d2moe_kv_append``: q [N][q_heads][dim] or None, k and v
    [N][heads][dim] (views with packed heads will do), block_table
    [n_seqs][max_pages], positions [N] and token_seq [N] int32, cos and sin
    [n_rot][dim/2] float32 (n_rot >= 1).  Returns q_out [N][q_heads][dim] of the cache's
    type (None without q)."""
    rows, q_out, po = _append_args(q, k, v, cache, q_out, stream)
    _run("d2moe_kv_append", cache.index, stream, *rows, cache._ref,
         *_place_args(rows[-1], cache, block_table, positions, token_seq),
         *_turn_args(cos, sin, cache.head_dim // 2, cache.index), po)
    return q_out


def kv_append_norm(q, k: torch.Tensor, v: torch.Tensor, cache: KVCache, block_table: torch.Tensor,
                   positions: torch.Tensor, token_seq: torch.Tensor | None = None, q_weight=None,
                   k_weight=None, eps: float = 1e-6, cos=None, sin=None, interleaved: bool = False,
                   q_out: torch.Tensor | None = None, stream=None):
    """``d2moe_kv_append_norm``: kv_append with RMS norms of the heads of q and k
    before the rotation, q_weight and k_weight [dim] float32 (None: no norm of
    these).  cos and sin [n_rot][half] float32 rotate the first 2 * half values of a
    head (half even, at most dim/2), value i with i + half, or neighbours when
    ``interleaved``."""
    rows, q_out, po = _append_args(q, k, v, cache, q_out, stream)
    dev, D = cache.index, cache.head_dim
    half = 0 if cos is None else cos.shape[1]
    f32 = torch.float32
    _run("d2moe_kv_append_norm", dev, stream, *rows, cache._ref,
         *_place_args(rows[-1], cache, block_table, positions, token_seq),
         None if q_weight is None else _arg(q_weight, (D,), f32, dev, "q_weight"),
         None if k_weight is None else _arg(k_weight, (D,), f32, dev, "k_weight"), eps,
         *_turn_args(cos, sin, half, dev), 2 * half, int(interleaved), po)
    return q_out


def attn_decode_workspace(B: int, q_heads: int, cache: KVCache, max_len: int) -> int:
    n = ctypes.c_size_t()
    _check("d2moe_attn_decode_workspace",
           lib().d2moe_attn_decode_workspace(B, q_heads, cache.n_heads, cache.head_dim, max_len,
                                             ctypes.byref(n)))
    return n.value


def attn_decode(q: torch.Tensor, cache: KVCache, block_table: torch.Tensor, lengths: torch.Tensor,
                scale: float | None = None, window: int = 0, max_len: int | None = None,
                out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                stream=None) -> torch.Tensor:
    """``d2moe_attn_decode``: q [B][q_heads][dim] of the cache's type,
    block_table [B][max_pages] and lengths [B] int32 (device) -> out
    [B][q_heads][dim].  ``scale`` is 1 / sqrt(dim) when not given, ``max_len``
    the length that fills a row of the table."""
    dev, dtype, D = cache.index, cache.k.dtype, cache.head_dim
    B, heads = q.shape[:2]
    shape = (B, heads, D)
    pq, qs = _rows(q, shape, dtype, dev, "q")
    pages = block_table.shape[1]
    if max_len is None:
        max_len = min(pages * cache.page_size, 0x7fffffff)
    if out is None:
        out = _new(q, shape, dtype, stream)
        po = out.data_ptr()
    else:
        po = _arg(out, shape, dtype, dev, "out")
    if workspace is None:
        need = attn_decode_workspace(B, heads, cache, max_len)
        if need:
            workspace = _new(q, (need,), torch.uint8, stream)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on GPU {dev}")
    pw, nw = (None, 0) if workspace is None else (workspace.data_ptr(), workspace.nbytes)
    _run("d2moe_attn_decode", dev, stream, pq, qs, B, heads, cache._ref,
         _arg(block_table, (B, pages), torch.int32, dev, "block_table"), pages,
         _arg(lengths, (B,), torch.int32, dev, "lengths"), max_len, window,
         D ** -0.5 if scale is None else scale, po, pw, nw)
    return out


def attn_prefix_workspace(B: int, q_heads: int, cache: KVCache, max_prefix: int,
                          max_rest: int) -> int:
    n = ctypes.c_size_t()
    _check("d2moe_attn_prefix_workspace",
           lib().d2moe_attn_prefix_workspace(B, q_heads, cache.n_heads, cache.head_dim, max_prefix,
                                             max_rest, ctypes.byref(n)))
    return n.value


def attn_prefix(q: torch.Tensor, cache: KVCache, block_table: torch.Tensor, lengths: torch.Tensor,
                prefix_table: torch.Tensor, prefix_lens: torch.Tensor, scale: float | None = None,
                max_prefix: int | None = None, max_rest: int | None = None,
                out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                stream=None) -> torch.Tensor:
    """``d2moe_attn_prefix``: attn_decode where sequence b's first prefix_lens[b] tokens
    lie in the pages of prefix_table [prefix_pages], the others in those of its row of
    block_table [B][max_pages]; prefix_lens [B] int32.  ``max_prefix`` and ``max_rest``,
    the most tokens of either kind expected, are what the tables have room for when not
    given."""
    dev, dtype, D = cache.index, cache.k.dtype, cache.head_dim
    B, heads = q.shape[:2]
    shape, i32 = (B, heads, D), torch.int32
    pq, qs = _rows(q, shape, dtype, dev, "q")
    pages, head_pages = block_table.shape[1], prefix_table.shape[0]
    if max_prefix is None:
        max_prefix = min(head_pages * cache.page_size, 1 << 30)
    if max_rest is None:
        max_rest = min(pages * cache.page_size, 1 << 30)
    if out is None:
        out = _new(q, shape, dtype, stream)
        po = out.data_ptr()
    else:
        po = _arg(out, shape, dtype, dev, "out")
    if workspace is None:
        need = attn_prefix_workspace(B, heads, cache, max_prefix, max_rest)
        workspace = _new(q, (need,), torch.uint8, stream)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on GPU {dev}")
    _run("d2moe_attn_prefix", dev, stream, pq, qs, B, heads, cache._ref,
         _arg(block_table, (B, pages), i32, dev, "block_table"), pages,
         _arg(lengths, (B,), i32, dev, "lengths"),
         _arg(prefix_table, (head_pages,), i32, dev, "prefix_table"), head_pages,
         _arg(prefix_lens, (B,), i32, dev, "prefix_lens"), max_prefix, max_rest,
         D ** -0.5 if scale is None else scale, po, workspace.data_ptr(), workspace.nbytes)
    return out


def block_norm(x: torch.Tensor, y: torch.Tensor, eps: float = 1e-5, pre_weight=None,
               post_weight=None, gate=None, x_scale: float = 1.0, y_scale: float = 1.0,
               h: torch.Tensor | None = None, h_dtype=torch.bfloat16, stream=None):
    """``d2moe_block_norm``: x [T][d] float32, updated in place to
    x_scale * x + y_scale * gate * postnorm(y); returns h = prenorm(x) (h_dtype;
    None: only x is updated).  y [T][d]; gate [d] or [T][d] (rows may be
    strided); pre_weight, post_weight [d] float32 or None."""
    shape, dev, f32 = x.shape, x.get_device(), torch.float32
    T, d = shape
    px, py = _arg(x, shape, f32, dev, "x"), _arg(y, shape, y.dtype, dev, "y")
    pg, gs, gd = None, 0, D2MOE_F32
    if gate is not None:
        rows = gate.dim() == 2
        if gate.shape != (shape if rows else (d,)) or gate.get_device() != dev or \
                (d > 1 and gate.stride(-1) != 1):
            raise ValueError(f"gate must be [d] or [T][d] = {(T, d)} on GPU {dev}, rows contiguous")
        # one row alone has no stride
        pg, gs, gd = gate.data_ptr(), gate.stride(0) if rows and T > 1 else 0, _dtype_code(gate)
    ph, hd = None, D2MOE_F32
    if h is not None:
        ph, hd = _arg(h, shape, h.dtype, dev, "h"), _dtype_code(h)
    elif h_dtype is not None:
        h = _new(y, shape, h_dtype, stream)
        ph, hd = h.data_ptr(), _dtype_code(h)
    _run("d2moe_block_norm", dev, stream, px, x_scale, py, _dtype_code(y), y_scale,
         None if post_weight is None else _arg(post_weight, (d,), f32, dev, "post_weight"), pg, gd,
         gs, None if pre_weight is None else _arg(pre_weight, (d,), f32, dev, "pre_weight"), T, d,
         eps, ph, hd)
    return h


def sample(logits: torch.Tensor, u: torch.Tensor, temperature=None, top_k=None, top_p=None,
           min_p=None, tokens: torch.Tensor | None = None, probs: torch.Tensor | None = None,
           stream=None):
    """``d2moe_sample``: logits [B][V] float32 or bfloat16 (rows may be strided), u [B]
    float32 in [0, 1); temperature, top_p, min_p [B] float32 and top_k [B] int32, each
    or None.  Returns (tokens [B] int32, probs [B] float32)."""
    (B, V), dev, f32, i32 = logits.shape, logits.get_device(), torch.float32, torch.int32
    if logits.dtype not in _CODES:
        raise TypeError(f"unsupported dtype {logits.dtype}")
    if V > 1 and logits.stride(1) != 1:
        raise ValueError("logits must have contiguous rows")
    tokens = _new(u, (B,), i32, stream) if tokens is None else tokens
    probs = _new(u, (B,), f32, stream) if probs is None else probs

    def opt(t, dtype, what):
        return None if t is None else _arg(t, (B,), dtype, dev, what)

    _run("d2moe_sample", dev, stream, logits.data_ptr(), _CODES[logits.dtype],
         logits.stride(0) if B > 1 else V, B, V, _arg(u, (B,), f32, dev, "u"),
         opt(temperature, f32, "temperature"), opt(top_k, i32, "top_k"), opt(top_p, f32, "top_p"),
         opt(min_p, f32, "min_p"), _arg(tokens, (B,), i32, dev, "tokens"),
         _arg(probs, (B,), f32, dev, "probs"))
    return tokens, probs


def stream_read(buf: torch.Tensor, sink: torch.Tensor, stream=None) -> None:
    """``d2moe_stream_read``: read all of ``buf`` once (plain HBM read
    kernel, a measurement helper); ``sink`` is a device int32 tensor with one
    word per workgroup."""
    _check("d2moe_stream_read",
           lib().d2moe_stream_read(_ptr(buf), buf.numel() * buf.element_size(), _ptr(sink),
                                   sink.numel(), _stream(stream)))


# ---- streamed weights: HEBF order, memory budget, streamed forward -------------

def hebf_order(hist, b_min=2, b_max=8, resident=None):
    """``d2moe_hebf_order`` on host arrays: hist [E][L] int -> list of units
    (expert, bits, load_from, load_to, count) in I/O order."""
    import numpy as np
    h = np.ascontiguousarray(hist, dtype=np.int32)
    E = h.shape[0]
    res = None if resident is None else np.ascontiguousarray(resident, dtype=np.uint8)
    units = (_Unit * max(1, h.size))()
    n = ctypes.c_int32()
    _check("d2moe_hebf_order",
           lib().d2moe_hebf_order(h.ctypes.data_as(_P), E, b_min, b_max,
                                  None if res is None else res.ctypes.data_as(_P), units,
                                  ctypes.byref(n)))
    return [(u.expert, u.bits, u.load_from, u.load_to, u.count) for u in units[:n.value]]


def budget_plan(want, level_bytes, budget, resident):
    """``d2moe_budget_plan`` on host arrays: want [n_layers][E] level counts,
    level_bytes [K], resident [n_layers][E] uint8 (updated in place).
    Returns the actions as (action, layer, expert, level) tuples."""
    import numpy as np
    w = np.ascontiguousarray(want, dtype=np.uint8)
    lb = np.ascontiguousarray(level_bytes, dtype=np.int64)
    assert resident.dtype == np.uint8 and resident.flags["C_CONTIGUOUS"]
    nl, E = w.shape
    n = ctypes.c_int32()
    cap = 64
    while True:
        acts = (_BudgetAction * cap)()
        rc = lib().d2moe_budget_plan(w.ctypes.data_as(_P), nl, E, lb.ctypes.data_as(_P), lb.size,
                                     int(budget), resident.ctypes.data_as(_P), acts, cap,
                                     ctypes.byref(n))
        if rc == EINVAL and n.value > cap:
            cap = n.value
            continue
        _check("d2moe_budget_plan", rc)
        return [(a.action, a.layer, a.expert, a.level) for a in acts[:n.value]]


def moe_forward_streamed(x, host_w13: MWQ, host_w2: MWQ, w13: MWQ, w2: MWQ, resident, r: Routing,
                         k: int, hist_host, units, events, io_stream, out=None, workspace=None,
                         stream=None):
    """``d2moe_moe_forward_streamed``: host_w13 / host_w2 hold pinned host
    tensors, w13 / w2 the device copy; resident is a host uint8 numpy array
    [E] (updated in place); units as returned by hebf_order; events: one
    torch.cuda.Event per unit; io_stream: a torch.cuda.Stream, which waits for
    the work already on ``stream`` before its first copy."""
    import numpy as np
    T, d = x.shape
    E, d_ff = w13.n_experts, w2.cols
    if out is None:
        out = torch.empty_like(x)
    need = moe_forward_workspace(T, d, d_ff, E, k)
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=x.device)
    h = np.ascontiguousarray(hist_host, dtype=np.int32)
    assert resident.dtype == np.uint8 and resident.flags["C_CONTIGUOUS"]
    arr_u = (_Unit * max(1, len(units)))(*[_Unit(*u) for u in units])
    for ev in events:
        if ev.cuda_event == 0:
            ev.record(io_stream)          # torch creates the HIP event at its first record
    arr_e = (ctypes.c_void_p * max(1, len(units)))(*[ev.cuda_event for ev in events])
    c_h13, c_h2, c13, c2, cr = host_w13._c(), host_w2._c(), w13._c(), w2._c(), r._c()
    _check("d2moe_moe_forward_streamed",
           lib().d2moe_moe_forward_streamed(
               _ptr(x), _dtype_code(x), T, d, d_ff, E, k, ctypes.byref(c_h13), ctypes.byref(c_h2),
               ctypes.byref(c13), ctypes.byref(c2), resident.ctypes.data_as(_P), ctypes.byref(cr),
               h.ctypes.data_as(_P), arr_u, len(units), _ptr(out), _ptr(workspace),
               workspace.numel(), _stream(stream), ctypes.c_void_p(io_stream.cuda_stream), arr_e))
    return out
