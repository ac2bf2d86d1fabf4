"""Thin ctypes binding of libpt.so (see include/pt.h): argument marshalling only.

PyTorch is used for device memory (the four arenas, inputs, labels) and for the
HIP stream handle; every step of the training path runs in the library's
kernels.  There is no fallback: if the library is missing, loading fails.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
import threading

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpt.so")

PT_OK, PT_EINVAL, PT_ESTATE, PT_ENOMEM, PT_EDEVICE, PT_ECACHE_MISS = range(6)
PT_VIT_PRELN, PT_BERT_POSTLN = 0, 1
PT_F32, PT_BF16 = 0, 1
PT_SGDM, PT_ADAMW = 0, 1
PT_HEAD_DEFAULT, PT_HEAD_CLS = 0, 1
ATTN_ORDERS = {"full": 0, "causal": 1, "prefix": 2}
KIND_PARAM, KIND_GRAD, KIND_MOMENT1, KIND_MOMENT2, KIND_SHADOW = range(5)
ACT_HK, ACT_HL, ACT_LOGITS, ACT_DHK = range(4)
PROF_CATEGORIES = ("gemm_generic", "gemm_nn", "gemm_nt", "gemm_tn", "attn_fwd", "attn_bwd", "ln_fwd", "ln_bwd",
                   "colsum", "opt", "norms", "cache", "wgrad_block", "splitk_reduce")
_STATUS = {0: "PT_OK", 1: "PT_EINVAL", 2: "PT_ESTATE", 3: "PT_ENOMEM", 4: "PT_EDEVICE", 5: "PT_ECACHE_MISS"}


class PtConfig(C.Structure):
    _fields_ = [("arch", C.c_int32), ("dtype", C.c_int32), ("L", C.c_int32), ("D", C.c_int32), ("H", C.c_int32),
                ("F", C.c_int32), ("S", C.c_int32), ("B", C.c_int32), ("n_out", C.c_int32), ("img", C.c_int32),
                ("patch", C.c_int32), ("chans", C.c_int32), ("vocab", C.c_int32), ("max_pos", C.c_int32),
                ("ln_eps", C.c_float), ("optimizer", C.c_int32), ("head", C.c_int32), ("grad_accum", C.c_int32),
                ("k_min", C.c_int32), ("act8", C.c_int32), ("cache_slots", C.c_int64), ("host_slots", C.c_int64), ("window_slots", C.c_int64)]


class PtAttentionRule(C.Structure):
    _fields_ = [("order", C.c_int32), ("n", C.c_int32), ("cap", C.c_float), ("slopes", C.c_void_p), ("documents", C.c_void_p),
                ("prefix", C.c_void_p)]


class PtOptHparams(C.Structure):
    _fields_ = [("lr", C.c_float), ("momentum", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float),
                ("eps", C.c_float), ("weight_decay", C.c_float)]


class PtHeads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("sample", C.c_int64), ("row", C.c_int64), ("head", C.c_int64)]


class PtAttention(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("nb", C.c_int32), ("Sq", C.c_int32), ("Sk", C.c_int32), ("H", C.c_int32), ("Hkv", C.c_int32),
                ("dh", C.c_int32), ("order", C.c_int32), ("q0", C.c_int32), ("scale", C.c_float), ("cap", C.c_float),
                ("slopes", C.c_void_p), ("q_documents", C.c_void_p), ("k_documents", C.c_void_p), ("prefix", C.c_void_p)]


class PtError(RuntimeError):
    def __init__(self, status, msg=""):
        super().__init__(f"{_STATUS.get(status, status)}: {msg}")
        self.status = status


_lib = None


def load_library():
    """Loads libpt.so; raises if it has not been built (no fallback path)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2102_03161_amd.build`")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    P = C.POINTER
    sig = {
        "pt_query_arena_bytes": [P(PtConfig), P(sz), P(sz), P(sz), P(sz)],
        "pt_create": [P(PtConfig), vp, vp, vp, vp, vp, P(vp)],
        "pt_destroy": [vp],
        "pt_set_freeze_boundary": [vp, i32],
        "pt_get_freeze_boundary": [vp, P(i32)],
        "pt_set_attention": [vp, P(PtAttentionRule)],
        "pt_frozen_forward": [vp, vp, i32, P(i64), P(vp)],
        "pt_active_fwd_bwd": [vp, vp, vp, P(C.c_float)],
        "pt_last_loss": [vp, P(C.c_float)],
        "pt_layer_grad_norms": [vp, P(C.c_float)],
        "pt_layer_grad_norms_begin": [vp],
        "pt_layer_grad_norms_end": [vp, P(C.c_float)],
        "pt_layer_grad_norms_static": [vp, P(C.c_float)],
        "pt_optimizer_step": [vp, P(PtOptHparams)],
        "pt_accumulate_grads": [vp, i32],
        "pt_finish_accumulation": [vp, P(C.c_float)],
        "pt_next_boundary": [P(C.c_float), i32, i32, C.c_double, P(i32)],
        "pt_num_tensors": [vp, P(i32)],
        "pt_tensor_info": [vp, i32, C.c_char_p, sz, P(i64), P(i32), P(i32), P(i32), P(i32)],
        "pt_write_tensor": [vp, i32, i32, P(C.c_float)],
        "pt_read_tensor": [vp, i32, i32, P(C.c_float)],
        "pt_get_step_count": [vp, P(i64)],
        "pt_set_step_count": [vp, i64],
        "pt_read_activation": [vp, i32, P(C.c_float), sz],
        "pt_cache_row": [vp, i64, vp, sz, P(i32)],
        "pt_cache_stats": [vp, P(i64), P(i64), P(i64), P(i64)],
        "pt_time_frozen_forward": [vp, vp, i32, P(i64), i32, P(C.c_float), P(C.c_float)],
        "pt_attach_host_tier": [vp, vp, sz],
        "pt_cache_prefetch": [vp, P(i64), i32, P(i32)],
        "pt_host_tier_stats": [vp, P(i64), P(i64), P(i64), P(i64)],
        "pt_attention_workspace": [P(PtAttention), P(sz)],
        "pt_attention_fwd": [P(PtAttention), P(PtHeads), P(PtHeads), P(PtHeads), P(PtHeads), vp, vp],
        "pt_attention_bwd": [P(PtAttention), P(PtHeads), P(PtHeads), P(PtHeads), P(PtHeads), vp, P(PtHeads), P(PtHeads), P(PtHeads),
                             P(PtHeads), vp, sz, vp],
        "pt_gelu8_fwd": [i32, vp, vp, vp, vp, i64, i32, vp],
        "pt_gelu8_bwd": [i32, vp, vp, vp, vp, vp, i64, i32, vp],
        "pt_profile_enable": [vp, i32],
        "pt_profile_reset": [vp],
        "pt_profile_read": [vp, i32, P(C.c_double), P(i64), P(C.c_double)],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = C.c_int
    lib.pt_last_error.argtypes = [vp]
    lib.pt_last_error.restype = C.c_char_p
    _lib = lib
    return lib


def make_config(w: dict, B: int | None = None, cache_slots: int = 0, grad_accum: bool = False,
                host_slots: int = 0, window_slots: int = 0, k_min: int = 0, act8: bool = False) -> PtConfig:
    """pt_config from a workload dict (see synth.WORKLOADS)."""
    return PtConfig(
        arch=PT_VIT_PRELN if w["arch"] == "vit" else PT_BERT_POSTLN,
        dtype=PT_BF16 if w["dtype"] == "bf16" else PT_F32,
        L=w["L"], D=w["D"], H=w["H"], F=w["F"], S=w["S"], B=w["B"] if B is None else B, n_out=w["n_out"],
        img=w["img"], patch=w["patch"], chans=w["chans"], vocab=w["vocab"], max_pos=w["max_pos"],
        ln_eps=w["ln_eps"], optimizer=PT_ADAMW if w["optimizer"] == "adamw" else PT_SGDM,
        head=PT_HEAD_CLS if w.get("head", "default") == "cls" else PT_HEAD_DEFAULT, grad_accum=1 if grad_accum else 0,
        k_min=k_min, act8=1 if act8 else 0, cache_slots=cache_slots, host_slots=host_slots, window_slots=window_slots)


def query_arena_bytes(cfg: PtConfig):
    lib = load_library()
    a, b, c, d = C.c_size_t(), C.c_size_t(), C.c_size_t(), C.c_size_t()
    st = lib.pt_query_arena_bytes(C.byref(cfg), C.byref(a), C.byref(b), C.byref(c), C.byref(d))
    if st != PT_OK:
        raise PtError(st, "pt_query_arena_bytes")
    return a.value, b.value, c.value, d.value


def next_boundary(norms, L: int, k_prev: int, alpha: float) -> int:
    lib = load_library()
    arr = np.ascontiguousarray(norms, dtype=np.float32)
    out = C.c_int32()
    st = lib.pt_next_boundary(arr.ctypes.data_as(C.POINTER(C.c_float)), L, k_prev, alpha, C.byref(out))
    if st != PT_OK:
        raise PtError(st, "pt_next_boundary")
    return out.value


# ---- operators by themselves (no context) ---------------------------------------
# Tensors are PyTorch's, on one GPU; work goes to that GPU's current stream, outputs and scratch come from the caching
# allocator on it.  A call takes the host about as long as a short kernel takes the GPU, so nothing here formats a message
# or imports a module unless something is wrong.
_torch = None
_DTYPES = {}


def _op_setup():
    global _torch
    import torch
    _torch = torch
    _DTYPES.update({torch.float32: PT_F32, torch.bfloat16: PT_BF16})
    return torch


def _refuse(what: str):
    raise PtError(PT_EINVAL, what)


def _dtype_of(t) -> int:
    if not _DTYPES:
        _op_setup()
    d = _DTYPES.get(t.dtype)
    return _refuse(f"dtype {t.dtype}: float32 or bfloat16") if d is None else d


def _device_of(first, *others) -> int:
    """The index of the GPU that all tensors are on (None: no tensor)."""
    at = first.get_device()
    if at < 0:
        _refuse(f"tensors must be on a GPU, not on {first.device}")
    for t in others:
        if t is not None and t.get_device() != at:
            _refuse(f"a tensor on {t.device}, the first on {first.device}")
    return at


class _Args(threading.local):
    """Room for the structs of one call of this thread, filled in one go: a pt_attention and up to eight pt_heads behind it.  (A
    call reads them before it returns; making ten ctypes objects takes longer than a short kernel.)"""

    def __init__(self):
        self.buf = C.create_string_buffer(80 + 8 * 32)
        self.at = C.addressof(self.buf)
        self.heads = [self.at + 80 + 32 * i for i in range(8)]


_args = _Args()
_PACK = {n: struct.Struct("9i2f4x4Q" + n * "Qqqq").pack_into for n in (4, 8)}


def _fast_library():
    """The library with pointers taken as plain addresses."""
    global _fast
    load_library()
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    lib.pt_attention_fwd.argtypes = [vp] * 7
    lib.pt_attention_bwd.argtypes = [vp] * 11 + [sz, vp]
    lib.pt_gelu8_fwd.argtypes = [i32, vp, vp, vp, vp, i64, i32, vp]
    lib.pt_gelu8_bwd.argtypes = [i32, vp, vp, vp, vp, vp, i64, i32, vp]
    _fast = lib
    return lib


_fast = None


def _launch(at: int, call, *args):
    """call(*args, current stream of GPU `at`), with that GPU as the current one."""
    if at == _torch.cuda.current_device():
        st = call(*args, _torch._C._cuda_getCurrentRawStream(at))
    else:
        with _torch.cuda.device(at):
            st = call(*args, _torch._C._cuda_getCurrentRawStream(at))
    if st != PT_OK:
        raise PtError(st, (load_library().pt_last_error(None) or b"").decode())


def _heads(t, name: str, shape, dtype) -> tuple:
    """The four fields of a pt_heads."""
    if t.shape != shape or t.dtype is not dtype:
        _refuse(f"{name}: {t.dtype} {tuple(t.shape)}, not {dtype} {tuple(shape)}")
    a, b, c, d = t.stride()
    if d != 1 and t.numel() > 0:
        _refuse(f"{name}: the head size must be contiguous")
    return t.data_ptr(), a, b, c


def _plain(t, dtype, shape, name: str):
    if t is None:
        _refuse(f"{name} is None")
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        _refuse(f"{name}: {dtype} {list(shape)}, contiguous (got {t.dtype} {list(t.shape)})")
    return t.data_ptr()


class AttentionRule:
    """What a query sees and how its scores are bent (pt_attention in include/pt.h).

    order        "full", "causal", or "prefix" (causal, and the first prefix[sample] keys)
    scale        None: 1 / sqrt(head size)
    cap          0, or c of c tanh(s / c)
    slopes       float32 [H]: a bias of -slope |i - j|
    documents    int32 [nb, keys], below 0: padding; q_documents int32 [nb, queries], None: the same tensor
    prefix       int32 [nb]
    q0           position of query 0 among the keys
    """

    def __init__(self, order="full", scale=None, cap=0.0, slopes=None, documents=None, q_documents=None, prefix=None, q0=0):
        if order not in ATTN_ORDERS:
            _refuse(f"order {order!r}: one of {', '.join(ATTN_ORDERS)}")
        if not 0 <= q0 < 1 << 24 or not (cap == 0.0 or 1e-38 <= cap <= 3e38) or not (scale is None or 0.0 < scale <= 3e38):
            _refuse(f"q0 {q0}, cap {cap}, scale {scale}: q0 in 0 .. 2^24, cap not negative, scale positive")
        self.order, self.scale, self.cap, self.q0 = order, scale, cap, q0
        self.slopes, self.documents, self.prefix = slopes, documents, prefix
        self.q_documents = documents if q_documents is None else q_documents
        if self.q_documents is not None and documents is None:
            _refuse("documents of the queries and of the keys go together")

    def _fields(self, q, k) -> tuple:
        """The fields of pt_attention for these tensors."""
        if q.dim() != 4 or k.dim() != 4:
            _refuse("q, k and v: [samples, rows, heads, head size]")
        nb, Sq, H, dh = q.shape
        kb, Sk, Hkv, kd = k.shape
        if kb != nb or kd != dh:
            _refuse(f"q {tuple(q.shape)} and k {tuple(k.shape)} differ in samples or head size")
        dtype = _dtype_of(q)
        slopes = qd = kdoc = prefix = 0
        if self.slopes is not None:
            slopes = _plain(self.slopes, _torch.float32, (H,), "slopes")
        if self.documents is not None:
            kdoc = _plain(self.documents, _torch.int32, (nb, Sk), "documents")
            qd = kdoc if self.q_documents is self.documents and Sq == Sk else _plain(self.q_documents, _torch.int32, (nb, Sq), "q_documents")
        if self.order == "prefix":
            if self.prefix is None:
                _refuse("order \"prefix\" needs prefix lengths")
            prefix = _plain(self.prefix, _torch.int32, (nb,), "prefix")
        return (dtype, nb, Sq, Sk, H, Hkv, dh, ATTN_ORDERS[self.order], self.q0,
                (dh ** -0.5 if dh else 1.0) if self.scale is None else self.scale, self.cap, slopes, qd, kdoc, prefix)

    def describe(self, q, k) -> PtAttention:
        return PtAttention(*self._fields(q, k))


_FULL = AttentionRule()


def attention_forward(q, k, v, rule: AttentionRule | None = None, out=None, want_lse: bool = True):
    """(o, lse): q [nb, Sq, H, dh], k and v [nb, Sk, Hkv, dh], views of any strides that are multiples of 16 bytes; o like q, lse
    float32 [nb, H, Sq] (None if not wanted)."""
    rule = rule or _FULL
    a = rule._fields(q, k)
    qs, ks, dtype = q.shape, k.shape, q.dtype
    hq, hk, hv = _heads(q, "q", qs, dtype), _heads(k, "k", ks, dtype), _heads(v, "v", ks, dtype)
    at = _device_of(q, k, v, out, rule.slopes, rule.documents, rule.q_documents, rule.prefix)
    _, nb, Sq, _, H, _, dh = a[:7]
    o = _torch.empty_like(q, memory_format=_torch.contiguous_format) if out is None else out
    lse = _torch.empty((nb, H, Sq), dtype=_torch.float32, device=q.device) if want_lse else None
    lib, args = _fast or _fast_library(), _args
    _PACK[4](args.buf, 0, *a, *hq, *hk, *hv, *((o.data_ptr(), Sq * H * dh, H * dh, dh) if out is None else _heads(o, "out", qs, dtype)))
    _launch(at, lib.pt_attention_fwd, args.at, *args.heads[:4], lse.data_ptr() if want_lse else None)
    return o, lse


def attention_backward(q, k, v, o, lse, do, rule: AttentionRule | None = None, grads=None):
    """(dq, dk, dv) of the call that returned (o, lse); grads: tensors (views) to write them to."""
    rule = rule or _FULL
    a = rule._fields(q, k)
    qs, ks, dtype = q.shape, k.shape, q.dtype
    _, nb, Sq, Sk, H, Hkv, dh = a[:7]
    hq, hk, hv = _heads(q, "q", qs, dtype), _heads(k, "k", ks, dtype), _heads(v, "v", ks, dtype)
    ho, hd = _heads(o, "o", qs, dtype), _heads(do, "do", qs, dtype)
    stats = _plain(lse, _torch.float32, (nb, H, Sq), "lse")
    at = _device_of(q, k, v, o, lse, do, rule.slopes, rule.documents, rule.q_documents, rule.prefix, *(grads or ()))
    if grads is None:
        dense = _torch.contiguous_format
        dq, dk, dv = _torch.empty_like(q, memory_format=dense), _torch.empty_like(k, memory_format=dense), _torch.empty_like(k, memory_format=dense)
        rq, rk = (Sq * H * dh, H * dh, dh), (Sk * Hkv * dh, Hkv * dh, dh)
        out = (dq.data_ptr(), *rq, dk.data_ptr(), *rk, dv.data_ptr(), *rk)
    else:
        dq, dk, dv = grads
        out = (*_heads(dq, "dq", qs, dtype), *_heads(dk, "dk", ks, dtype), *_heads(dv, "dv", ks, dtype))
    lib, args = _fast or _fast_library(), _args
    _PACK[8](args.buf, 0, *a, *hq, *hk, *hv, *ho, *hd, *out)
    floats = nb * H * Sq * (2 if dtype is _torch.float32 else 1)      # as many as pt_attention_workspace asks for, which the call checks
    ws = _torch.empty(floats, dtype=_torch.float32, device=q.device)
    h = args.heads
    _launch(at, lib.pt_attention_bwd, args.at, h[0], h[1], h[2], h[3], stats, h[4], h[5], h[6], h[7], ws.data_ptr(), 4 * floats)
    return dq, dk, dv


def gelu8_forward(h):
    """(g, codes, exps): GELU of h [rows, F] and the 8-bit checkpoint of h that gelu8_backward reads."""
    dtype = _dtype_of(h)
    if h.dim() != 2 or not h.is_contiguous():
        _refuse("h: [rows, F], contiguous")
    T, F = h.shape
    at, dev = _device_of(h), h.device
    g = _torch.empty_like(h)
    codes = _torch.empty((T, F), dtype=_torch.int8, device=dev)
    exps = _torch.empty((T, (F + 31) // 32), dtype=_torch.uint8, device=dev)
    lib = _fast or _fast_library()
    _launch(at, lib.pt_gelu8_fwd, dtype, h.data_ptr(), g.data_ptr(), codes.data_ptr(), exps.data_ptr(), T, F)
    return g, codes, exps


def gelu8_backward(codes, exps, dg, want_activation: bool = True, out=None):
    """(dh, g): dg GELU'(x) and GELU(x) (None if not wanted) of the checkpointed x; out: where dh goes (it may be dg itself)."""
    dtype = _dtype_of(dg)
    if dg.dim() != 2 or not dg.is_contiguous():
        _refuse("dg: [rows, F], contiguous")
    T, F = dg.shape
    pc = _plain(codes, _torch.int8, (T, F), "codes")
    pe = _plain(exps, _torch.uint8, (T, (F + 31) // 32), "exps")
    at = _device_of(dg, codes, exps, out)
    dh = _torch.empty_like(dg) if out is None else out
    pd = dh.data_ptr() if out is None else _plain(out, dg.dtype, (T, F), "out")
    g = _torch.empty_like(dg) if want_activation else None
    lib = _fast or _fast_library()
    _launch(at, lib.pt_gelu8_bwd, dtype, pc, pe, dg.data_ptr(), pd, g.data_ptr() if want_activation else None, T, F)
    return dh, g


class Context:
    """Owns the device arenas (torch tensors) and a pt_ctx."""

    def __init__(self, cfg: PtConfig, device="cuda:0", stream=None):
        import torch
        self.torch = torch
        self.lib = load_library()
        self.cfg = cfg
        self.device = torch.device(device)
        sizes = query_arena_bytes(cfg)
        with torch.cuda.device(self.device):
            self.arenas = [torch.empty(max(n, 256), dtype=torch.uint8, device=self.device) for n in sizes]
            self.stream = torch.cuda.current_stream(self.device) if stream is None else stream
            h = C.c_void_p()
            st = self.lib.pt_create(C.byref(cfg), *[C.c_void_p(a.data_ptr()) for a in self.arenas[:3]],
                                    C.c_void_p(self.arenas[3].data_ptr()) if cfg.cache_slots + cfg.window_slots > 0 else None,
                                    C.c_void_p(self.stream.cuda_stream), C.byref(h))
        if st != PT_OK:
            raise PtError(st, "pt_create")
        self.h = h
        self.esz = 2 if cfg.dtype == PT_BF16 else 4
        self._names = None
        self.host_tier = None
        if cfg.host_slots > 0:
            # the lower cache tier: pinned host memory owned here, attached once
            nbytes = cfg.host_slots * cfg.S * cfg.D * self.esz
            self.host_tier = torch.empty(nbytes, dtype=torch.uint8, pin_memory=True)
            self._chk(self.lib.pt_attach_host_tier(self.h, C.c_void_p(self.host_tier.data_ptr()), nbytes))

    def close(self):
        if self.h:
            self.lib.pt_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _chk(self, st, allow=()):
        if st != PT_OK and st not in allow:
            raise PtError(st, (self.lib.pt_last_error(self.h) or b"").decode())
        return st

    # ---- the five calls ------------------------------------------------------
    def set_freeze_boundary(self, k: int):
        self._chk(self.lib.pt_set_freeze_boundary(self.h, k))

    def get_freeze_boundary(self) -> int:
        k = C.c_int32()
        self._chk(self.lib.pt_get_freeze_boundary(self.h, C.byref(k)))
        return k.value

    def set_attention(self, rule: AttentionRule | None):
        """Attention of every block under `rule` (its scale and q0 are the context's own: 1 / sqrt(D / H) and 0), from the next
        batch on; None: plain attention.  documents [n, S] and prefix [n] describe the batches' samples by position.  The tensors may be
        temporaries of the current stream, whichever stream the context works on."""
        if rule is None:
            self._chk(self.lib.pt_set_attention(self.h, None))
            return
        if rule.scale is not None or rule.q0 != 0 or rule.q_documents is not rule.documents:
            _refuse("a context's rule has neither scale nor q0, and one set of documents")
        if not _DTYPES:
            _op_setup()
        r = PtAttentionRule(ATTN_ORDERS[rule.order], 0, rule.cap)
        given = [t for t in (rule.documents, rule.prefix if rule.order == "prefix" else None) if t is not None]
        if given:
            r.n = given[0].shape[0]
        if rule.slopes is not None:
            r.slopes = _plain(rule.slopes, _torch.float32, (self.cfg.H,), "slopes")
        if rule.documents is not None:
            r.documents = _plain(rule.documents, _torch.int32, (r.n, self.cfg.S), "documents")
        if rule.order == "prefix" and rule.prefix is not None:
            r.prefix = _plain(rule.prefix, _torch.int32, (r.n,), "prefix")
        for t in (rule.slopes, *given):
            if t is not None and t.device != self.arenas[0].device:
                _refuse(f"a tensor on {t.device}, the context on {self.arenas[0].device}")
        here = _torch.cuda.current_stream(self.device)
        if here != self.stream:     # the copies wait for what made the tensors, and the tensors' memory for the copies
            self.stream.wait_stream(here)
            for t in (rule.slopes, *given):
                if t is not None:
                    t.record_stream(self.stream)
        self._chk(self.lib.pt_set_attention(self.h, r))

    def frozen_forward(self, d_input, sample_ids=None) -> int:
        """d_input: torch tensor on the device.  Returns the device pointer of h_k."""
        nb = int(d_input.shape[0])
        ids = None
        if sample_ids is not None:
            arr = np.ascontiguousarray(sample_ids, dtype=np.int64)
            assert arr.shape == (nb,)
            ids = arr.ctypes.data_as(C.POINTER(C.c_int64))
        out = C.c_void_p()
        self._chk(self.lib.pt_frozen_forward(self.h, C.c_void_p(d_input.data_ptr()), nb, ids, C.byref(out)))
        return out.value

    def active_fwd_bwd(self, d_hk: int, d_labels, want_loss=True):
        loss = C.c_float()
        self._chk(self.lib.pt_active_fwd_bwd(self.h, C.c_void_p(d_hk), C.c_void_p(d_labels.data_ptr()),
                                             C.byref(loss) if want_loss else None))
        return loss.value if want_loss else None

    def last_loss(self) -> float:
        loss = C.c_float()
        self._chk(self.lib.pt_last_loss(self.h, C.byref(loss)))
        return loss.value

    def layer_grad_norms(self) -> np.ndarray:
        out = np.zeros(self.cfg.L + 2, dtype=np.float32)
        self._chk(self.lib.pt_layer_grad_norms(self.h, out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    def layer_grad_norms_static(self) -> np.ndarray:
        out = np.zeros(self.cfg.L + 2, dtype=np.float32)
        self._chk(self.lib.pt_layer_grad_norms_static(self.h, out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    def layer_grad_norms_begin(self):
        self._chk(self.lib.pt_layer_grad_norms_begin(self.h))

    def layer_grad_norms_end(self) -> np.ndarray:
        out = np.zeros(self.cfg.L + 2, dtype=np.float32)
        self._chk(self.lib.pt_layer_grad_norms_end(self.h, out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    def accumulate_grads(self, first: bool):
        self._chk(self.lib.pt_accumulate_grads(self.h, 1 if first else 0))

    def finish_accumulation(self, want_loss: bool = True):
        out = C.c_float()
        self._chk(self.lib.pt_finish_accumulation(self.h, C.byref(out) if want_loss else None))
        return out.value if want_loss else None

    def optimizer_step(self, lr, momentum=0.9, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0):
        hp = PtOptHparams(lr, momentum, beta1, beta2, eps, weight_decay)
        self._chk(self.lib.pt_optimizer_step(self.h, C.byref(hp)))

    # ---- tensor table --------------------------------------------------------
    def tensors(self):
        """[(id, name, shape, group, decayed)] in arena order."""
        if self._names is None:
            n = C.c_int32()
            self._chk(self.lib.pt_num_tensors(self.h, C.byref(n)))
            out = []
            for i in range(n.value):
                buf = C.create_string_buffer(64)
                numel, rows, cols, grp, dec = C.c_int64(), C.c_int32(), C.c_int32(), C.c_int32(), C.c_int32()
                self._chk(self.lib.pt_tensor_info(self.h, i, buf, 64, C.byref(numel), C.byref(rows), C.byref(cols),
                                                  C.byref(grp), C.byref(dec)))
                shape = (cols.value,) if rows.value == 1 else (rows.value, cols.value)
                out.append((i, buf.value.decode(), shape, grp.value, bool(dec.value)))
            self._names = out
        return self._names

    def write_tensor(self, tid: int, kind: int, arr):
        a = np.ascontiguousarray(arr, dtype=np.float32)
        self._chk(self.lib.pt_write_tensor(self.h, tid, kind, a.ctypes.data_as(C.POINTER(C.c_float))))

    def read_tensor(self, tid: int, kind: int) -> np.ndarray:
        _, _, shape, _, _ = self.tensors()[tid]
        out = np.empty(shape, dtype=np.float32)
        self._chk(self.lib.pt_read_tensor(self.h, tid, kind, out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    def get_step_count(self) -> int:
        t = C.c_int64()
        self._chk(self.lib.pt_get_step_count(self.h, C.byref(t)))
        return t.value

    def set_step_count(self, t: int):
        self._chk(self.lib.pt_set_step_count(self.h, t))

    def read_activation(self, which: int, shape) -> np.ndarray:
        out = np.empty(shape, dtype=np.float32)
        self._chk(self.lib.pt_read_activation(self.h, which, out.ctypes.data_as(C.POINTER(C.c_float)), out.size))
        return out

    # ---- cache ---------------------------------------------------------------
    def cache_row(self, sample_id: int):
        """(raw row bytes as uint8 array, k the row was written at) or None on a miss."""
        n = self.cfg.S * self.cfg.D * self.esz
        out = np.empty(n, dtype=np.uint8)
        k = C.c_int32()
        st = self._chk(self.lib.pt_cache_row(self.h, sample_id, C.c_void_p(out.ctypes.data), n, C.byref(k)),
                       allow=(PT_ECACHE_MISS,))
        return None if st == PT_ECACHE_MISS else (out, k.value)

    def cache_stats(self):
        a, b, c, d = C.c_int64(), C.c_int64(), C.c_int64(), C.c_int64()
        self._chk(self.lib.pt_cache_stats(self.h, C.byref(a), C.byref(b), C.byref(c), C.byref(d)))
        return {"hits": a.value, "advances": b.value, "misses": c.value, "block_runs": d.value}

    def time_frozen_forward(self, d_input, sample_ids, reps: int = 3):
        """(ms per call recomputing the prefix, ms per call served from the cache) for this batch."""
        ids = np.ascontiguousarray(sample_ids, dtype=np.int64)
        a, b = C.c_float(), C.c_float()
        self._chk(self.lib.pt_time_frozen_forward(self.h, C.c_void_p(d_input.data_ptr()), len(ids),
                                                  ids.ctypes.data_as(C.POINTER(C.c_int64)), reps, C.byref(a), C.byref(b)))
        return a.value, b.value

    def cache_prefetch(self, sample_ids) -> int:
        ids = np.ascontiguousarray(sample_ids, dtype=np.int64)
        n = C.c_int32()
        self._chk(self.lib.pt_cache_prefetch(self.h, ids.ctypes.data_as(C.POINTER(C.c_int64)), len(ids), C.byref(n)))
        return n.value

    def host_tier_stats(self):
        a, b, c, d = C.c_int64(), C.c_int64(), C.c_int64(), C.c_int64()
        self._chk(self.lib.pt_host_tier_stats(self.h, C.byref(a), C.byref(b), C.byref(c), C.byref(d)))
        return {"rows_to_device": a.value, "rows_to_host": b.value, "prefetched": c.value, "prefetched_used": d.value}

    # ---- kernel timing ---------------------------------------------------------
    def profile_enable(self, on: bool):
        self._chk(self.lib.pt_profile_enable(self.h, 1 if on else 0))

    def profile_reset(self):
        self._chk(self.lib.pt_profile_reset(self.h))

    def profile_read(self) -> dict:
        """{category: (total_ms, launches, work)}"""
        out = {}
        for i, name in enumerate(PROF_CATEGORIES):
            ms, n, wk = C.c_double(), C.c_int64(), C.c_double()
            self._chk(self.lib.pt_profile_read(self.h, i, C.byref(ms), C.byref(n), C.byref(wk)))
            out[name] = (ms.value, n.value, wk.value)
        return out
