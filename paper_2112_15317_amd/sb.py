"""Thin Python binding of libsb (include/sb.h): argument marshalling only.

Every function has the name of the C entry point it calls and takes torch
tensors that live on the GPU (torch provides device memory and streams, and
nothing else here): the tensor's dtype selects SB_F32 / SB_BF16, its data
pointer is passed through, and the current torch stream is the HIP stream
unless one is given.  Every step of the computation runs in libsb's HIP
kernels.  A non-OK status raises ``SBError``.

The library must have been built (``python -m paper_2112_15317_amd.build``);
if ``libsb.so`` is missing, loading fails loudly: there is no fallback.
"""
from __future__ import annotations

import ctypes
import os
import threading

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsb.so")

SB_OK, SB_ERR_INVALID_ARG, SB_ERR_UNSUPPORTED, SB_ERR_WORKSPACE, SB_ERR_HIP = range(5)
SB_F32, SB_BF16 = 0, 1
SB_NCHW, SB_NCHW8C = 0, 1
SB_FUSE_RELU = 1
SB_PACKED_FILTERS = 2
SB_UNALIGNED = 4
SB_TOP_PROBS = 8
SB_PASS_FWD, SB_PASS_BWD_DATA, SB_PASS_BWD_WEIGHT, SB_PASS_FWD_POOL = 0, 1, 2, 3
SIZE_MAX = 2 ** 64 - 1          # (size_t)-1: the workspace queries' "not supported"
SB_FC_FWD, SB_FC_BWD = 0, 1
SB_ACT_SIGMOID, SB_ACT_SILU, SB_ACT_GELU, SB_ACT_GELU_TANH, SB_ACT_RELU = range(5)
SB_SGD_MAX_TENSORS = 64
SB_ADAMW_MAX_TENSORS, SB_ADAMW_BLOCK = 512, 256
SB_MAX_EXPERTS, SB_LOGP_MAX_TOP = 512, 32
SB_NOALLOC_SCRATCH_BYTES = 40 << 20

_vp = ctypes.c_void_p
_i = ctypes.c_int
_sz = ctypes.c_size_t


class sb_conv3x3_desc(ctypes.Structure):
    _fields_ = [("n", _i), ("c", _i), ("h", _i), ("w", _i), ("k", _i),
                ("dtype", _i), ("flags", ctypes.c_uint), ("layout", _i)]


class sb_fc_desc(ctypes.Structure):
    _fields_ = [("m", _i), ("k_in", _i), ("n_shard", _i), ("dtype", _i),
                ("ldx", _i), ("ldy", _i), ("flags", ctypes.c_uint)]


class sb_adamw_desc(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", _i), ("seed", ctypes.c_uint32)]


class sb_adamw_plan(ctypes.Structure):
    _fields_ = [("tensors", _i), ("moments", _i), ("groups", _i), ("blocks", _i)]


class sb_adamw_tensor(ctypes.Structure):
    _fields_ = [("w", _vp), ("copy", _vp), ("g", _vp), ("m", _vp), ("v", _vp), ("m_top", _vp),
                ("v_top", _vp), ("first", ctypes.c_uint64), ("n", _sz),
                ("grad_scale", ctypes.c_float), ("decay", ctypes.c_float)]


class sb_gated_desc(ctypes.Structure):
    _fields_ = [("m", _i), ("k_in", _i), ("n_shard", _i), ("dtype", _i), ("act", _i),
                ("ldx", _i), ("ldy", _i), ("flags", ctypes.c_uint)]


class sb_embed_desc(ctypes.Structure):
    _fields_ = [("tokens", _i), ("vocab", _i), ("width", _i), ("first", _i), ("dtype", _i),
                ("ldy", _i), ("scale", ctypes.c_float)]


class sb_expert_desc(ctypes.Structure):
    _fields_ = [("tokens", _i), ("top", _i), ("experts", _i), ("first", _i), ("width", _i),
                ("dtype", _i), ("ldx", _i), ("ldr", _i)]


class sb_token_logp_desc(ctypes.Structure):
    _fields_ = [("m", _i), ("classes", _i), ("ldz", _i), ("dtype", _i), ("top", _i),
                ("flags", ctypes.c_uint)]


class sb_modulo_desc(ctypes.Structure):
    _fields_ = [("workers", _i), ("mp", _i), ("batch", _i), ("features", _i)]


class sb_shard_desc(ctypes.Structure):
    _fields_ = [("workers", _i), ("mp", _i), ("rows", _i), ("shard", _i)]


# Every exported symbol of include/sb.h with its ctypes signature.
SIGNATURES = {
    "sb_status_string": (ctypes.c_char_p, [_i]),
    "sb_version": (_i, []),
    "sb_conv3x3_workspace_bytes": (_sz, [ctypes.POINTER(sb_conv3x3_desc), _i]),
    "sb_conv3x3_packed_bytes": (_sz, [ctypes.POINTER(sb_conv3x3_desc), _i]),
    "sb_conv3x3_pack_filters": (_i, [ctypes.POINTER(sb_conv3x3_desc), _i, _vp, _vp, _sz, _vp]),
    "sb_conv3x3_pack_filters_many": (_i, [_i, ctypes.POINTER(sb_conv3x3_desc),
                                          ctypes.POINTER(_i), ctypes.POINTER(_vp),
                                          ctypes.POINTER(_vp), ctypes.POINTER(_sz), _vp]),
    "sb_conv3x3_plan_string": (_sz, [ctypes.POINTER(sb_conv3x3_desc), _i, ctypes.c_char_p, _sz]),
    "sb_conv3x3_fwd": (_i, [ctypes.POINTER(sb_conv3x3_desc), _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sb_conv3x3_fwd_pool": (_i, [ctypes.POINTER(sb_conv3x3_desc), _vp, _vp, _vp, _vp, _vp, _vp,
                                 _sz, _vp]),
    "sb_conv3x3_bwd_data": (_i, [ctypes.POINTER(sb_conv3x3_desc), _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sb_conv3x3_bwd_weight": (_i, [ctypes.POINTER(sb_conv3x3_desc), _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sb_conv3x3_bwd_weight_noalloc": (_i, [ctypes.POINTER(sb_conv3x3_desc), _vp, _vp, _vp, _vp,
                                           _vp]),
    "sb_conv3x3_bwd_weight_many_workspace_bytes": (_sz, [_i, ctypes.POINTER(sb_conv3x3_desc)]),
    "sb_conv3x3_bwd_weight_many": (_i, [_i, ctypes.POINTER(sb_conv3x3_desc), ctypes.POINTER(_vp),
                                        ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                        ctypes.POINTER(_vp), _vp, _sz, _vp]),
    "sb_relu_maxpool_fwd": (_i, [_i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp]),
    "sb_relu_maxpool_bwd": (_i, [_i, _i, _i, _i, _i, _i, _vp, _vp, _vp, _vp]),
    "sb_fc_workspace_bytes": (_sz, [ctypes.POINTER(sb_fc_desc), _i]),
    "sb_fc_shard_fwd": (_i, [ctypes.POINTER(sb_fc_desc), _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "sb_fc_shard_bwd": (_i, [ctypes.POINTER(sb_fc_desc), _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i,
                             _vp, _sz, _vp]),
    "sb_gated_workspace_bytes": (_sz, [ctypes.POINTER(sb_gated_desc), _i]),
    "sb_gated_shard_fwd": (_i, [ctypes.POINTER(sb_gated_desc), _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                _vp, _sz, _vp]),
    "sb_gated_shard_bwd": (_i, [ctypes.POINTER(sb_gated_desc), _vp, _vp, _vp, _vp, _vp, _vp, _vp,
                                _vp, _vp, _vp, _i, _vp, _sz, _vp]),
    "sb_modulo_fwd": (_i, [ctypes.POINTER(sb_modulo_desc), _i, _i, _vp, _sz, _vp, _vp]),
    "sb_modulo_bwd": (_i, [ctypes.POINTER(sb_modulo_desc), _i, _i, _vp, _sz, _vp, _sz, _vp]),
    "sb_shard_fwd": (_i, [ctypes.POINTER(sb_shard_desc), _i, _vp, _sz, _vp, _vp]),
    "sb_shard_bwd": (_i, [ctypes.POINTER(sb_shard_desc), _i, _vp, _sz, _vp, _sz, _vp]),
    "sb_model_average": (_i, [_i, _i, _sz, _vp, _sz, _vp]),
    "sb_model_average_replicas": (_i, [_i, _sz, ctypes.POINTER(_vp), _vp]),
    "sb_log_softmax_nll": (_i, [_i, _i, _i, _vp, _vp, ctypes.c_float, _vp, _vp, _vp, _vp]),
    "sb_sgd_update": (_i, [_i, ctypes.POINTER(_vp), ctypes.POINTER(_vp), ctypes.POINTER(_sz),
                           ctypes.POINTER(ctypes.c_float), ctypes.c_float, _vp]),
    "sb_adamw_plan_bytes": (_sz, [_i]),
    "sb_adamw_make_plan": (_i, [_i, _i, ctypes.POINTER(sb_adamw_tensor), _vp, _sz,
                                ctypes.POINTER(sb_adamw_plan), _vp]),
    "sb_adamw_update": (_i, [ctypes.POINTER(sb_adamw_desc), ctypes.POINTER(sb_adamw_plan), _vp, _vp,
                             _vp]),
    "sb_adamw_advance": (_i, [_vp, _vp]),
    "sb_adamw_unpack": (_i, [_sz, _vp, _vp, _vp, _vp, _vp, _vp, _vp]),
    "sb_embed_workspace_bytes": (_sz, [ctypes.POINTER(sb_embed_desc)]),
    "sb_embed_fwd": (_i, [ctypes.POINTER(sb_embed_desc), _vp, _vp, _vp, _vp]),
    "sb_embed_bwd": (_i, [ctypes.POINTER(sb_embed_desc), _vp, _vp, _vp, _i, _vp, _sz, _vp]),
    "sb_expert_workspace_bytes": (_sz, [ctypes.POINTER(sb_expert_desc)]),
    "sb_expert_sort": (_i, [ctypes.POINTER(sb_expert_desc), _vp, _vp, _vp, _vp, _sz, _vp]),
    "sb_expert_gather": (_i, [ctypes.POINTER(sb_expert_desc), _vp, _vp, _vp, _vp]),
    "sb_expert_combine": (_i, [ctypes.POINTER(sb_expert_desc), _vp, _vp, _vp, _vp, _vp, _vp]),
    "sb_expert_combine_bwd": (_i, [ctypes.POINTER(sb_expert_desc), _vp, _vp, _vp, _vp, _vp, _vp,
                                   _vp]),
    "sb_token_logp_workspace_bytes": (_sz, [ctypes.POINTER(sb_token_logp_desc)]),
    "sb_token_logp_fwd": (_i, [ctypes.POINTER(sb_token_logp_desc), _vp, _vp, _vp, _vp, _vp, _vp,
                               _vp, _vp, _sz, _vp]),
    "sb_token_logp_bwd": (_i, [ctypes.POINTER(sb_token_logp_desc), _vp, _vp, _vp, _vp, _vp, _vp,
                               _vp, _vp, _vp, _vp, _vp]),
}

_lock = threading.Lock()
_lib = None


class SBError(RuntimeError):
    def __init__(self, fn, status):
        self.status = status
        super().__init__("%s failed: %s" % (fn, status_name(status)))


def load():
    """Load libsb.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(
                    "libsb.so not found at %s: build it with "
                    "`python -m paper_2112_15317_amd.build` (no fallback exists)" % LIB_PATH)
            lib = ctypes.CDLL(LIB_PATH)
            for name, (res, args) in SIGNATURES.items():
                fn = getattr(lib, name)
                fn.restype = res
                fn.argtypes = args
            _lib = lib
    return _lib


def status_name(status: int) -> str:
    return load().sb_status_string(int(status)).decode()


def _check(fn, status):
    if status != SB_OK:
        raise SBError(fn, status)


# ----------------------------------------------------------- marshalling --
def _dtype_code(t):
    import torch
    if t.dtype == torch.float32:
        return SB_F32
    if t.dtype == torch.bfloat16:
        return SB_BF16
    raise TypeError("libsb takes float32 or bfloat16 tensors, got %s" % t.dtype)


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("libsb takes device tensors")
    if not t.is_contiguous():
        raise ValueError("libsb takes contiguous tensors (strides go in the descriptor)")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


_torch = _get_device = _raw_stream = None      # of torch, once a call has needed them


def _stream_for(t, stream):
    """The stream of a call on t's device, which has to be the current one.  (Where torch
    has it, by its number alone: a Stream object takes 2.5 of the 9 us of a small call.)"""
    global _torch, _get_device, _raw_stream
    if _torch is None:
        import torch
        _get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream",
                              lambda dev: torch.cuda.current_stream().cuda_stream)
        _torch = torch                       # last: other threads look at it
    on = getattr(t, "device", None)          # of a tensor; None and addresses have none
    if on is None:
        if stream is not None:
            return _stream(stream)
        return _raw_stream(_torch.cuda.current_device())
    dev = _get_device()
    if on.index != dev:
        raise ValueError("tensors on %s, current device %d" % (on, dev))
    return _raw_stream(dev) if stream is None else _stream(stream)


def _ws(ws):
    if ws is None:
        return None, 0
    return ws.data_ptr(), ws.numel() * ws.element_size()


def conv_desc(n, c, h, w, k, dtype=SB_F32, relu=False, packed=False, layout=SB_NCHW):
    return sb_conv3x3_desc(n, c, h, w, k, dtype,
                           (SB_FUSE_RELU if relu else 0) | (SB_PACKED_FILTERS if packed else 0),
                           layout)


def fc_desc(m, k_in, n_shard, dtype=SB_F32, ldx=None, ldy=None, relu=False):
    return sb_fc_desc(m, k_in, n_shard, dtype, ldx or k_in, ldy or n_shard,
                      SB_FUSE_RELU if relu else 0)


def gated_desc(m, k_in, n_shard, dtype=SB_F32, act=SB_ACT_SILU, ldx=None, ldy=None,
               unaligned=False):
    """unaligned: the workspace query includes room for x and weights at any address."""
    return sb_gated_desc(m, k_in, n_shard, dtype, act, ldx or k_in, ldy or n_shard,
                         SB_UNALIGNED if unaligned else 0)


# --------------------------------------------------------- entry points --
def sb_version():
    return load().sb_version()


def sb_conv3x3_workspace_bytes(desc, pass_):
    return load().sb_conv3x3_workspace_bytes(ctypes.byref(desc), pass_)


def sb_conv3x3_plan_string(desc, pass_):
    buf = ctypes.create_string_buffer(512)
    n = load().sb_conv3x3_plan_string(ctypes.byref(desc), pass_, buf, 512)
    if n == 0:
        raise SBError("sb_conv3x3_plan_string", SB_ERR_INVALID_ARG)
    return buf.value.decode()


def sb_conv3x3_packed_bytes(desc, pass_):
    return load().sb_conv3x3_packed_bytes(ctypes.byref(desc), pass_)


def sb_conv3x3_pack_filters(desc, pass_, w, packed, stream=None):
    _check("sb_conv3x3_pack_filters", load().sb_conv3x3_pack_filters(
        ctypes.byref(desc), pass_, _ptr(w), _ptr(packed),
        packed.numel() * packed.element_size(), _stream(stream)))


class PackList:
    """Marshalled arguments of sb_conv3x3_pack_filters_many for a fixed list
    of (desc, pass, filters, packed buffer): built once, passed to every
    call (the buffers must stay alive)."""

    def __init__(self, items):
        n = len(items)
        self.count = n
        self.descs = (sb_conv3x3_desc * n)(*[d for d, _, _, _ in items])
        self.passes = (_i * n)(*[p for _, p, _, _ in items])
        self.w = (_vp * n)(*[_ptr(w) for _, _, w, _ in items])
        self.packed = (_vp * n)(*[_ptr(o) for _, _, _, o in items])
        self.nbytes = (_sz * n)(*[o.numel() * o.element_size() for _, _, _, o in items])


def sb_conv3x3_pack_filters_many(plist, stream=None):
    _check("sb_conv3x3_pack_filters_many", load().sb_conv3x3_pack_filters_many(
        plist.count, plist.descs, plist.passes, plist.w, plist.packed, plist.nbytes,
        _stream(stream)))


def sb_conv3x3_fwd(desc, x, w, bias, y, ws=None, stream=None):
    p, nb = _ws(ws)
    _check("sb_conv3x3_fwd", load().sb_conv3x3_fwd(
        ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias), _ptr(y), p, nb, _stream(stream)))


def sb_conv3x3_fwd_pool(desc, x, w, bias, y, idx, ws=None, stream=None):
    p, nb = _ws(ws)
    _check("sb_conv3x3_fwd_pool", load().sb_conv3x3_fwd_pool(
        ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias), _ptr(y), _ptr(idx), p, nb,
        _stream(stream)))


def sb_conv3x3_bwd_data(desc, dy, w, relu_mask_src, dx, ws=None, stream=None):
    p, nb = _ws(ws)
    _check("sb_conv3x3_bwd_data", load().sb_conv3x3_bwd_data(
        ctypes.byref(desc), _ptr(dy), _ptr(w), _ptr(relu_mask_src), _ptr(dx), p, nb,
        _stream(stream)))


def sb_conv3x3_bwd_weight(desc, x, dy, dw, db, ws=None, stream=None):
    p, nb = _ws(ws)
    _check("sb_conv3x3_bwd_weight", load().sb_conv3x3_bwd_weight(
        ctypes.byref(desc), _ptr(x), _ptr(dy), _ptr(dw), _ptr(db), p, nb, _stream(stream)))


class WgradList:
    """Host arrays of a sb_conv3x3_bwd_weight_many call (kept alive with the
    object, so a recorded call can be issued again)."""

    def __init__(self, descs, x, dy, dw, db):
        n = len(descs)
        self.count = n
        self.descs = (sb_conv3x3_desc * n)(*descs)
        self.x = (_vp * n)(*[_ptr(t) for t in x])
        self.dy = (_vp * n)(*[_ptr(t) for t in dy])
        self.dw = (_vp * n)(*[_ptr(t) for t in dw])
        self.db = (_vp * n)(*[_ptr(t) for t in db])

    def workspace_bytes(self):
        return load().sb_conv3x3_bwd_weight_many_workspace_bytes(self.count, self.descs)


def sb_conv3x3_bwd_weight_many(wlist, ws=None, stream=None):
    p, nb = _ws(ws)
    _check("sb_conv3x3_bwd_weight_many", load().sb_conv3x3_bwd_weight_many(
        wlist.count, wlist.descs, wlist.x, wlist.dy, wlist.dw, wlist.db, p, nb,
        _stream(stream)))


def sb_conv3x3_bwd_weight_noalloc(desc, x, dy, dw, db, stream=None):
    _check("sb_conv3x3_bwd_weight_noalloc", load().sb_conv3x3_bwd_weight_noalloc(
        ctypes.byref(desc), _ptr(x), _ptr(dy), _ptr(dw), _ptr(db), _stream(stream)))


def sb_relu_maxpool_fwd(n, c, h, w, dtype, layout, x, y, idx, stream=None):
    _check("sb_relu_maxpool_fwd", load().sb_relu_maxpool_fwd(
        n, c, h, w, dtype, layout, _ptr(x), _ptr(y), _ptr(idx), _stream(stream)))


def sb_relu_maxpool_bwd(n, c, h, w, dtype, layout, dy, idx, dx, stream=None):
    _check("sb_relu_maxpool_bwd", load().sb_relu_maxpool_bwd(
        n, c, h, w, dtype, layout, _ptr(dy), _ptr(idx), _ptr(dx), _stream(stream)))


def sb_fc_workspace_bytes(desc, pass_):
    return load().sb_fc_workspace_bytes(ctypes.byref(desc), pass_)


def sb_fc_shard_fwd(desc, x, w_shard, b_shard, y, ws=None, stream=None):
    p, nb = _ws(ws)
    _check("sb_fc_shard_fwd", load().sb_fc_shard_fwd(
        ctypes.byref(desc), _ptr(x), _ptr(w_shard), _ptr(b_shard), _ptr(y), p, nb,
        _stream(stream)))


def sb_fc_shard_bwd(desc, x, w_shard, dy, relu_mask_src, dx_partial, dw_shard, db_shard,
                    accumulate=False, ws=None, stream=None):
    p, nb = _ws(ws)
    _check("sb_fc_shard_bwd", load().sb_fc_shard_bwd(
        ctypes.byref(desc), _ptr(x), _ptr(w_shard), _ptr(dy), _ptr(relu_mask_src),
        _ptr(dx_partial), _ptr(dw_shard), _ptr(db_shard), 1 if accumulate else 0, p, nb,
        _stream(stream)))


# ---------------------------------------------------------- gated FC shard --
def sb_gated_workspace_bytes(desc, pass_):
    return load().sb_gated_workspace_bytes(ctypes.byref(desc), pass_)


def sb_gated_shard_fwd(desc, x, w_gate, w_up, b_gate, b_up, y, pre=None, ws=None, stream=None):
    """pre: fp32 [2][m][n_shard], kept for the backward, or None."""
    p, nb = _ws(ws)
    _check("sb_gated_shard_fwd", load().sb_gated_shard_fwd(
        ctypes.byref(desc), _ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(b_gate), _ptr(b_up), _ptr(y),
        _ptr(pre), p, nb, _stream_for(w_gate, stream)))


def sb_gated_shard_bwd(desc, x, w_gate, w_up, pre, dy, dx_partial, dw_gate, dw_up, db_gate, db_up,
                       accumulate=False, ws=None, stream=None):
    p, nb = _ws(ws)
    _check("sb_gated_shard_bwd", load().sb_gated_shard_bwd(
        ctypes.byref(desc), _ptr(x), _ptr(w_gate), _ptr(w_up), _ptr(pre), _ptr(dy),
        _ptr(dx_partial), _ptr(dw_gate), _ptr(dw_up), _ptr(db_gate), _ptr(db_up),
        1 if accumulate else 0, p, nb, _stream_for(w_gate, stream)))


# ------------------------------------------------ modulo and shard layers --
# Slotted buffers: worker w's slot starts at w * stride elements; by default
# the stride is the tensor's element count divided by the number of workers
# (a contiguous [workers][...] tensor).
def modulo_desc(workers, mp, batch, features):
    return sb_modulo_desc(workers, mp, batch, features)


def shard_desc(workers, mp, rows, shard):
    return sb_shard_desc(workers, mp, rows, shard)


def _slot_stride(t, workers, stride):
    if stride is not None:
        return int(stride)
    if t is None or isinstance(t, int):
        raise ValueError("give the slot stride for a raw pointer")
    return t.numel() // workers


def sb_modulo_fwd(desc, iproc, k, local, gathered, local_stride=None, stream=None):
    _check("sb_modulo_fwd", load().sb_modulo_fwd(
        ctypes.byref(desc), int(iproc), int(k), _ptr(local),
        _slot_stride(local, desc.workers, local_stride), _ptr(gathered), _stream(stream)))


def sb_modulo_bwd(desc, iproc, k, dgathered, dlocal, dg_stride=None, dl_stride=None,
                  stream=None):
    _check("sb_modulo_bwd", load().sb_modulo_bwd(
        ctypes.byref(desc), int(iproc), int(k), _ptr(dgathered),
        _slot_stride(dgathered, desc.workers, dg_stride), _ptr(dlocal),
        _slot_stride(dlocal, desc.workers, dl_stride), _stream(stream)))


def sb_shard_fwd(desc, iproc, parts, full, parts_stride=None, stream=None):
    _check("sb_shard_fwd", load().sb_shard_fwd(
        ctypes.byref(desc), int(iproc), _ptr(parts),
        _slot_stride(parts, desc.workers, parts_stride), _ptr(full), _stream(stream)))


def sb_shard_bwd(desc, iproc, dfull, dparts, df_stride=None, dp_stride=None, stream=None):
    _check("sb_shard_bwd", load().sb_shard_bwd(
        ctypes.byref(desc), int(iproc), _ptr(dfull),
        _slot_stride(dfull, desc.workers, df_stride), _ptr(dparts),
        _slot_stride(dparts, desc.workers, dp_stride), _stream(stream)))


def sb_model_average(workers, mp, params, n=None, stride=None, stream=None):
    """params: `workers` slots of fp32 parameters (a contiguous
    [workers][...] tensor by default: n = stride = numel / workers)."""
    st = _slot_stride(params, workers, stride)
    _check("sb_model_average", load().sb_model_average(
        int(workers), int(mp), int(st if n is None else n), _ptr(params), st, _stream(stream)))


SB_MAX_REPLICAS = 64


def sb_model_average_replicas(replicas, n=None, stream=None):
    """replicas: one fp32 tensor (or device pointer) per replica; each is
    replaced by the mean of all.  n defaults to the first tensor's numel."""
    k = len(replicas)
    if n is None:
        n = replicas[0].numel()
    for t in replicas:
        if not isinstance(t, int) and (str(t.dtype) != "torch.float32" or t.numel() < n):
            raise ValueError("replicas must be fp32 tensors of at least n elements")
    ptrs = (_vp * max(k, 1))(*[_ptr(t) for t in replicas])
    _check("sb_model_average_replicas", load().sb_model_average_replicas(
        int(k), int(n), ptrs, _stream(stream)))


# --------------------------------------------------- loss and SGD update --
def sb_log_softmax_nll(m, classes, z, labels, scale, logp=None, loss=None, dz=None, ldz=None,
                       stream=None):
    """z, logp, dz: fp32 [m][ldz] (ldz defaults to classes); labels: int32 [m]."""
    _check("sb_log_softmax_nll", load().sb_log_softmax_nll(
        int(m), int(classes), int(ldz or classes), _ptr(z), _ptr(labels), float(scale),
        _ptr(logp), _ptr(loss), _ptr(dz), _stream(stream)))


class SgdList:
    """Marshalled arguments of sb_sgd_update for a fixed list of
    (parameter, gradient, scale) fp32 tensors: built once, passed to every
    call (the tensors must stay alive)."""

    def __init__(self, items):
        import torch
        n = len(items)
        if not 1 <= n <= SB_SGD_MAX_TENSORS:
            raise ValueError("1 to %d tensors per update" % SB_SGD_MAX_TENSORS)
        for w, g, _ in items:
            if w.dtype != torch.float32 or g.dtype != torch.float32 or w.numel() != g.numel():
                raise ValueError("fp32 parameter and gradient of equal size")
        self.count = n
        self.w = (_vp * n)(*[_ptr(w) for w, _, _ in items])
        self.g = (_vp * n)(*[_ptr(g) for _, g, _ in items])
        self.n = (_sz * n)(*[w.numel() for w, _, _ in items])
        self.scale = (ctypes.c_float * n)(*[float(sc) for _, _, sc in items])


def sb_sgd_update(slist, lr, stream=None):
    _check("sb_sgd_update", load().sb_sgd_update(
        slist.count, slist.w, slist.g, slist.n, slist.scale, float(lr), _stream(stream)))


# ------------------------------------------------------------------- AdamW --
class AdamwList:
    """The plan of sb_adamw_update for a fixed list of tensors, in device memory
    (sb_adamw_make_plan): built once, passed to every call (the list and its
    tensors must stay alive until the calls' kernels have run).  The plan is
    written before this returns, so that any stream may use it; a list built
    while its stream is captured is the graph's alone (while another stream is
    captured, none is built).  stream: where the plan is written, the current one
    by default.

    items: dicts of a parameter ``w``, its gradient ``g`` (fp32) and moments
    ``m`` and ``v`` (fp32; or uint8, with their references ``m_top`` and
    ``v_top``, int16, one for each SB_ADAMW_BLOCK elements), and, if wanted,
    ``copy`` (bfloat16, gets the new w), ``scale`` (of the gradient, 1),
    ``decay`` (0) and ``first`` (the number of the tensor's first element
    among the random numbers; by default the tensors follow one another).
    ``adamw_moments`` makes zero moments."""

    def __init__(self, items, stream=None):
        import torch
        n = len(items)
        if not 1 <= n <= SB_ADAMW_MAX_TENSORS:
            raise ValueError("1 to %d tensors per update" % SB_ADAMW_MAX_TENSORS)
        self.moments = 8 if items[0]["m"].dtype == torch.uint8 else 32
        kind = torch.uint8 if self.moments == 8 else torch.float32
        self.count = n
        self.tensors = (sb_adamw_tensor * n)()
        first = 0
        device = items[0]["w"].device
        for t, it in zip(self.tensors, items):
            w, g, m, v = it["w"], it["g"], it["m"], it["v"]
            if any(x is not None and x.device != device for x in
                   (w, g, m, v, it.get("copy"), it.get("m_top"), it.get("v_top"))):
                raise ValueError("the tensors of an update are on one device")
            size = w.numel()
            copy, m_top, v_top = it.get("copy"), it.get("m_top"), it.get("v_top")
            if (w.dtype != torch.float32 or g.dtype != torch.float32 or m.dtype != kind
                    or v.dtype != kind or not size == g.numel() == m.numel() == v.numel()):
                raise ValueError("fp32 parameter and gradient, moments of one type, of equal size")
            if copy is not None and (copy.dtype != torch.bfloat16 or copy.numel() != size):
                raise ValueError("the copy is bfloat16, of the parameter's size")
            if self.moments == 8:
                tops = (size + SB_ADAMW_BLOCK - 1) // SB_ADAMW_BLOCK
                for top in (m_top, v_top):
                    if top is None or top.dtype != torch.int16 or top.numel() != tops:
                        raise ValueError("int16 references, one for each %d elements"
                                         % SB_ADAMW_BLOCK)
            t.w, t.copy, t.g, t.m, t.v = _ptr(w), _ptr(copy), _ptr(g), _ptr(m), _ptr(v)
            t.m_top, t.v_top = _ptr(m_top), _ptr(v_top)
            t.first = it.get("first", first)
            t.n = size
            t.grad_scale, t.decay = it.get("scale", 1.0), it.get("decay", 0.0)
            first = t.first + size
        need = load().sb_adamw_plan_bytes(n)
        current = torch.cuda.current_stream()
        s = (current if stream is None else stream if isinstance(stream, torch.cuda.Stream)
             else torch.cuda.ExternalStream(_stream(stream)))
        other = torch.cuda.is_current_stream_capturing() and s != current
        with torch.cuda.stream(s):
            capturing = torch.cuda.is_current_stream_capturing()
            if other and not capturing:
                raise ValueError("the plan's stream is not part of the capture under way")
            # The stream's own memory: what used it before on another stream, and may
            # still be at work, could write over the plan.
            self.plan = torch.empty((need,), dtype=torch.uint8, device=device)
            self.info = sb_adamw_plan()
            _check("sb_adamw_make_plan", load().sb_adamw_make_plan(
                self.moments, n, self.tensors, _ptr(self.plan), need, ctypes.byref(self.info),
                _stream_for(self.plan, s)))
        if not capturing:
            s.synchronize()


def adamw_moments(w, moments=32):
    """Zero moments for parameter w as AdamwList takes them (a dict)."""
    import torch
    n = w.numel()
    if moments == 32:
        return {k: torch.zeros(n, dtype=torch.float32, device=w.device) for k in ("m", "v")}
    if moments != 8:
        raise ValueError("moments of 32 or 8 bits")
    tops = (n + SB_ADAMW_BLOCK - 1) // SB_ADAMW_BLOCK
    d = {k: torch.zeros(n, dtype=torch.uint8, device=w.device) for k in ("m", "v")}
    d.update({k: torch.zeros(tops, dtype=torch.int16, device=w.device) for k in ("m_top", "v_top")})
    return d


def sb_adamw_update(alist, lr, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0, steps_done=None,
                    stream=None):
    """step: the number of this update (from 1), or, with the int32 device
    counter steps_done, what is added to its value."""
    d = sb_adamw_desc(lr, beta1, beta2, eps, step, seed & 0xffffffff)
    _check("sb_adamw_update", load().sb_adamw_update(
        ctypes.byref(d), ctypes.byref(alist.info), alist.plan.data_ptr(), _counter(steps_done),
        _stream_for(alist.plan, stream)))


def _counter(t):
    if t is not None and not isinstance(t, int) and str(t.dtype) != "torch.int32":
        raise ValueError("the counter is int32")
    return _ptr(t)


def sb_adamw_advance(steps_done, stream=None):
    _check("sb_adamw_advance", load().sb_adamw_advance(
        _counter(steps_done), _stream_for(steps_done, stream)))


def sb_adamw_unpack(n, m, m_top, v, v_top, m_out, v_out, stream=None):
    """The fp32 values of n moments in bytes (either pair may be None)."""
    _check("sb_adamw_unpack", load().sb_adamw_unpack(
        int(n), _ptr(m), _ptr(m_top), _ptr(v), _ptr(v_top), _ptr(m_out), _ptr(v_out),
        _stream_for(m if m is not None else v if v is not None else 0, stream)))


# -------------------------------------------------------------- embedding --
_types = None                   # torch's types by sb_dtype, then int32


def _kinds(desc):
    """The types of a call: the descriptor's, int32, float32."""
    global _types
    if _types is None:
        import torch
        _types = (torch.float32, torch.bfloat16, torch.int32)
    return _types[desc.dtype if desc.dtype in (SB_F32, SB_BF16) else 0], _types[2], _types[0]


def _at(t, kind):
    """The address of a device tensor of that type, of None and of an address itself."""
    if t is None or t.__class__ is int:
        return t
    if t.dtype is not kind:
        raise ValueError("a tensor of %s, expected %s" % (t.dtype, kind))
    if not t.is_cuda:
        raise ValueError("libsb takes device tensors")
    if not t.is_contiguous():
        raise ValueError("libsb takes contiguous tensors (strides go in the descriptor)")
    return t.data_ptr()


def embed_desc(tokens, vocab, width, dtype=SB_F32, first=0, ldy=None, scale=1.0):
    """first: the id of the table's first row (a vocabulary shard's)."""
    return sb_embed_desc(tokens, vocab, width, first, dtype, ldy or width, scale)


def sb_embed_workspace_bytes(desc):
    return load().sb_embed_workspace_bytes(ctypes.byref(desc))


def sb_embed_fwd(desc, table, ids, y, stream=None):
    """ids: int32."""
    row, i32, _ = _kinds(desc)
    _check("sb_embed_fwd", load().sb_embed_fwd(
        ctypes.byref(desc), _at(table, row), _at(ids, i32), _at(y, row),
        _stream_for(table, stream)))


def sb_embed_bwd(desc, ids, dy, dtable, accumulate=False, ws=None, stream=None):
    """dtable: fp32 [vocab][width]."""
    p, nb = _ws(ws)
    row, i32, f32 = _kinds(desc)
    _check("sb_embed_bwd", load().sb_embed_bwd(
        ctypes.byref(desc), _at(ids, i32), _at(dy, row), _at(dtable, f32), 1 if accumulate else 0,
        p, nb, _stream_for(dtable, stream)))


# ------------------------------------------------------------ expert rows --
def expert_desc(tokens, top, experts, width, dtype=SB_F32, first=0, ldx=None, ldr=None):
    """first: the worker's first expert."""
    return sb_expert_desc(tokens, top, experts, first, width, dtype, ldx or width, ldr or width)


def sb_expert_workspace_bytes(desc):
    return load().sb_expert_workspace_bytes(ctypes.byref(desc))


def sb_expert_sort(desc, ids, place, offsets, ws=None, stream=None):
    """All int32: ids and place [tokens][top], offsets [experts + 1]."""
    p, nb = _ws(ws)
    i32 = _kinds(desc)[1]
    _check("sb_expert_sort", load().sb_expert_sort(
        ctypes.byref(desc), _at(ids, i32), _at(place, i32), _at(offsets, i32), p, nb,
        _stream_for(offsets, stream)))


def sb_expert_gather(desc, x, place, xs, stream=None):
    row, i32, _ = _kinds(desc)
    _check("sb_expert_gather", load().sb_expert_gather(
        ctypes.byref(desc), _at(x, row), _at(place, i32), _at(xs, row), _stream_for(x, stream)))


def sb_expert_combine(desc, ys, place, weights, y, add=None, stream=None):
    """weights: fp32 [tokens][top], or None (1 each: the gather's backward); add: rows
    like y's that the sum starts from, or y itself."""
    row, i32, f32 = _kinds(desc)
    _check("sb_expert_combine", load().sb_expert_combine(
        ctypes.byref(desc), _at(ys, row), _at(place, i32), _at(weights, f32), _at(add, row),
        _at(y, row), _stream_for(y, stream)))


def sb_expert_combine_bwd(desc, dy, ys, place, weights, dys, dweights=None, stream=None):
    row, i32, f32 = _kinds(desc)
    _check("sb_expert_combine_bwd", load().sb_expert_combine_bwd(
        ctypes.byref(desc), _at(dy, row), _at(ys, row), _at(place, i32), _at(weights, f32),
        _at(dys, row), _at(dweights, f32), _stream_for(dy, stream)))


# ------------------------------------------------- token log-probabilities --
def token_logp_desc(m, classes, top=0, dtype=SB_F32, ldz=None, probs=False):
    """probs: the alternatives' probabilities in place of their logarithms."""
    return sb_token_logp_desc(m, classes, ldz or classes, dtype, top, SB_TOP_PROBS if probs else 0)


def sb_token_logp_workspace_bytes(desc):
    return load().sb_token_logp_workspace_bytes(ctypes.byref(desc))


def sb_token_logp_fwd(desc, z, targets, logp, entropy, stats, top_ids=None, top_values=None,
                      ws=None, stream=None):
    """targets, top_ids: int32; logp, entropy, stats [m][2], top_values: fp32.
    targets, logp and entropy may be None."""
    p, nb = _ws(ws)
    row, i32, f32 = _kinds(desc)
    _check("sb_token_logp_fwd", load().sb_token_logp_fwd(
        ctypes.byref(desc), _at(z, row), _at(targets, i32), _at(logp, f32), _at(entropy, f32),
        _at(stats, f32), _at(top_ids, i32), _at(top_values, f32), p, nb, _stream_for(z, stream)))


def sb_token_logp_bwd(desc, z, stats, targets, dlogp, entropy, dentropy, top_ids, top_values, dtop,
                      dz, stream=None):
    """dlogp, dentropy and dtop, and what they go with, may be None; dz may be z."""
    row, i32, f32 = _kinds(desc)
    _check("sb_token_logp_bwd", load().sb_token_logp_bwd(
        ctypes.byref(desc), _at(z, row), _at(stats, f32), _at(targets, i32), _at(dlogp, f32),
        _at(entropy, f32), _at(dentropy, f32), _at(top_ids, i32), _at(top_values, f32),
        _at(dtop, f32), _at(dz, row), _stream_for(z, stream)))
