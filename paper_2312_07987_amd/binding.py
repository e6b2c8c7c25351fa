"""ctypes binding of libswitchhead.so: the same entry points as include/switchhead.h, with
argument marshalling only.  Tensors are torch tensors on the GPU (device memory and streams
are all torch is used for); every step of the layer runs inside the library's kernels.

There is no fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libswitchhead.so")

SH_OK, SH_ERR_INVALID_ARG, SH_ERR_UNSUPPORTED, SH_ERR_WORKSPACE_TOO_SMALL, SH_ERR_HIP = range(5)
SH_F32, SH_BF16 = 0, 1

STATIC_WORKSPACE_BYTES = 16 << 20

EXPORTS = ("switchhead_workspace_bytes", "switchhead_workspace_parts", "switchhead_forward", "switchhead_forward_static", "switchhead_backward",
           "switchhead_get_routing", "switchhead_get_intermediates", "switchhead_last_error",
           "switchhead_set_kernel_family", "switchhead_version",
           "switchhead_profile_enable", "switchhead_profile_read",
           "switchhead_attention_workspace_bytes", "switchhead_attention_forward", "switchhead_attention_backward",
           "switchhead_qk_norm_workspace_bytes", "switchhead_qk_norm_rope_forward", "switchhead_qk_norm_rope_backward",
           "switchhead_packed_workspace_bytes", "switchhead_forward_packed", "switchhead_backward_packed")


class sh_shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("B", "T", "d_model", "nheads", "d_head", "E", "k", "causal", "dtype", "qk_experts", "rope", "T_q")]


class _Description(ctypes.Structure):
    """`places`: what the fields say about the tensors, kept until a field changes."""

    def __setattr__(self, name, value):
        super().__setattr__(name, value)
        if name != "places":
            self.__dict__.pop("places", None)


class sh_attention(_Description):
    _fields_ = ([(n, ctypes.c_int32) for n in ("nseq", "nheads", "nkv_heads", "d_head", "causal", "dtype", "total_q", "total_k",
                                               "max_q", "max_k", "prefix")] + [("scale", ctypes.c_float)] +
                [(n, ctypes.c_int64) for n in ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head", "o_row", "o_head",
                                               "kp_row", "kp_head", "vp_row", "vp_head")])


class sh_qk_norm(_Description):
    _fields_ = ([(n, ctypes.c_int32) for n in ("tokens", "nheads", "nkv_heads", "d_head", "rope_dim", "dtype")] +
                [("eps", ctypes.c_float), ("theta", ctypes.c_float)] +
                [(n, ctypes.c_int64) for n in ("q_row", "q_head", "k_row", "k_head", "yq_row", "yq_head", "yk_row", "yk_head")])


class sh_packing(ctypes.Structure):
    _fields_ = [("nseq", ctypes.c_int32), ("max_len", ctypes.c_int32), ("offsets", ctypes.c_void_p), ("q_norm", ctypes.c_void_p),
                ("k_norm", ctypes.c_void_p), ("norm_eps", ctypes.c_float)]


class SwitchHeadError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("switchhead error %d: %s" % (code, msg))
        self.code = code


_lib = None


def lib():
    """Loads libswitchhead.so (once).  Raises if it is missing: build it first with
    `python -m paper_2312_07987_amd.build`."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            LIB_PATH + " is missing: build it with `python -m paper_2312_07987_amd.build` "
            "(there is no fallback implementation)")
    L = ctypes.CDLL(LIB_PATH)
    vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
    shp = ctypes.POINTER(sh_shape)
    L.switchhead_workspace_bytes.restype = sz
    L.switchhead_workspace_bytes.argtypes = [shp]
    L.switchhead_workspace_parts.restype = i32
    L.switchhead_workspace_parts.argtypes = [shp, ctypes.POINTER(sz), ctypes.POINTER(sz)]
    L.switchhead_forward.restype = i32
    L.switchhead_forward.argtypes = [shp] + [vp] * 10 + [vp, sz, vp]
    L.switchhead_forward_static.restype = i32
    L.switchhead_forward_static.argtypes = [shp] + [vp] * 10 + [vp]
    L.switchhead_backward.restype = i32
    L.switchhead_backward.argtypes = [shp] + [vp] * 8 + [vp, sz] + [vp] * 9 + [vp]
    L.switchhead_get_routing.restype = i32
    L.switchhead_get_routing.argtypes = [shp, vp, sz, vp, vp, vp, vp, vp]
    L.switchhead_get_intermediates.restype = i32
    L.switchhead_get_intermediates.argtypes = [shp, vp, sz, vp, vp, vp, vp, vp, vp]
    L.switchhead_last_error.restype = ctypes.c_char_p
    L.switchhead_last_error.argtypes = []
    L.switchhead_set_kernel_family.restype = i32
    L.switchhead_set_kernel_family.argtypes = [i32]
    L.switchhead_version.restype = ctypes.c_char_p
    L.switchhead_version.argtypes = []
    L.switchhead_profile_enable.restype = i32
    L.switchhead_profile_enable.argtypes = [i32]
    L.switchhead_profile_read.restype = i32
    L.switchhead_profile_read.argtypes = [ctypes.c_char_p, sz, ctypes.POINTER(ctypes.c_float),
                                          ctypes.POINTER(i32), i32]
    att, nrm = ctypes.POINTER(sh_attention), ctypes.POINTER(sh_qk_norm)
    L.switchhead_attention_workspace_bytes.restype = sz
    L.switchhead_attention_workspace_bytes.argtypes = [att, i32]
    L.switchhead_attention_forward.restype = i32
    L.switchhead_attention_forward.argtypes = [att] + [vp] * 12 + [sz, vp]
    L.switchhead_attention_backward.restype = i32
    L.switchhead_attention_backward.argtypes = [att] + [vp] * 14 + [sz, vp]
    L.switchhead_qk_norm_workspace_bytes.restype = sz
    L.switchhead_qk_norm_workspace_bytes.argtypes = [nrm]
    L.switchhead_qk_norm_rope_forward.restype = i32
    L.switchhead_qk_norm_rope_forward.argtypes = [nrm] + [vp] * 7 + [vp]
    L.switchhead_qk_norm_rope_backward.restype = i32
    L.switchhead_qk_norm_rope_backward.argtypes = [nrm] + [vp] * 12 + [sz, vp]
    pkg = ctypes.POINTER(sh_packing)
    L.switchhead_packed_workspace_bytes.restype = sz
    L.switchhead_packed_workspace_bytes.argtypes = [shp, pkg]
    L.switchhead_forward_packed.restype = i32
    L.switchhead_forward_packed.argtypes = [shp, pkg] + [vp] * 10 + [vp, sz, vp]
    L.switchhead_backward_packed.restype = i32
    L.switchhead_backward_packed.argtypes = [shp, pkg] + [vp] * 8 + [vp, sz] + [vp] * 11 + [vp]
    _lib = L
    return L


def make_shape(B, T, d_model, nheads, d_head, E, k, causal=1, dtype="bf16", qk_experts=0, rope=0, T_q=0):
    code = {"f32": SH_F32, "fp32": SH_F32, "bf16": SH_BF16}[dtype] if isinstance(dtype, str) else int(dtype)
    return sh_shape(B, T, d_model, nheads, d_head, E, k, int(causal), code, int(qk_experts), int(rope), int(T_q))


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(stream):
    if stream is None:
        import torch
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    return ctypes.c_void_p(int(stream))


def _check(code):
    if code != SH_OK:
        raise SwitchHeadError(code, lib().switchhead_last_error().decode())


def switchhead_workspace_bytes(shape):
    return int(lib().switchhead_workspace_bytes(ctypes.byref(shape)))


def switchhead_workspace_parts(shape):
    """(kept bytes, scratch bytes) of the workspace of this shape."""
    kept, scratch = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().switchhead_workspace_parts(ctypes.byref(shape), ctypes.byref(kept), ctypes.byref(scratch)))
    return int(kept.value), int(scratch.value)


def switchhead_last_error():
    return lib().switchhead_last_error().decode()


def switchhead_set_kernel_family(family):
    return int(lib().switchhead_set_kernel_family(int(family)))


def switchhead_version():
    return lib().switchhead_version().decode()


def switchhead_forward(shape, x, W_Q, W_K, W_V, W_O, W_S, W_D, b_S, b_D, y, workspace, stream=None):
    _check(lib().switchhead_forward(ctypes.byref(shape), _ptr(x), _ptr(W_Q), _ptr(W_K), _ptr(W_V), _ptr(W_O),
                                    _ptr(W_S), _ptr(W_D), _ptr(b_S), _ptr(b_D), _ptr(y),
                                    _ptr(workspace), workspace.numel() * workspace.element_size(),
                                    _stream(stream)))


def switchhead_forward_static(shape, x, W_Q, W_K, W_V, W_O, W_S, W_D, b_S, b_D, y, stream=None):
    _check(lib().switchhead_forward_static(ctypes.byref(shape), _ptr(x), _ptr(W_Q), _ptr(W_K), _ptr(W_V), _ptr(W_O),
                                           _ptr(W_S), _ptr(W_D), _ptr(b_S), _ptr(b_D), _ptr(y), _stream(stream)))


def switchhead_backward(shape, x, W_Q, W_K, W_V, W_O, W_S, W_D, dy, workspace,
                        dx, dW_Q, dW_K, dW_V, dW_O, dW_S, dW_D, db_S, db_D, stream=None):
    _check(lib().switchhead_backward(ctypes.byref(shape), _ptr(x), _ptr(W_Q), _ptr(W_K), _ptr(W_V), _ptr(W_O),
                                     _ptr(W_S), _ptr(W_D), _ptr(dy),
                                     _ptr(workspace), workspace.numel() * workspace.element_size(),
                                     _ptr(dx), _ptr(dW_Q), _ptr(dW_K), _ptr(dW_V), _ptr(dW_O),
                                     _ptr(dW_S), _ptr(dW_D), _ptr(db_S), _ptr(db_D), _stream(stream)))


def switchhead_get_routing(shape, workspace, topk_idx, gate, perm, expert_offsets, stream=None):
    _check(lib().switchhead_get_routing(ctypes.byref(shape), _ptr(workspace),
                                        workspace.numel() * workspace.element_size(),
                                        _ptr(topk_idx), _ptr(gate), _ptr(perm), _ptr(expert_offsets),
                                        _stream(stream)))


def switchhead_get_intermediates(shape, workspace, Q, K, V, ctx, lse, stream=None):
    _check(lib().switchhead_get_intermediates(ctypes.byref(shape), _ptr(workspace),
                                              workspace.numel() * workspace.element_size(),
                                              _ptr(Q), _ptr(K), _ptr(V), _ptr(ctx), _ptr(lse), _stream(stream)))


def switchhead_profile_enable(on):
    _check(lib().switchhead_profile_enable(int(bool(on))))


def switchhead_profile_read(max_entries=64):
    """Returns {step label: (total milliseconds, occurrences)} since the last read."""
    buf = ctypes.create_string_buffer(64 * max_entries)
    ms = (ctypes.c_float * max_entries)()
    cnt = (ctypes.c_int32 * max_entries)()
    n = lib().switchhead_profile_read(buf, len(buf), ms, cnt, max_entries)
    names = buf.value.decode().split("\n")[:n]
    return {names[i]: (float(ms[i]), int(cnt[i])) for i in range(n)}


# ---- operators beside the layer ---------------------------------------------------------------------------------------------
# These calls compare every tensor with the description and the types that the library reads it by: a gradient with other strides than its
# tensor's (torch.empty_like of a view of a fused projection is dense), 64-bit offsets (torch.cumsum's result) or a tensor on another device would otherwise be read, or
# written past its end, as what it is not.
def _addr(t):
    return None if t is None else t.data_ptr()


_torch = None


def _import_torch():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


def _launch(fn, device, stream, *args):
    """Calls fn(*args, stream) with GPU `device` current (-1: the tensors are in host memory): its current stream where none is given."""
    if device < 0:
        raise SwitchHeadError(SH_ERR_INVALID_ARG, "the tensors must be on a GPU")
    if device != _torch._C._cuda_getDevice():
        with _torch.cuda.device(device):
            return _check(fn(*args, _torch.cuda.current_stream().cuda_stream if stream is None else int(stream)))
    code = fn(*args, _torch._C._cuda_getCurrentRawStream(device) if stream is None else int(stream))
    if code != SH_OK:
        _check(code)


def _refuse(text, *args):
    raise SwitchHeadError(SH_ERR_INVALID_ARG, text % args)


def _dtype_code(t):
    torch = _import_torch()
    codes = {torch.float32: SH_F32, torch.bfloat16: SH_BF16}
    if t.dtype not in codes:
        _refuse("tensors are float32 or bfloat16, not %s", t.dtype)
    return codes[t.dtype]


def _rows(name, t, like=None, heads=None):
    """Row and head stride of a [rows, heads, d_head] tensor, its rows' elements next to each other."""
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        _refuse("%s must be [rows, heads, d_head] with the elements of a head next to each other", name)
    if like is not None and (t.dtype != like.dtype or t.device != like.device or t.shape[2] != like.shape[2]):
        _refuse("%s has another type, device or head width", name)
    if heads is not None and t.shape[1] != heads:
        _refuse("%s has %d heads, not %d", name, t.shape[1], heads)
    rows, head = t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2], t.stride(1) if t.shape[1] > 1 else t.shape[2]
    if rows == 0 or head == 0:
        _refuse("%s is broadcast along its rows or heads", name)
    return rows, head


def _place(rows, heads, d, row, head):
    """Shape and strides that a description means by these fields."""
    head = head or d
    return (rows, heads, d), (row or heads * head, head, 1)


def _attention_places(a):
    """Shapes and strides of Q, K, V, O and the prefix, the storage type."""
    try:
        return a.places
    except AttributeError:
        pass
    torch = _import_torch()
    q, k, d = (a.total_q, a.nheads), (a.total_k, a.nkv_heads), a.d_head
    a.places = (_place(*q, d, a.q_row, a.q_head), _place(*k, d, a.k_row, a.k_head), _place(*k, d, a.v_row, a.v_head), _place(*q, d, a.o_row, a.o_head),
                _place(a.prefix, a.nkv_heads, d, a.kp_row, a.kp_head), _place(a.prefix, a.nkv_heads, d, a.vp_row, a.vp_head),
                torch.bfloat16 if a.dtype == SH_BF16 else torch.float32)
    return a.places


def _norm_places(a):
    try:
        return a.places
    except AttributeError:
        pass
    torch = _import_torch()
    n, H, Hk, d = a.tokens, a.nheads, a.nkv_heads, a.d_head
    a.places = (_place(n, H, d, a.q_row, a.q_head), _place(n, Hk, d, a.k_row, a.k_head), _place(n, H, d, a.yq_row, a.yq_head), _place(n, Hk, d, a.yk_row, a.yk_head),
                torch.bfloat16 if a.dtype == SH_BF16 else torch.float32)
    return a.places


def _lies(name, t, place, dtype, device):
    """t lies as the description says (strides along one row or one head mean nothing)."""
    shape, stride = place
    if t is None:   # (a tensor without rows may be missing)
        if shape[0]:
            _refuse("%s is missing", name)
        return
    if t.shape == shape and t.stride() == stride and t.dtype is dtype and t.get_device() == device:
        return
    if tuple(t.shape) != shape or t.dtype != dtype:
        _refuse("%s is %s %s, the description says %s %s", name, tuple(t.shape), t.dtype, shape, dtype)
    if t.get_device() != device:
        _refuse("%s is on another device", name)
    if 0 not in shape and any(n > 1 and a != b for n, a, b in zip(shape, t.stride(), stride)):
        _refuse("%s has strides %s, the description says %s", name, t.stride(), stride)


def _dense(name, t, dtype, least, device):
    """t holds at least `least` elements of this type without gaps, or is None (the library refuses that where it must not be)."""
    if t is None:
        return
    if t.dtype is not dtype or t.numel() < least or not t.is_contiguous() or t.get_device() != device:
        _refuse("%s must be at least %d elements of %s without gaps on the tensors' device, not %s %s%s", name, least, dtype, tuple(t.shape), t.dtype,
                "" if t.is_contiguous() else " with gaps")


def _workspace(t, device):
    if not t.is_contiguous() or t.get_device() != device:
        _refuse("the workspace must be without gaps and on the tensors' device")
    return t.data_ptr(), t.numel() * t.element_size()


def _lengths(a, device, q_offsets, q_lengths, k_offsets, k_lengths):
    i32 = _torch.int32
    _dense("q_offsets", q_offsets, i32, a.nseq + 1, device)
    if k_offsets is not q_offsets:
        _dense("k_offsets", k_offsets, i32, a.nseq + 1, device)
    _dense("q_lengths", q_lengths, i32, a.nseq, device)
    _dense("k_lengths", k_lengths, i32, a.nseq, device)
    return _addr(q_offsets), _addr(q_lengths), _addr(k_offsets), _addr(k_lengths)


def make_attention(Q, K, V, O, nseq, max_q, max_k, causal=1, K_prefix=None, V_prefix=None, scale=0.0):
    """The description of attention over these tensors: Q, O [total_q, nheads, d_head], K, V [total_k, nkv_heads, d_head], strided as they
    are (views of a fused projection, slices of a cache).  Valid for any tensors of the same shapes and strides; gradients have the strides of their tensors."""
    q, k, v, o = _rows("Q", Q), _rows("K", K, Q), _rows("V", V, Q, K.shape[1]), _rows("O", O, Q, Q.shape[1])
    if V.shape[0] != K.shape[0] or O.shape[0] != Q.shape[0]:
        _refuse("K and V, and Q and O, must have the same number of rows")
    if (K_prefix is None) != (V_prefix is None):
        _refuse("K_prefix and V_prefix come together")
    prefix, kp, vp = 0, (0, 0), (0, 0)
    if K_prefix is not None:
        kp, vp, prefix = _rows("K_prefix", K_prefix, Q, K.shape[1]), _rows("V_prefix", V_prefix, Q, K.shape[1]), K_prefix.shape[0]
        if V_prefix.shape[0] != prefix:
            _refuse("K_prefix and V_prefix must have the same number of rows")
    a = sh_attention(nseq, Q.shape[1], K.shape[1], Q.shape[2], int(causal), _dtype_code(Q), Q.shape[0], K.shape[0], max_q, max_k, prefix,
                     scale, *q, *k, *v, *o, *kp, *vp)
    return a


def switchhead_attention_workspace_bytes(attention, backward=False):
    return int(lib().switchhead_attention_workspace_bytes(attention, int(backward)))


def switchhead_attention_forward(attention, Q, K, V, q_offsets, k_offsets, O, lse, workspace, q_lengths=None, k_lengths=None,
                                 K_prefix=None, V_prefix=None, stream=None):
    q, k, v, o, kp, vp, dtype = _attention_places(attention)
    device = Q.get_device()
    _lies("Q", Q, q, dtype, device)
    _lies("K", K, k, dtype, device)
    _lies("V", V, v, dtype, device)
    _lies("O", O, o, dtype, device)
    if attention.prefix:
        _lies("K_prefix", K_prefix, kp, dtype, device)
        _lies("V_prefix", V_prefix, vp, dtype, device)
    _dense("lse", lse, _torch.float32, attention.nheads * attention.total_q, device)
    lengths = _lengths(attention, device, q_offsets, q_lengths, k_offsets, k_lengths)
    _launch(lib().switchhead_attention_forward, device, stream, attention, _addr(Q), _addr(K), _addr(V), _addr(K_prefix), _addr(V_prefix),
            *lengths, _addr(O), _addr(lse), *_workspace(workspace, device))


def switchhead_attention_backward(attention, Q, K, V, O, dO, lse, q_offsets, k_offsets, dQ, dK, dV, workspace, q_lengths=None,
                                  k_lengths=None, stream=None):
    q, k, v, o, _, _, dtype = _attention_places(attention)
    device = Q.get_device()
    for name, t, place in (("Q", Q, q), ("K", K, k), ("V", V, v), ("O", O, o), ("dO", dO, o), ("dQ", dQ, q), ("dK", dK, k), ("dV", dV, v)):
        _lies(name, t, place, dtype, device)
    _dense("lse", lse, _torch.float32, attention.nheads * attention.total_q, device)
    lengths = _lengths(attention, device, q_offsets, q_lengths, k_offsets, k_lengths)
    _launch(lib().switchhead_attention_backward, device, stream, attention, _addr(Q), _addr(K), _addr(V), _addr(O), _addr(dO),
            _addr(lse), *lengths, _addr(dQ), _addr(dK), _addr(dV), *_workspace(workspace, device))


def make_qk_norm(Q, K, Y_Q, Y_K, rope_dim, eps=1e-6, theta=0.0):
    """The description of norms and rotation of these tensors, [tokens, heads, d_head] each; K and Y_K may be None.  Valid for any tensors of the same
    shapes and strides; gradients have the strides of their tensors."""
    q, yq = _rows("Q", Q), _rows("Y_Q", Y_Q, Q, Q.shape[1])
    if Y_Q.shape[0] != Q.shape[0] or (K is None) != (Y_K is None) or (K is not None and (K.shape[0] != Q.shape[0] or Y_K.shape[0] != Q.shape[0])):
        _refuse("Q, K and the outputs must have the same number of rows")
    k, yk, kv = (0, 0), (0, 0), 0
    if K is not None:
        k, yk, kv = _rows("K", K, Q), _rows("Y_K", Y_K, Q, K.shape[1]), K.shape[1]
    a = sh_qk_norm(Q.shape[0], Q.shape[1], kv, Q.shape[2], rope_dim, _dtype_code(Q), eps, theta, *q, *k, *yq, *yk)
    return a


def switchhead_qk_norm_workspace_bytes(norm):
    return int(lib().switchhead_qk_norm_workspace_bytes(norm))


def _norm_inputs(norm, Q, K, w_Q, w_K, positions, q, k, dtype, device):
    _lies("Q", Q, q, dtype, device)
    if norm.nkv_heads:
        _lies("K", K, k, dtype, device)
    _dense("w_Q", w_Q, dtype, norm.d_head, device)
    _dense("w_K", w_K, dtype, norm.d_head, device)
    _dense("positions", positions, _torch.int32, norm.tokens, device)


def switchhead_qk_norm_rope_forward(norm, Q, K, w_Q, w_K, positions, Y_Q, Y_K, stream=None):
    q, k, yq, yk, dtype = _norm_places(norm)
    device = Q.get_device()
    _norm_inputs(norm, Q, K, w_Q, w_K, positions, q, k, dtype, device)
    _lies("Y_Q", Y_Q, yq, dtype, device)
    if norm.nkv_heads:
        _lies("Y_K", Y_K, yk, dtype, device)
    _launch(lib().switchhead_qk_norm_rope_forward, device, stream, norm, _addr(Q), _addr(K), _addr(w_Q), _addr(w_K), _addr(positions),
            _addr(Y_Q), _addr(Y_K))


def switchhead_qk_norm_rope_backward(norm, Q, K, w_Q, w_K, positions, dY_Q, dY_K, dQ, dK, dw_Q, dw_K, workspace, stream=None):
    q, k, yq, yk, dtype = _norm_places(norm)
    device = Q.get_device()
    _norm_inputs(norm, Q, K, w_Q, w_K, positions, q, k, dtype, device)
    _lies("dY_Q", dY_Q, yq, dtype, device)
    _lies("dQ", dQ, q, dtype, device)
    if norm.nkv_heads:
        _lies("dY_K", dY_K, yk, dtype, device)
        _lies("dK", dK, k, dtype, device)
    _dense("dw_Q", dw_Q, _torch.float32, norm.d_head, device)
    _dense("dw_K", dw_K, _torch.float32, norm.d_head, device)
    _launch(lib().switchhead_qk_norm_rope_backward, device, stream, norm, _addr(Q), _addr(K), _addr(w_Q), _addr(w_K), _addr(positions),
            _addr(dY_Q), _addr(dY_K), _addr(dQ), _addr(dK), _addr(dw_Q), _addr(dw_K), *_workspace(workspace, device))


def make_packing(offsets, max_len, q_norm=None, k_norm=None, norm_eps=1e-6):
    """Packed sequences of a layer call: offsets int32 [nseq + 1] on the GPU, weights of the norms or None (all kept alive by the packing)."""
    _dense("offsets", offsets, _import_torch().int32, 2, offsets.get_device())
    p = sh_packing(offsets.numel() - 1, max_len, _addr(offsets), _addr(q_norm), _addr(k_norm), norm_eps)
    p.tensors = (offsets, q_norm, k_norm)
    return p


def _packing_fits(packing, shape, x, *gradients):
    torch, device = _import_torch(), x.get_device()
    offsets, q_norm, k_norm = getattr(packing, "tensors", (None, None, None))
    _dense("offsets", offsets, torch.int32, packing.nseq + 1, device)
    for t in (q_norm, k_norm):
        _dense("a norm's weights", t, torch.bfloat16 if shape.dtype == SH_BF16 else torch.float32, shape.d_head, device)
    for t in gradients:
        _dense("a norm's gradient", t, torch.float32, shape.d_head, device)
    return device


def switchhead_packed_workspace_bytes(shape, packing):
    return int(lib().switchhead_packed_workspace_bytes(shape, packing))


def switchhead_forward_packed(shape, packing, x, W_Q, W_K, W_V, W_O, W_S, W_D, b_S, b_D, y, workspace, stream=None):
    device = _packing_fits(packing, shape, x)
    _launch(lib().switchhead_forward_packed, device, stream, shape, packing, _addr(x), _addr(W_Q), _addr(W_K), _addr(W_V), _addr(W_O),
            _addr(W_S), _addr(W_D), _addr(b_S), _addr(b_D), _addr(y), *_workspace(workspace, device))


def switchhead_backward_packed(shape, packing, x, W_Q, W_K, W_V, W_O, W_S, W_D, dy, workspace, dx, dW_Q, dW_K, dW_V, dW_O, dW_S, dW_D, db_S, db_D,
                               dq_norm=None, dk_norm=None, stream=None):
    device = _packing_fits(packing, shape, x, dq_norm, dk_norm)
    _launch(lib().switchhead_backward_packed, device, stream, shape, packing, _addr(x), _addr(W_Q), _addr(W_K), _addr(W_V), _addr(W_O),
            _addr(W_S), _addr(W_D), _addr(dy), *_workspace(workspace, device), _addr(dx), _addr(dW_Q),
            _addr(dW_K), _addr(dW_V), _addr(dW_O), _addr(dW_S), _addr(dW_D), _addr(db_S), _addr(db_D), _addr(dq_norm), _addr(dk_norm))
