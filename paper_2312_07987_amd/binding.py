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


class sh_attention(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("nseq", "nheads", "nkv_heads", "d_head", "causal", "dtype", "total_q", "total_k",
                                               "max_q", "max_k", "prefix")] + [("scale", ctypes.c_float)] +
                [(n, ctypes.c_int64) for n in ("q_row", "q_head", "k_row", "k_head", "v_row", "v_head", "o_row", "o_head",
                                               "kp_row", "kp_head", "vp_row", "vp_head")])


class sh_qk_norm(ctypes.Structure):
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
def _addr(t):
    return None if t is None else t.data_ptr()


_torch = None


def _launch(fn, device, stream, *args):
    """Calls fn(*args, stream) with `device` current: its current stream where none is given."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    cuda = _torch.cuda
    if device.type != "cuda":
        raise SwitchHeadError(SH_ERR_INVALID_ARG, "the tensors must be on a GPU")
    here = cuda.current_device()
    if device.index is not None and device.index != here:
        with cuda.device(device):
            return _check(fn(*args, cuda.current_stream().cuda_stream if stream is None else int(stream)))
    if stream is None:
        stream = _torch._C._cuda_getCurrentRawStream(here)
    code = fn(*args, int(stream))
    if code != SH_OK:
        _check(code)


def _dtype_code(t):
    import torch
    codes = {torch.float32: SH_F32, torch.bfloat16: SH_BF16}
    if t.dtype not in codes:
        raise SwitchHeadError(SH_ERR_INVALID_ARG, "tensors are float32 or bfloat16, not %s" % t.dtype)
    return codes[t.dtype]


def _rows(name, t, like=None, heads=None):
    """Row and head stride of a [rows, heads, d_head] tensor, its rows' elements next to each other."""
    if t.dim() != 3 or (t.shape[2] > 1 and t.stride(2) != 1):
        raise SwitchHeadError(SH_ERR_INVALID_ARG, "%s must be [rows, heads, d_head] with the elements of a head next to each other" % name)
    if like is not None and (t.dtype != like.dtype or t.device != like.device or t.shape[2] != like.shape[2]):
        raise SwitchHeadError(SH_ERR_INVALID_ARG, "%s has another type, device or head width" % name)
    if heads is not None and t.shape[1] != heads:
        raise SwitchHeadError(SH_ERR_INVALID_ARG, "%s has %d heads, not %d" % (name, t.shape[1], heads))
    rows, head = t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2], t.stride(1) if t.shape[1] > 1 else t.shape[2]
    if rows == 0 or head == 0:
        raise SwitchHeadError(SH_ERR_INVALID_ARG, "%s is broadcast along its rows or heads" % name)
    return rows, head


def make_attention(Q, K, V, O, nseq, max_q, max_k, causal=1, K_prefix=None, V_prefix=None, scale=0.0):
    """The description of attention over these tensors: Q, O [total_q, nheads, d_head], K, V [total_k, nkv_heads, d_head], strided as they
    are (views of a fused projection, slices of a cache).  Valid for any tensors of the same shapes and strides."""
    q, k, v, o = _rows("Q", Q), _rows("K", K, Q), _rows("V", V, Q, K.shape[1]), _rows("O", O, Q, Q.shape[1])
    if V.shape[0] != K.shape[0] or O.shape[0] != Q.shape[0]:
        raise SwitchHeadError(SH_ERR_INVALID_ARG, "K and V, and Q and O, must have the same number of rows")
    if (K_prefix is None) != (V_prefix is None):
        raise SwitchHeadError(SH_ERR_INVALID_ARG, "K_prefix and V_prefix come together")
    prefix, kp, vp = 0, (0, 0), (0, 0)
    if K_prefix is not None:
        kp, vp, prefix = _rows("K_prefix", K_prefix, Q, K.shape[1]), _rows("V_prefix", V_prefix, Q, K.shape[1]), K_prefix.shape[0]
        if V_prefix.shape[0] != prefix:
            raise SwitchHeadError(SH_ERR_INVALID_ARG, "K_prefix and V_prefix must have the same number of rows")
    return sh_attention(nseq, Q.shape[1], K.shape[1], Q.shape[2], int(causal), _dtype_code(Q), Q.shape[0], K.shape[0], max_q, max_k, prefix,
                        scale, *q, *k, *v, *o, *kp, *vp)


def switchhead_attention_workspace_bytes(attention, backward=False):
    return int(lib().switchhead_attention_workspace_bytes(attention, int(backward)))


def switchhead_attention_forward(attention, Q, K, V, q_offsets, k_offsets, O, lse, workspace, q_lengths=None, k_lengths=None,
                                 K_prefix=None, V_prefix=None, stream=None):
    _launch(lib().switchhead_attention_forward, Q.device, stream, attention, _addr(Q), _addr(K), _addr(V), _addr(K_prefix), _addr(V_prefix),
            _addr(q_offsets), _addr(q_lengths), _addr(k_offsets), _addr(k_lengths), _addr(O), _addr(lse),
            _addr(workspace), workspace.numel() * workspace.element_size())


def switchhead_attention_backward(attention, Q, K, V, O, dO, lse, q_offsets, k_offsets, dQ, dK, dV, workspace, q_lengths=None,
                                  k_lengths=None, stream=None):
    _launch(lib().switchhead_attention_backward, Q.device, stream, attention, _addr(Q), _addr(K), _addr(V), _addr(O), _addr(dO), _addr(lse),
            _addr(q_offsets), _addr(q_lengths), _addr(k_offsets), _addr(k_lengths), _addr(dQ), _addr(dK), _addr(dV),
            _addr(workspace), workspace.numel() * workspace.element_size())


def make_qk_norm(Q, K, Y_Q, Y_K, rope_dim, eps=1e-6, theta=0.0):
    """The description of norms and rotation of these tensors, [tokens, heads, d_head] each; K and Y_K may be None."""
    q, yq = _rows("Q", Q), _rows("Y_Q", Y_Q, Q, Q.shape[1])
    if Y_Q.shape[0] != Q.shape[0] or (K is None) != (Y_K is None) or (K is not None and (K.shape[0] != Q.shape[0] or Y_K.shape[0] != Q.shape[0])):
        raise SwitchHeadError(SH_ERR_INVALID_ARG, "Q, K and the outputs must have the same number of rows")
    k, yk, kv = (0, 0), (0, 0), 0
    if K is not None:
        k, yk, kv = _rows("K", K, Q), _rows("Y_K", Y_K, Q, K.shape[1]), K.shape[1]
    return sh_qk_norm(Q.shape[0], Q.shape[1], kv, Q.shape[2], rope_dim, _dtype_code(Q), eps, theta, *q, *k, *yq, *yk)


def switchhead_qk_norm_workspace_bytes(norm):
    return int(lib().switchhead_qk_norm_workspace_bytes(norm))


def switchhead_qk_norm_rope_forward(norm, Q, K, w_Q, w_K, positions, Y_Q, Y_K, stream=None):
    _launch(lib().switchhead_qk_norm_rope_forward, Q.device, stream, norm, _addr(Q), _addr(K), _addr(w_Q), _addr(w_K), _addr(positions),
            _addr(Y_Q), _addr(Y_K))


def switchhead_qk_norm_rope_backward(norm, Q, K, w_Q, w_K, positions, dY_Q, dY_K, dQ, dK, dw_Q, dw_K, workspace, stream=None):
    _launch(lib().switchhead_qk_norm_rope_backward, Q.device, stream, norm, _addr(Q), _addr(K), _addr(w_Q), _addr(w_K), _addr(positions),
            _addr(dY_Q), _addr(dY_K), _addr(dQ), _addr(dK), _addr(dw_Q), _addr(dw_K),
            _addr(workspace), workspace.numel() * workspace.element_size())


def make_packing(offsets, max_len, q_norm=None, k_norm=None, norm_eps=1e-6):
    """Packed sequences of a layer call: offsets int32 [nseq + 1] on the GPU (kept alive by the packing), weights of the norms or None."""
    p = sh_packing(offsets.numel() - 1, max_len, _addr(offsets), _addr(q_norm), _addr(k_norm), norm_eps)
    p.tensors = (offsets, q_norm, k_norm)
    return p


def switchhead_packed_workspace_bytes(shape, packing):
    return int(lib().switchhead_packed_workspace_bytes(shape, packing))


def switchhead_forward_packed(shape, packing, x, W_Q, W_K, W_V, W_O, W_S, W_D, b_S, b_D, y, workspace, stream=None):
    _launch(lib().switchhead_forward_packed, x.device, stream, shape, packing, _addr(x), _addr(W_Q), _addr(W_K), _addr(W_V), _addr(W_O),
            _addr(W_S), _addr(W_D), _addr(b_S), _addr(b_D), _addr(y), _addr(workspace), workspace.numel() * workspace.element_size())


def switchhead_backward_packed(shape, packing, x, W_Q, W_K, W_V, W_O, W_S, W_D, dy, workspace, dx, dW_Q, dW_K, dW_V, dW_O, dW_S, dW_D, db_S, db_D,
                               dq_norm=None, dk_norm=None, stream=None):
    _launch(lib().switchhead_backward_packed, x.device, stream, shape, packing, _addr(x), _addr(W_Q), _addr(W_K), _addr(W_V), _addr(W_O),
            _addr(W_S), _addr(W_D), _addr(dy), _addr(workspace), workspace.numel() * workspace.element_size(), _addr(dx), _addr(dW_Q),
            _addr(dW_K), _addr(dW_V), _addr(dW_O), _addr(dW_S), _addr(dW_D), _addr(db_S), _addr(db_D), _addr(dq_norm), _addr(dk_norm))
