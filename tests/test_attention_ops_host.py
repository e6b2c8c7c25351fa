"""Argument checks of the attention and norm operators: every refusal comes before anything is launched, so none of this needs a GPU
(made-up addresses stand for device memory)."""
import ctypes

import pytest

from paper_2312_07987_amd import binding as b

P = 0x10000   # an address that is never read


def lib():
    return b.lib()


def attention(**over):
    f = dict(nseq=3, nheads=4, nkv_heads=2, d_head=64, causal=1, dtype=b.SH_BF16, total_q=100, total_k=200, max_q=50, max_k=80, prefix=0, scale=0.0)
    f.update(over)
    return b.sh_attention(**f)


def forward(a, ws=1 << 40, **over):
    p = dict(Q=P, K=P, V=P, KP=None, VP=None, qo=P, ql=None, ko=P, kl=None, O=P, lse=P, workspace=P)
    p.update(over)
    return lib().switchhead_attention_forward(ctypes.byref(a), *p.values(), ws, None)


def backward(a, ws=1 << 40, **over):
    p = dict(Q=P, K=P, V=P, O=P, dO=P, lse=P, qo=P, ql=None, ko=P, kl=None, dQ=P, dK=P, dV=P, workspace=P)
    p.update(over)
    return lib().switchhead_attention_backward(ctypes.byref(a), *p.values(), ws, None)


INVALID = [dict(nseq=-1), dict(total_q=-1), dict(total_k=-5), dict(max_q=-1), dict(max_k=-1), dict(prefix=-1), dict(nheads=0), dict(nkv_heads=0), dict(d_head=0),
           dict(nkv_heads=3), dict(causal=2), dict(dtype=7), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
           dict(o_row=10, o_head=64), dict(o_row=256, o_head=32)]
UNSUPPORTED = [dict(d_head=257), dict(nheads=5000, nkv_heads=1), dict(q_row=-4), dict(k_head=-1), dict(v_row=1 << 23), dict(total_q=1 << 30, nheads=4),
               dict(total_k=1 << 30, nheads=8, nkv_heads=2), dict(nseq=1 << 24)]


@pytest.mark.parametrize("over", INVALID + UNSUPPORTED, ids=str)
def test_descriptions_that_are_refused(over):
    a = attention(**over)
    code = b.SH_ERR_INVALID_ARG if over in INVALID else b.SH_ERR_UNSUPPORTED
    assert b.switchhead_attention_workspace_bytes(a) == 0 and b.switchhead_last_error()
    assert forward(a) == code and backward(a) == code


@pytest.mark.parametrize("name", ["Q", "K", "V", "qo", "ko", "O", "workspace"])
def test_forward_without_a_tensor(name):
    assert forward(attention(), **{name: None}) == b.SH_ERR_INVALID_ARG


@pytest.mark.parametrize("name", ["Q", "K", "V", "O", "dO", "lse", "qo", "ko", "dQ", "dK", "dV", "workspace"])
def test_backward_without_a_tensor(name):
    assert backward(attention(), **{name: None}) == b.SH_ERR_INVALID_ARG


def test_addresses_and_workspace():
    a = attention()
    assert forward(a, Q=P + 1) == b.SH_ERR_INVALID_ARG and forward(a, qo=P + 2) == b.SH_ERR_INVALID_ARG and forward(a, lse=P + 2) == b.SH_ERR_INVALID_ARG
    assert backward(a, dK=P + 1) == b.SH_ERR_INVALID_ARG
    assert forward(a, workspace=P + 128) == b.SH_ERR_INVALID_ARG
    assert forward(a, ws=b.switchhead_attention_workspace_bytes(a) - 1) == b.SH_ERR_WORKSPACE_TOO_SMALL
    assert backward(a, ws=b.switchhead_attention_workspace_bytes(a, True) - 1) == b.SH_ERR_WORKSPACE_TOO_SMALL
    f32 = attention(dtype=b.SH_F32)
    assert forward(f32, Q=P + 2) == b.SH_ERR_INVALID_ARG


def test_prefix():
    a = attention(prefix=10)
    assert forward(a) == b.SH_ERR_INVALID_ARG and forward(a, KP=P) == b.SH_ERR_INVALID_ARG
    assert backward(a) == b.SH_ERR_UNSUPPORTED


def test_gradients_need_rows_of_their_own():
    # keys that lie over each other can be read, but their gradient cannot be written
    a = attention(k_row=64, k_head=64)
    assert b.switchhead_attention_workspace_bytes(a) > 0
    assert backward(a) == b.SH_ERR_INVALID_ARG


def test_nothing_to_do_is_no_error():
    for over in (dict(nseq=0), dict(total_q=0, max_q=0), dict(max_q=0)):
        assert forward(attention(**over)) == b.SH_OK
    assert forward(attention(total_q=0), Q=None, O=None) == b.SH_OK
    assert backward(attention(nseq=0)) == b.SH_OK and backward(attention(total_q=0, total_k=0), Q=None, K=None, V=None, O=None, dO=None, lse=None, dQ=None, dK=None, dV=None) == b.SH_OK


@pytest.mark.parametrize("over", [dict(nseq=1 << 23, nheads=4096, nkv_heads=4096), dict(nseq=1 << 23, nheads=4096, nkv_heads=4096, max_q=1),
                                  dict(nheads=64, nkv_heads=64, total_q=1 << 20, max_q=1 << 20)], ids=str)
def test_grids_that_no_launch_holds(over):
    """Sizes whose work-groups pass 2^32 threads are refused, not cut."""
    a = attention(**over)
    if a.nseq > 3:
        assert b.switchhead_attention_workspace_bytes(a) == 0 and forward(a) == b.SH_ERR_UNSUPPORTED and backward(a) == b.SH_ERR_UNSUPPORTED
    else:   # the largest rows that are not joined from parts fit
        assert b.switchhead_attention_workspace_bytes(a) > 0


def test_null_descriptions():
    assert lib().switchhead_attention_workspace_bytes(None, 0) == 0
    assert lib().switchhead_qk_norm_workspace_bytes(None) == 0


def norm(**over):
    f = dict(tokens=10, nheads=4, nkv_heads=2, d_head=64, rope_dim=64, dtype=b.SH_BF16, eps=1e-6, theta=0.0)
    f.update(over)
    return b.sh_qk_norm(**f)


def norm_forward(a, **over):
    p = dict(Q=P, K=P, wq=P, wk=P, pos=P, YQ=2 * P, YK=2 * P)
    p.update(over)
    return lib().switchhead_qk_norm_rope_forward(ctypes.byref(a), *p.values(), None)


def norm_backward(a, ws=1 << 40, **over):
    p = dict(Q=P, K=P, wq=P, wk=P, pos=P, dYQ=2 * P, dYK=2 * P, dQ=3 * P, dK=3 * P, dwq=P, dwk=P, workspace=P)
    p.update(over)
    return lib().switchhead_qk_norm_rope_backward(ctypes.byref(a), *p.values(), ws, None)


NORM_INVALID = [dict(tokens=-1), dict(nheads=0), dict(nkv_heads=-1), dict(d_head=0), dict(rope_dim=3), dict(rope_dim=66), dict(rope_dim=-2), dict(dtype=4),
                dict(eps=-1.0), dict(eps=float("nan")), dict(theta=-2.0), dict(theta=float("inf"))]
NORM_UNSUPPORTED = [dict(d_head=300), dict(nheads=5000), dict(q_row=-1), dict(yk_row=1 << 23)]


@pytest.mark.parametrize("over", NORM_INVALID + NORM_UNSUPPORTED, ids=str)
def test_norm_descriptions_that_are_refused(over):
    a = norm(**over)
    code = b.SH_ERR_INVALID_ARG if over in NORM_INVALID else b.SH_ERR_UNSUPPORTED
    assert b.switchhead_qk_norm_workspace_bytes(a) == 0
    assert norm_forward(a) == code and norm_backward(a) == code


def test_norm_tensors():
    a = norm()
    for name in ("Q", "K", "YQ", "YK"):
        assert norm_forward(a, **{name: None}) == b.SH_ERR_INVALID_ARG
    for name in ("Q", "K", "dYQ", "dYK", "dQ", "dK", "workspace"):
        assert norm_backward(a, **{name: None}) == b.SH_ERR_INVALID_ARG
    assert norm_forward(a, wq=P + 1) == b.SH_ERR_INVALID_ARG and norm_forward(a, pos=P + 2) == b.SH_ERR_INVALID_ARG
    assert norm_backward(a, dwq=P + 2) == b.SH_ERR_INVALID_ARG
    assert norm_backward(a, ws=b.switchhead_qk_norm_workspace_bytes(a) - 1) == b.SH_ERR_WORKSPACE_TOO_SMALL
    # an output over its input with other strides; outputs whose rows overlap
    assert norm_forward(norm(q_row=1024, q_head=64), YQ=P) == b.SH_ERR_INVALID_ARG
    assert norm_backward(norm(q_row=1024, q_head=64), dQ=2 * P) == b.SH_ERR_INVALID_ARG
    assert norm_forward(norm(yq_row=64, yq_head=64)) == b.SH_ERR_INVALID_ARG
    assert norm_backward(norm(k_row=64, k_head=64)) == b.SH_ERR_INVALID_ARG
    assert norm_forward(norm(tokens=0), Q=None, K=None, YQ=None, YK=None) == b.SH_OK


def test_binding_checks_of_tensors():
    torch = pytest.importorskip("torch")
    t = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype)
    q, k = t(10, 4, 64), t(20, 2, 64)
    ok = b.make_attention(q, k, k, q, 3, 5, 8)
    assert (ok.nheads, ok.nkv_heads, ok.d_head, ok.total_q, ok.total_k, ok.q_row, ok.k_row) == (4, 2, 64, 10, 20, 256, 128)
    fused = t(10, 8, 64)
    v = b.make_attention(fused[:, :4], fused[:, 4:6], fused[:, 6:], q, 3, 5, 8)
    assert (v.q_row, v.k_row, v.v_head, v.o_row) == (512, 512, 64, 256)
    bad = [lambda: b.make_attention(q.half(), k.half(), k.half(), q.half(), 3, 5, 8), lambda: b.make_attention(q, k.float(), k, q, 3, 5, 8),
           lambda: b.make_attention(q, k, t(20, 1, 64), q, 3, 5, 8), lambda: b.make_attention(q, k, t(19, 2, 64), q, 3, 5, 8),
           lambda: b.make_attention(q, k, k, t(10, 4, 32), 3, 5, 8), lambda: b.make_attention(q, k, k, q, 3, 5, 8, K_prefix=k),
           lambda: b.make_attention(q, t(1, 2, 64).expand(20, 2, 64), k, q, 3, 5, 8), lambda: b.make_attention(q, t(20, 2, 128)[..., ::2], k, q, 3, 5, 8),
           lambda: b.make_attention(q[0], k, k, q, 3, 5, 8), lambda: b.make_qk_norm(q, k, q, k, 64), lambda: b.make_qk_norm(q, None, q, q, 64),
           lambda: b.make_qk_norm(q, None, t(9, 4, 64), None, 64),
           lambda: b.switchhead_attention_forward(ok, q, k, k, q, q, q, None, q)]   # tensors in host memory
    for call in bad:
        with pytest.raises(b.SwitchHeadError):
            call()


def shape(**over):
    f = dict(B=1, T=100, d_model=64, nheads=2, d_head=32, E=4, k=2, causal=1, dtype="f32")
    f.update(over)
    return b.make_shape(**f)


def packing(**over):
    f = dict(nseq=3, max_len=50, offsets=P, q_norm=None, k_norm=None, norm_eps=1e-6)
    f.update(over)
    return b.sh_packing(*f.values())


def packed_forward(s, p, ws=1 << 40, **over):
    a = dict(x=P, W_Q=P, W_K=P, W_V=P, W_O=P, W_S=P, W_D=P, b_S=None, b_D=None, y=P, workspace=P)
    a.update(over)
    return lib().switchhead_forward_packed(ctypes.byref(s), ctypes.byref(p) if p else None, *a.values(), ws, None)


def packed_backward(s, p, ws=1 << 40, **over):
    a = dict(x=P, W_Q=P, W_K=P, W_V=P, W_O=P, W_S=P, W_D=P, dy=P, workspace=P)
    a.update(over)
    return lib().switchhead_backward_packed(ctypes.byref(s), ctypes.byref(p), *a.values(), ws, *[P] * 11, None)


def test_packed_layer_refusals():
    ok = shape(), packing()
    need = b.switchhead_packed_workspace_bytes(*ok)
    assert need >= b.switchhead_workspace_bytes(ok[0])
    assert packed_forward(*ok, ws=need - 1) == packed_backward(*ok, ws=need - 1) == b.SH_ERR_WORKSPACE_TOO_SMALL
    for s, p in ((shape(B=2), packing()), (shape(), packing(nseq=0)), (shape(), packing(max_len=0)), (shape(), packing(q_norm=P)), (shape(), packing(k_norm=P)),
                 (shape(), packing(norm_eps=-1.0)), (shape(), packing(norm_eps=float("nan"))), (shape(), packing(q_norm=P + 2, k_norm=P)),
                 (shape(), packing(offsets=P + 2)), (shape(T=0), packing())):
        assert b.switchhead_packed_workspace_bytes(s, p) == 0 and b.switchhead_last_error()
        assert packed_forward(s, p) == b.SH_ERR_INVALID_ARG and packed_backward(s, p) == b.SH_ERR_INVALID_ARG
    assert packed_forward(shape(), None) == b.SH_ERR_INVALID_ARG
    # sizes can be asked for before there are offsets
    assert b.switchhead_packed_workspace_bytes(shape(), packing(offsets=None)) == need
    assert packed_forward(shape(), packing(offsets=None)) == b.SH_ERR_INVALID_ARG
    # a prefix: forward only
    assert packed_backward(shape(T_q=60), packing()) == b.SH_ERR_UNSUPPORTED
    for n in ("x", "W_Q", "W_O", "y", "workspace"):
        assert packed_forward(*ok, **{n: None}) == b.SH_ERR_INVALID_ARG
