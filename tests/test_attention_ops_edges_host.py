"""Refusals of the attention and norm operators at the edges of their descriptions: nothing is launched, so none of this needs a GPU (made-up addresses
stand for device memory)."""
import ctypes

import pytest

from paper_2312_07987_amd import binding as b

P = 0x10000   # an address that is never read


def attention_backward(a, ws=1 << 50, **over):
    p = dict(Q=P, K=2 * P, V=3 * P, O=4 * P, dO=5 * P, lse=6 * P, qo=7 * P, ql=None, ko=7 * P, kl=None, dQ=8 * P, dK=9 * P, dV=10 * P, workspace=11 * P)
    p.update(over)
    return b.lib().switchhead_attention_backward(ctypes.byref(a), *p.values(), ws, None)


@pytest.mark.parametrize("d_head,dtype,rows", [(64, b.SH_BF16, 1 << 29), (128, b.SH_BF16, 1 << 28), (65, b.SH_BF16, 1 << 28), (256, b.SH_F32, 1 << 26), (32, b.SH_F32, 1 << 29)])
def test_rows_whose_dot_products_no_launch_holds(d_head, dtype, rows):
    """Several lanes form a row's <dO, O>: 2^32 of them are refused before anything runs, a few less are not (the workspace is checked next)."""
    a = b.sh_attention(nseq=1, nheads=64, nkv_heads=1, d_head=d_head, causal=1, dtype=dtype, total_q=rows // 64, total_k=8, max_q=8, max_k=8)
    assert attention_backward(a) == b.SH_ERR_UNSUPPORTED
    a.total_q -= 8
    assert attention_backward(a, ws=0) == b.SH_ERR_WORKSPACE_TOO_SMALL


def norm_forward(a, Q=P, Y=2 * P, K=None, YK=None):
    return b.lib().switchhead_qk_norm_rope_forward(ctypes.byref(a), Q, K, None, None, None, Y, YK, None)


def norm_backward(a, dY=2 * P, dQ=3 * P, K=None, dYK=None, dK=None, ws=1 << 40):
    return b.lib().switchhead_qk_norm_rope_backward(ctypes.byref(a), P, K, None, None, None, dY, dYK, dQ, dK, None, None, P, ws, None)


def test_one_token_in_place_needs_the_same_head_strides():
    """Heads of one token are work of different groups of lanes: with other head strides one would write what another has yet to read."""
    a = b.sh_qk_norm(tokens=1, nheads=4, nkv_heads=0, d_head=64, rope_dim=0, dtype=b.SH_BF16, q_head=128, yq_head=64)
    assert norm_forward(a, Y=P) == b.SH_ERR_INVALID_ARG and norm_backward(a, dQ=2 * P) == b.SH_ERR_INVALID_ARG
    a = b.sh_qk_norm(tokens=1, nheads=1, nkv_heads=3, d_head=64, rope_dim=0, dtype=b.SH_BF16, k_head=128, yk_head=64)
    assert norm_forward(a, K=3 * P, YK=3 * P) == b.SH_ERR_INVALID_ARG and norm_backward(a, K=P, dYK=4 * P, dK=4 * P) == b.SH_ERR_INVALID_ARG
    # one head: its stride means nothing, but the rows' does (refused before a launch for the workspace, so as to launch nothing here)
    a = b.sh_qk_norm(tokens=4, nheads=1, nkv_heads=0, d_head=64, rope_dim=0, dtype=b.SH_BF16, q_row=512, q_head=128, yq_row=512, yq_head=64)
    assert norm_backward(a, dQ=2 * P, ws=0) == b.SH_ERR_WORKSPACE_TOO_SMALL
    a = b.sh_qk_norm(tokens=4, nheads=1, nkv_heads=0, d_head=64, rope_dim=0, dtype=b.SH_BF16, q_row=512, yq_row=64)
    assert norm_backward(a, dQ=2 * P) == b.SH_ERR_INVALID_ARG


def test_outputs_over_what_is_still_read():
    """Refused where the addresses say so: dK and dV are written before dQ's kernel reads K (and the rest, where it works the scores out again)."""
    a = b.sh_attention(nseq=1, nheads=4, nkv_heads=4, d_head=64, causal=1, dtype=b.SH_BF16, total_q=10, total_k=10, max_q=10, max_k=10)
    for out, at in (("dK", 1), ("dK", 2), ("dK", 3), ("dK", 5), ("dV", 1), ("dV", 2), ("dV", 3), ("dV", 5), ("dQ", 2), ("dQ", 3), ("dQ", 9), ("dQ", 10), ("dV", 9)):
        assert attention_backward(a, **{out: at * P}) == b.SH_ERR_INVALID_ARG, (out, at)
    assert b"gradient" in b.lib().switchhead_last_error()
    for at in (2, 3, 5, 6):
        p = dict(Q=P, K=2 * P, V=3 * P, KP=5 * P, VP=6 * P, qo=7 * P, ql=None, ko=7 * P, kl=None, O=at * P, lse=None, workspace=11 * P)
        a.prefix = 3
        assert b.lib().switchhead_attention_forward(ctypes.byref(a), *p.values(), 1 << 40, None) == b.SH_ERR_INVALID_ARG
    n = b.sh_qk_norm(tokens=4, nheads=2, nkv_heads=2, d_head=64, rope_dim=0, dtype=b.SH_BF16)
    for Y, YK in ((3 * P, 4 * P), (2 * P, P), (2 * P, 2 * P)):
        assert norm_forward(n, Q=P, K=3 * P, Y=Y, YK=YK) == b.SH_ERR_INVALID_ARG
    for dQ, dK in ((5 * P, 8 * P), (6 * P, 8 * P), (8 * P, P), (8 * P, 2 * P), (8 * P, 8 * P)):
        assert norm_backward(n, K=5 * P, dYK=6 * P, dQ=dQ, dK=dK) == b.SH_ERR_INVALID_ARG


def test_prefix_whose_tiles_pass_32_bits():
    a = b.sh_attention(nseq=1, nheads=1, nkv_heads=1, d_head=1, causal=1, dtype=b.SH_BF16, total_q=10, total_k=10, max_q=10, max_k=10, prefix=1 << 30)
    assert b.switchhead_attention_workspace_bytes(a) == 0
    a.prefix -= 1
    assert b.switchhead_attention_workspace_bytes(a) > 0


# ---- the binding compares tensors with the description -----------------------------------------------------------------------
def tensors(dtype="bfloat16"):
    torch = pytest.importorskip("torch")
    z = lambda *s, dt=getattr(torch, dtype): torch.zeros(*s, dtype=dt)
    fused = z(10, 8, 64)
    t = dict(Q=fused[:, :4], K=fused[:, 4:6], V=fused[:, 6:], O=z(10, 4, 64), dO=z(10, 4, 64), lse=z(4, 10, dt=torch.float32),
             q_offsets=z(4, dt=torch.int32), k_offsets=z(4, dt=torch.int32), workspace=z(1 << 20, dt=torch.uint8))
    grad = torch.zeros_like(fused, memory_format=torch.contiguous_format)
    t.update(dQ=grad[:, :4], dK=grad[:, 4:6], dV=grad[:, 6:])
    return torch, t, b.make_attention(t["Q"], t["K"], t["V"], t["O"], 3, 5, 5)


def refused(call, text):
    with pytest.raises(b.SwitchHeadError, match=text) as e:
        call()
    assert e.value.code == b.SH_ERR_INVALID_ARG


FORWARD = ("Q", "K", "V", "q_offsets", "k_offsets", "O", "lse", "workspace")
BACKWARD = ("Q", "K", "V", "O", "dO", "lse", "q_offsets", "k_offsets", "dQ", "dK", "dV", "workspace")


def both(a, t, **over):
    """The forward and the backward call with these tensors in other places, without those that a call does not take."""
    u = dict(t, **over)
    extra = {n: u[n] for n in ("q_lengths", "k_lengths") if n in u}
    calls = []
    if not set(over) & {"dO", "dQ", "dK", "dV"}:
        calls.append(lambda: b.switchhead_attention_forward(a, *[u[n] for n in FORWARD], **extra))
    return calls + [lambda: b.switchhead_attention_backward(a, *[u[n] for n in BACKWARD], **extra)]


def test_attention_tensors_that_the_description_does_not_mean():
    torch, t, a = tensors()
    for call in both(a, t):   # right in everything but where they are
        refused(call, "must be on a GPU")
    for name in ("dQ", "dK", "dV", "Q", "K", "V"):   # dense, as torch.empty_like makes them of views: their rows are not where the strides say
        like = torch.empty_like(t["Q" if name[-1] == "Q" else "K"])
        assert like.is_contiguous()
        for call in both(a, t, **{name: like}):
            refused(call, name + " has strides")
    for name in ("O", "dO"):
        for call in both(a, t, **{name: t["Q"]}):
            refused(call, name + " has strides")
    for name in FORWARD[:3] + ("O", "dO", "dQ", "dK", "dV"):
        for bad in (t[name].float(), t[name][:9], t[name][:, :1], t[name][..., :32]):
            for call in both(a, t, **{name: bad}):
                refused(call, name + " is")
    for name in ("O", "dO", "dQ", "dK", "dV"):
        refused(both(a, t, **{name: None})[-1], name + " is missing")
    int64 = torch.cumsum(torch.zeros(4, dtype=torch.int32), 0)
    assert int64.dtype == torch.int64
    short, strided = torch.zeros(3, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)[::2]
    for name in ("q_offsets", "k_offsets"):
        for bad in (int64, short, strided):
            for call in both(a, t, **{name: bad}):
                refused(call, name + " must be")
    for name in ("q_lengths", "k_lengths"):
        for bad in (int64[:3], short[:2], strided[:3]):
            for call in both(a, t, **{name: bad}):
                refused(call, name + " must be")
    for bad in (t["lse"].double(), t["lse"][:, :9], t["lse"][:3], torch.zeros(10, 4).t()):
        for call in both(a, t, lse=bad):
            refused(call, "lse must be")
    for call in both(a, t, workspace=t["workspace"][::2]):
        refused(call, "workspace must be")


def test_attention_places_follow_the_fields():
    """A description made by hand, or changed, is held to its fields; strides along one row or head mean nothing."""
    torch, t, a = tensors()
    hand = b.sh_attention(**{n: getattr(a, n) for n, _ in b.sh_attention._fields_})
    refused(both(hand, t)[0], "must be on a GPU")
    refused(both(hand, t, dK=torch.empty_like(t["K"]))[0], "dK has strides")
    dense = b.sh_attention(nseq=3, nheads=4, nkv_heads=2, d_head=64, causal=1, dtype=b.SH_BF16, total_q=10, total_k=10, max_q=5, max_k=5)
    own = {n: v.contiguous() if v.dim() == 3 else v for n, v in t.items()}
    refused(both(dense, own)[0], "must be on a GPU")
    refused(both(dense, t)[0], "Q has strides")
    a.k_row = 256
    refused(both(a, t)[0], "K has strides")
    one = [torch.zeros(1, 1, 64).as_strided((1, 1, 64), s) for s in ((64, 64, 1), (640, 7, 1))]
    a = b.make_attention(one[0], one[0], one[0], one[0], 1, 1, 1)
    off = torch.zeros(2, dtype=torch.int32)
    refused(lambda: b.switchhead_attention_forward(a, one[1], one[1], one[0], off, off, one[1], None, t["workspace"]), "must be on a GPU")


def test_prefix_tensors():
    torch, t, _ = tensors()
    kp = torch.zeros(7, 2, 64, dtype=torch.bfloat16)
    a = b.make_attention(t["Q"], t["K"], t["V"], t["O"], 3, 5, 5, 1, kp, kp)
    call = lambda **p: b.switchhead_attention_forward(a, *[t[n] for n in FORWARD], **p)
    refused(lambda: call(K_prefix=kp, V_prefix=kp), "must be on a GPU")
    refused(lambda: call(), "K_prefix is missing")
    refused(lambda: call(K_prefix=kp), "V_prefix is missing")
    refused(lambda: call(K_prefix=kp[:6], V_prefix=kp), "K_prefix is")
    refused(lambda: call(K_prefix=kp, V_prefix=torch.zeros(7, 4, 64, dtype=torch.bfloat16)[:, :2]), "V_prefix has strides")


def test_norm_tensors_that_the_description_does_not_mean():
    torch, t, _ = tensors()
    Q, K = t["Q"], t["K"]
    YQ, YK, w, pos = torch.zeros(10, 4, 64, dtype=Q.dtype), torch.zeros(10, 2, 64, dtype=Q.dtype), torch.zeros(64, dtype=Q.dtype), torch.zeros(10, dtype=torch.int32)
    a = b.make_qk_norm(Q, K, YQ, YK, 64)
    dw = torch.zeros(64)

    def forward(**o):
        u = dict(dict(Q=Q, K=K, w_Q=w, w_K=w, positions=pos, Y_Q=YQ, Y_K=YK), **o)
        return b.switchhead_qk_norm_rope_forward(a, **u)

    def backward(**o):
        u = dict(dict(Q=Q, K=K, w_Q=w, w_K=w, positions=pos, dY_Q=YQ, dY_K=YK, dQ=t["dQ"], dK=t["dK"], dw_Q=dw, dw_K=dw, workspace=t["workspace"]), **o)
        return b.switchhead_qk_norm_rope_backward(a, **u)

    refused(forward, "must be on a GPU")
    refused(backward, "must be on a GPU")
    for call in (forward, backward):
        for name in ("Q", "K"):
            good = dict(Q=Q, K=K)[name]
            refused(lambda: call(**{name: torch.empty_like(good)}), name + " has strides")
            refused(lambda: call(**{name: good.float()}), name + " is")
            refused(lambda: call(**{name: None}), name) if name == "K" else None
        for name in ("w_Q", "w_K"):
            for bad in (w.float(), w[:63], torch.zeros(128, dtype=Q.dtype)[::2]):
                refused(lambda: call(**{name: bad}), name + " must be")
        for bad in (pos.long(), pos[:9]):
            refused(lambda: call(positions=bad), "positions must be")
    for name, good in (("Y_Q", YQ), ("Y_K", YK)):
        refused(lambda: forward(**{name: good[:9]}), name + " is")
        refused(lambda: backward(**{"d" + name: good.float()}), "d" + name + " is")
    for name, good in (("dQ", Q), ("dK", K)):
        refused(lambda: backward(**{name: torch.empty_like(good)}), name + " has strides")
    for name in ("dw_Q", "dw_K"):
        for bad in (dw.double(), dw[:63]):
            refused(lambda: backward(**{name: bad}), name + " must be")
    refused(lambda: backward(workspace=t["workspace"][::2]), "workspace must be")


def test_packing_tensors():
    torch = pytest.importorskip("torch")
    off = torch.zeros(4, dtype=torch.int32)
    for bad in (off.long(), off[:1], torch.zeros(8, dtype=torch.int32)[::2]):
        refused(lambda: b.make_packing(bad, 5), "offsets must be")
    shape = b.make_shape(1, 100, 64, 2, 32, 4, 2, dtype="f32")
    x, ws, w = torch.zeros(1, 100, 64), torch.zeros(1 << 20, dtype=torch.uint8), torch.zeros(32)
    forward = lambda p: b.switchhead_forward_packed(shape, p, x, *[w] * 6, None, None, x, ws)
    backward = lambda p, *dn: b.switchhead_backward_packed(shape, p, x, *[w] * 6, x, ws, x, *[w] * 6, w, w, *dn)
    refused(lambda: forward(b.make_packing(off, 50, w, w)), "must be on a GPU")
    refused(lambda: backward(b.make_packing(off, 50, w, w), w, w), "must be on a GPU")
    for bad in (w[:31], w.double(), w.bfloat16()):
        refused(lambda: forward(b.make_packing(off, 50, w, bad)), "a norm's weights must be")
        refused(lambda: backward(b.make_packing(off, 50, bad, w)), "a norm's weights must be")
        refused(lambda: backward(b.make_packing(off, 50, w, w), w, bad), "a norm's gradient must be")
