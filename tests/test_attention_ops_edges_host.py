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
