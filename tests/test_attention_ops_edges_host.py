"""Refusals of the attention and norm operators at the edges of their descriptions: nothing is launched, so none of this needs a GPU (made-up addresses
stand for device memory)."""
import ctypes

import pytest

from paper_2312_07987_amd import binding as b

P = 0x10000   # an address that is never read


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
