"""CPU-only: dense attention over a cache with O in the place of Q takes Q's strides for O.  No kernel is launched here."""
import ctypes

import pytest

import paper_2602_12271_amd as pkg
from paper_2602_12271_amd import binding as B

A = [0x10000 * (i + 1) for i in range(8)]        # addresses that no launch sees: every call is refused before
S = B.MrtStrides


def cache(batch):
    st = S(1 << 20, 1 << 16, 128)
    return B.MrtCache8(batch, 2, 128, 64, 16, 0, st, st, 64, 8, 64, 8, A[0], A[1], A[2], A[3])


@pytest.mark.parametrize("o", [S(1 << 16, 1 << 12, 136), S(1 << 16, 1 << 13, 128), S(1 << 17, 1 << 12, 128)])
def test_other_strides(o):
    p = pkg.make_problem(batch=2, heads=4, head_dim=128, f_q=2, f_kv=4, h=2, w=4, scale=0.1, q_strides=(1 << 16, 1 << 12, 128),
                         o_strides=(o.batch, o.head, o.token))
    lib, c = pkg.load_library(), cache(2)
    assert lib.dense_attn_cache8_check(ctypes.byref(p), ctypes.byref(c), 0) == 0
    assert lib.dense_attn_fwd_cache8(A[4], ctypes.byref(c), A[4], A[5], ctypes.byref(p), None, 0, None, 0, None) == B.MRT_ERR_SHAPE
    assert "place of Q" in B.last_error()
