"""Dense attention with a frame offset at the end of 32 bits: refused under a mask where the frames pass it (the kernels'
limits of what a query sees would wrap and their loads reach behind the keys), as before everywhere else."""
import ctypes

import pytest
import torch

import paper_2602_12271_amd as pkg
from paper_2602_12271_amd import binding as B

from dense_training import Step, run, tensors

LAST = 2 ** 31 - 1


@pytest.mark.parametrize("kw", [dict(dtype=B.MRT_BF16), dict(dtype=B.MRT_F32, head_dim=37)], ids=["bf16", "f32"])
@pytest.mark.parametrize("offset,chunk,good", [(LAST, 1, False), (LAST - 1, 1, False), (LAST - 2, 1, True), (LAST - 2, LAST, True), (LAST, 0, True)])
def test_refusals(kw, offset, chunk, good):
    lib = pkg.load_library()
    p = pkg.make_problem(**{**dict(batch=2, heads=6, head_dim=128, f_q=2, f_kv=3, h=5, w=7, scale=0.1, q_frame_offset=offset), **kw})
    t = B.MrtDenseTrain(0, None, p.o, p.q, p.k, p.v)
    status = 0 if good else B.MRT_ERR_SHAPE
    assert B.dense_attn_check(p, chunk) == status
    assert lib.dense_attn_bwd_check(ctypes.byref(p), ctypes.byref(t), chunk) == status
    assert (B.dense_attn_bwd_workspace_bytes(p, t, chunk) > 0) == good
    assert (B.dense_attn_fwd_save_queries(p, t, chunk) > 0) == good
    if good:
        return
    at = [0x10000 * (i + 1) for i in range(10)]          # addresses that no launch sees
    assert lib.dense_attn_fwd(*at[:4], ctypes.byref(p), chunk, None) == status
    assert lib.dense_attn_fwd_save(*at[:5], ctypes.byref(p), ctypes.byref(t), chunk, at[9], 1 << 40, None) == status
    assert lib.dense_attn_bwd(*at[:9], ctypes.byref(p), ctypes.byref(t), chunk, at[9], 1 << 40, None) == status
    assert "q_frame_offset" in B.last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("chunk", [1, LAST])
def test_last_frames(dtype, chunk):
    """The last offset there is: every key is seen, so the results are those of no mask, up to the order of sums."""
    import dataclasses
    c = Step(2, 3, 7, 9, heads=2, dtype=dtype, chunk=chunk, offset=LAST - 2)
    q, k, v, do, _ = tensors(c, seed=61)
    got, want = run(c, q, k, v, do, None), run(dataclasses.replace(c, chunk=0), q, k, v, do, None)
    args = dict(c.args)
    args.pop("causal_chunk")
    o = [pkg.dense_attn_fwd(q, k, v, causal_chunk=n, **args) for n in (chunk, 0)]
    torch.cuda.synchronize()
    limit = 1e-2 if dtype == "bf16" else 1e-5
    for x, y in [*((got[n], want[n]) for n in got), tuple(o)]:
        assert float((x - y).float().norm()) <= limit * float(y.float().norm())
