"""The forward kernels that a training step's larger calls run: workgroups of 128 and 256 queries, with and without keys
that several share, and what keeps row statistics in them (shared heads, lengths that end inside a tile, empty sequences,
masks).  The library is asked which kernel a case takes, so that another rule for it does not drop one from the tests."""
import math

import pytest
import torch

from paper_2602_12271_amd import binding as B

from dense_training import Step, check, reference, run, tensors
from training_norms import check_norms

# name: (queries of a workgroup, whether workgroups share keys, step); on 256 compute units
SHAPES = {
    "256-padded": (256, False, Step(300, 300, heads=40, kv_heads=8, batch=3, kv_len=(300, 129, 0))),
    "256-few-keys": (256, False, Step(257, 90, heads=64, batch=2, kv_len=(90, 1))),
    "256-causal": (256, False, Step(400, 400, heads=16, kv_heads=2, batch=8, chunk=1, kv_len=(400, 399, 257, 256, 129, 64, 1, 0))),
    "256-frames": (256, False, Step(3, 3, 10, 13, heads=24, kv_heads=8, batch=5, chunk=1, kv_len=(390, 261, 131, 130, 0))),
    "256-chunks": (256, False, Step(6, 6, 10, 11, heads=16, kv_heads=4, batch=8, chunk=3)),
    "256-cache": (256, False, Step(2, 6, 9, 13, heads=32, kv_heads=8, batch=8, chunk=2, offset=2)),
    "256-tokens-outside-heads": (256, False, Step(3, 3, 10, 11, heads=16, kv_heads=4, batch=8, chunk=1, layout="bnhd")),
    "128-padded": (128, False, Step(130, 300, heads=64, kv_heads=16, batch=2, kv_len=(300, 33))),
    "128-causal": (128, False, Step(300, 300, heads=40, kv_heads=8, batch=3, chunk=1, kv_len=(300, 129, 0))),
    "128-shared-keys": (128, True, Step(1346, 1846, heads=1, batch=4, kv_len=(1846, 1000, 64, 0))),
    "128-shared-keys-chunks": (128, True, Step(5, 7, 16, 20, heads=2, batch=2, chunk=2, offset=2, kv_len=(2240, 1500))),
    "128-d64-padded": (128, False, Step(300, 300, heads=40, kv_heads=8, batch=3, dim=64, kv_len=(300, 129, 0))),
    "128-d64-frames": (128, False, Step(2, 2, 5, 16, heads=64, kv_heads=16, batch=4, dim=64, chunk=1, kv_len=(160, 81, 80, 0))),
    "f32-128": (128, False, Step(520, 520, heads=8, batch=8, dtype="f32")),
    "f32-128-padded": (128, False, Step(520, 520, heads=8, kv_heads=4, batch=8, dtype="f32", kv_len=(520, 519, 300, 256, 64, 17, 1, 0))),
    "f32-128-chunks-d64": (128, False, Step(4, 4, 13, 14, heads=16, kv_heads=4, batch=5, dim=64, dtype="f32", chunk=2, kv_len=(728, 500, 365, 90, 0))),
    "bf16-in-f32-128": (128, False, Step(520, 520, heads=8, batch=8, compute=1, kv_len=(520, 519, 300, 256, 64, 17, 1, 0))),
}


def kernel_of(c: Step):
    prob = B.make_problem(batch=c.batch, heads=c.heads, head_dim=c.dim, f_q=c.f_q, f_kv=c.f_kv, h=c.h, w=c.w, q_frame_offset=c.offset,
                          dtype=B.MRT_F32 if c.dtype == "f32" else B.MRT_BF16, compute=c.compute, scale=c.args["scale"])
    train = B.MrtDenseTrain(c.kv_heads, None, prob.q, prob.q, prob.k, prob.v)
    scratch = B.dense_attn_fwd_save_workspace_bytes(prob, train, c.chunk)
    return B.dense_attn_fwd_save_queries(prob, train, c.chunk, scratch), scratch > 0


@pytest.mark.parametrize("name", SHAPES)
def test_kernel(name):
    queries, shared, c = SHAPES[name]
    assert kernel_of(c) == (queries, shared)


def test_kernel_of_invalid_arguments():
    prob = B.make_problem(batch=1, heads=6, head_dim=128, f_q=1, f_kv=1, h=5, w=6)
    assert B.dense_attn_fwd_save_queries(prob, B.MrtDenseTrain(4), 0, 0) == 0
    assert B.dense_attn_fwd_save_queries(prob, B.MrtDenseTrain(3), -1, 0) == 0
    assert B.load_library().dense_attn_fwd_save_queries(None, None, 0, 0) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("name", SHAPES)
def test_training_step(name):
    queries, shared, c = SHAPES[name]
    assert kernel_of(c) == (queries, shared)
    q, k, v, do, kv_len = tensors(c, seed=51)
    ref, cost = reference(c, q, k, v, do)
    got = run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    print(f"  {name}: {check(c, got, ref, cost)}", flush=True)
    print(f"  {check_norms(c, got, ref)}", flush=True)


@pytest.mark.gpu
@pytest.mark.parametrize("name", [n for n, (_, _, c) in SHAPES.items() if c.kv_len])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_padding_holds_anything(name, value):
    c = SHAPES[name][2]
    q, k, v, do, kv_len = tensors(c, seed=52)
    want = run(c, q, k, v, do, kv_len)
    for b, n in enumerate(c.kv_len):
        k[b, :, n:], v[b, :, n:] = value, -value
    got = run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    for n in got:
        assert torch.equal(got[n], want[n]), n
