"""GPU: the dense attention's training step (dense_attn_fwd_save, dense_attn_bwd) against its formulas in 64 bits,
entry by entry within what the roundings of its operands may cost."""
import dataclasses

import pytest
import torch

import paper_2602_12271_amd as pkg

from dense_training import Step, check, reference, run, tensors

pytestmark = pytest.mark.gpu

CASES = {
    "one-token": Step(1, 1),
    "one-token-d64": Step(1, 1, dim=64, heads=3),
    "one-query-few-keys": Step(1, 5),
    "one-query-long": Step(1, 4111, heads=3, batch=2),
    "one-query-long-d64-shared": Step(1, 2049, heads=8, kv_heads=2, dim=64),
    "few-queries-one-key": Step(7, 1, heads=2),
    "tile-edges-31": Step(31, 31),
    "tile-edges-32": Step(32, 32, dim=64),
    "tile-edges-33": Step(33, 65),
    "tile-edges-257": Step(257, 129, heads=1),
    "more-queries-than-keys": Step(700, 40, dim=64),
    "frames": Step(2, 2, 17, 23, heads=3),
    "frames-d64": Step(2, 2, 17, 23, heads=3, dim=64, batch=2),
    "cache": Step(2, 6, 9, 11, chunk=2, offset=4),
    "cache-early": Step(2, 6, 9, 11, chunk=2, offset=0),
    "cache-d64-shared": Step(2, 6, 9, 11, heads=6, kv_heads=2, chunk=2, offset=2, dim=64),
    "chunk-causal": Step(6, 6, 7, 9, chunk=2),
    "chunk-causal-one-frame-d64": Step(5, 5, 5, 13, chunk=1, dim=64),
    "causal": Step(321, 321, chunk=1, heads=2),
    "causal-shared-d64": Step(203, 203, chunk=1, heads=4, kv_heads=1, dim=64, batch=2),
    "causal-offset": Step(40, 200, chunk=1, offset=160, heads=2),
    "keys-no-query-sees": Step(3, 40, 4, 4, chunk=2, offset=1),
    "shared": Step(150, 150, heads=6, kv_heads=3, batch=2),
    "padded": Step(130, 130, heads=2, batch=4, kv_len=(130, 77, 1, 0)),
    "padded-d64-shared-causal": Step(3, 3, 6, 7, heads=4, kv_heads=2, batch=3, dim=64, chunk=1, kv_len=(126, 50, 0)),
    "padded-beyond": Step(70, 70, batch=2, kv_len=(1000, -3)),
    "padded-one-query": Step(1, 3000, heads=2, batch=3, kv_len=(3000, 1100, 0)),
    "tokens-outside-heads": Step(2, 3, 8, 9, heads=4, kv_heads=2, batch=2, layout="bnhd"),
    "packed-d64": Step(2, 2, 8, 9, heads=4, batch=2, dim=64, layout="packed"),
    "sharp": Step(200, 200, sigma=2.0),
    "scale-one": Step(64, 96, dim=64, scale=1.0, sigma=0.5),
    "f32": Step(2, 2, 10, 13, dtype="f32", dim=64),
    "f32-d128-shared-causal": Step(97, 97, heads=4, kv_heads=2, chunk=1, dtype="f32"),
    "f32-odd-dim": Step(2, 3, 5, 7, dim=37, dtype="f32", chunk=1, offset=1),
    "f32-dim-1": Step(19, 23, dim=1, dtype="f32"),
    "f32-dim-96": Step(1, 1, 11, 13, dim=96, dtype="f32", batch=2, layout="bnhd"),
    "f32-padded": Step(75, 75, batch=4, dtype="f32", kv_len=(75, 64, 3, 0)),
    "f32-padded-causal": Step(3, 3, 5, 5, batch=3, dim=64, dtype="f32", chunk=1, kv_len=(75, 30, 0)),
    "f32-one-query": Step(1, 1030, heads=3, dtype="f32"),
    "f32-one-token": Step(1, 1, dtype="f32", dim=8),
    "bf16-in-f32": Step(2, 2, 9, 10, compute=1, chunk=1),
    "bf16-in-f32-dim-40": Step(60, 50, compute=1, dim=40),
}


@pytest.mark.parametrize("name", CASES)
def test_training_step(name):
    c = CASES[name]
    q, k, v, do, kv_len = tensors(c)
    ref, cost = reference(c, q, k, v, do)
    got = run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    print(f"  {name}: {check(c, got, ref, cost)}", flush=True)


# up to 32 rows (the queries of all heads that share keys) take a launch of their own
FEW = {
    "one-row": Step(1, 700, heads=3, batch=2),
    "thirty-two-rows": Step(32, 333, heads=2),
    "thirty-three-rows": Step(33, 333, heads=2),
    "rows-of-heads": Step(4, 517, heads=8, kv_heads=1, batch=2),
    "rows-of-heads-d64": Step(5, 130, heads=6, kv_heads=1, dim=64, batch=3),
    "a-tile-of-keys": Step(3, 32, dim=64),
    "keys-31": Step(3, 31, heads=1),
    "keys-129-d64": Step(2, 129, heads=1, dim=64),
    "causal": Step(20, 300, chunk=1, offset=280, heads=2),
    "causal-shared": Step(8, 100, chunk=1, offset=40, heads=4, kv_heads=1, dim=64),
    "chunks": Step(2, 9, 1, 12, chunk=3, offset=3, heads=2),
    "padded": Step(2, 400, heads=2, batch=4, kv_len=(400, 161, 1, 0)),
    "padded-causal": Step(6, 120, chunk=1, offset=60, batch=3, kv_len=(120, 64, 0), dim=64),
    "tokens-outside-heads": Step(3, 210, heads=6, kv_heads=2, batch=2, layout="bnhd"),
    "many-heads": Step(1, 64, heads=300, dim=64),
    "long": Step(16, 20011, heads=2, kv_heads=1, dim=64),
}


@pytest.mark.parametrize("name", FEW)
def test_few_queries(name):
    c = FEW[name]
    q, k, v, do, kv_len = tensors(c, seed=4)
    ref, cost = reference(c, q, k, v, do)
    got = run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    print(f"  {name}: {check(c, got, ref, cost)}", flush=True)
