"""GPU: how the training step and rotary positions are called: tiles whose streamed rows several workgroups share, scratch
and outputs of the caller, streams, captured graphs, what hidden rows hold, far addresses, and the step as a whole."""
import dataclasses
import math

import numpy as np
import pytest
import torch

import paper_2602_12271_amd as pkg
from paper_2602_12271_amd import binding

from dense_training import Step, check, reference, run, tensors, units
from test_gpu_rotary import bound, positions_of, turned

pytestmark = pytest.mark.gpu

# more than 32 rows, too few tiles to fill the GPU: workgroups share a tile's streamed rows
SHARED = {
    "one-head": Step(1, 1, 25, 40, heads=1),
    "one-head-d64": Step(1, 1, 33, 31, heads=1, dim=64),
    "causal": Step(400, 400, chunk=1, heads=2),
    "chunks-shared-d64": Step(6, 6, 9, 13, heads=4, kv_heads=1, chunk=2, dim=64),
    "few-keys-many-queries": Step(1500, 70, heads=2),
    "cache": Step(2, 9, 10, 11, heads=2, chunk=2, offset=6),
    "padded": Step(300, 300, batch=3, heads=1, kv_len=(300, 33, 0)),
    "padded-causal-d64": Step(900, 900, batch=2, heads=1, chunk=1, kv_len=(890, 430), dim=64),
    "f32-one-head": Step(1, 1, 25, 40, heads=1, dtype="f32"),
    "f32-d64": Step(1, 1, 24, 24, heads=1, dim=64, dtype="f32"),
    "f32-causal-shared": Step(333, 333, heads=4, kv_heads=2, chunk=1, dtype="f32", dim=64),
    "f32-cache": Step(2, 9, 10, 11, chunk=2, offset=6, dtype="f32", heads=1),
    "f32-odd-dim": Step(260, 520, heads=1, dim=51, dtype="f32"),
    "f32-padded": Step(200, 200, batch=4, heads=1, kv_len=(200, 64, 1, 0), dtype="f32"),
    "f32-one-query": Step(1, 2000, heads=2, kv_heads=1, dtype="f32"),
    "bf16-in-f32": Step(260, 260, heads=1, compute=1, chunk=1),
}


def describe(c, q, k, v, do):
    """The binding's description of a call and its scratch, forward and backward."""
    args = dict(c.args)
    a = [args.pop(n) for n in ("f_q", "f_kv", "h", "w", "causal_chunk", "q_frame_offset", "scale", "compute")]
    fwd = binding._train_problem(q, k, v, torch.empty_like(q), (), *a)
    bwd = binding._train_problem(q, k, v, torch.empty_like(q), (do, torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)), *a)
    return fwd, bwd


@pytest.mark.parametrize("name", SHARED)
def test_shared_tiles(name):
    c = SHARED[name]
    q, k, v, do, kv_len = tensors(c, seed=7)
    fwd, bwd = describe(c, q, k, v, do)
    stats = 8 * c.batch * c.heads * -(-c.nq // 32) * 32
    assert bwd[2] > stats + 256, "no tile is shared"
    ref, cost = reference(c, q, k, v, do)
    got = run(c, q, k, v, do, kv_len)
    again = run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    print(f"  {name}: {check(c, got, ref, cost)}", flush=True)
    for n in got:
        assert torch.equal(got[n], again[n]), f"{n}: other bits in a second call"


@pytest.mark.parametrize("name", ["f32-one-head", "f32-causal-shared", "f32-padded", "f32-odd-dim", "f32-one-query"])
def test_forward_with_and_without_scratch(name):
    c = SHARED[name]
    q, k, v, do, kv_len = tensors(c, seed=8)
    need = describe(c, q, k, v, do)[0][2]
    assert need > 0
    ref, cost = reference(c, q, k, v, do)
    poisoned = torch.full((need,), 255, dtype=torch.uint8, device="cuda")       # (NaN in every number)
    ways = {"torch's": None, "the caller's": poisoned, "too little": poisoned[:max(need - 256, 0)]}
    got = {}
    for way, ws in ways.items():
        o, lse = pkg.dense_attn_fwd_save(q, k, v, kv_len=kv_len, workspace=ws, **c.args)
        torch.cuda.synchronize()
        got[way] = o, lse
        print(f"  {name}, {way}: {check(c, dict(O=o, lse=lse), ref, cost)}", flush=True)
    assert all(torch.equal(x, y) for x, y in zip(got["torch's"], got["the caller's"]))


FULL = {          # fp32 products where the queries fill the GPU, or do without scratch
    "bf16-rows": Step(150, 150, heads=2, compute=1),
    "bf16-rows-causal-shared-d64": Step(150, 150, heads=4, kv_heads=2, chunk=1, dim=64, compute=1),
    "bf16-rows-padded": Step(100, 100, heads=2, batch=3, kv_len=(100, 33, 0), compute=1),
    "d64": Step(150, 150, heads=2, dim=64, dtype="f32"),
    "padded-d64": Step(100, 100, heads=2, batch=3, kv_len=(100, 33, 0), dim=64, dtype="f32"),
    "many-heads": Step(300, 300, heads=32, kv_heads=4, batch=4, dim=64, dtype="f32"),
    "sharp-d64": Step(150, 150, heads=2, dim=64, dtype="f32", sigma=20.0),
    "sharp": Step(150, 150, heads=2, dtype="f32", sigma=20.0, chunk=1),
    "many-heads-causal": Step(260, 260, heads=60, batch=3, chunk=1, dim=32, dtype="f32"),
}


@pytest.mark.parametrize("name", FULL)
def test_forward_that_shares_nothing(name):
    c = FULL[name]
    q, k, v, do, kv_len = tensors(c, seed=14)
    ref, cost = reference(c, q, k, v, do)
    o, lse = pkg.dense_attn_fwd_save(q, k, v, kv_len=kv_len, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"), **c.args)
    torch.cuda.synchronize()
    print(f"  {name}: {check(c, dict(O=o, lse=lse), ref, cost)}", flush=True)


SHARP = {
    "bf16": Step(150, 150, heads=2, sigma=6.0),
    "bf16-d64-causal-shared": Step(150, 150, heads=4, kv_heads=2, dim=64, chunk=1, sigma=6.0),
    "bf16-few": Step(3, 400, heads=2, sigma=6.0),
    "f32": Step(150, 150, heads=2, sigma=10.0, dtype="f32"),
    "f32-causal-d64": Step(150, 150, heads=2, sigma=10.0, dtype="f32", dim=64, chunk=1),
}


@pytest.mark.parametrize("name", SHARP)
def test_sharp_rows(name):
    """Logits of several hundred: rows whose weight lies on one or two keys."""
    c = SHARP[name]
    q, k, v, do, kv_len = tensors(c, seed=15)
    ref, cost = reference(c, q, k, v, do)
    got = run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    print(f"  {name}: {check(c, got, ref, cost)}", flush=True)


FEW_KEYS = {
    "causal-10": Step(10, 10, heads=8, chunk=1),
    "causal-33-shared": Step(33, 33, heads=8, kv_heads=2, batch=2, chunk=1, dim=64),
    "queries-16-of-4": Step(16, 4, heads=8),
    "queries-50-of-32": Step(50, 32, heads=4, dim=64),
    "two-keys": Step(3, 2, heads=30, batch=2),
    "causal-offset": Step(20, 60, heads=6, chunk=1, offset=9),
    "frames": Step(4, 4, 3, 3, heads=8, chunk=1),
    "padded": Step(40, 40, heads=6, batch=4, kv_len=(40, 32, 5, 1)),
}


@pytest.mark.parametrize("name", FEW_KEYS)
def test_rows_of_few_keys(name):
    """Rows that see few keys: O's rounding to bf16 does not reach dQ and dK, so that their error is that of two
    roundings, dS's and the result's: 2^-9 sqrt(4/3) of the 2-norm each at the most unlucky mantissas, 1.5 of a typical
    1.66e-3 in all (over a single key dQ and dK are zero: such a sequence is left out of the norm)."""
    c = FEW_KEYS[name]
    q, k, v, do, kv_len = tensors(c, seed=16)
    ref, cost = reference(c, q, k, v, do)
    got = run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    check(c, got, ref, cost)
    for n in ("dQ", "dK"):
        off = float((got[n].double() - ref[n]).norm() / ref[n].norm())
        print(f"  {name} {n}: {off:.2e}", flush=True)
        assert off <= 2 * 2.0 ** -9 * math.sqrt(4 / 3)


CALLS = {
    "bf16": Step(2, 2, 12, 13, heads=3, batch=2),
    "bf16-d64-shared-heads": Step(350, 350, heads=4, kv_heads=2, chunk=1, dim=64),
    "bf16-few": Step(3, 500, heads=6, kv_heads=3),
    "bf16-shared-tiles": SHARED["one-head"],
    "f32": Step(2, 2, 8, 9, heads=2, dim=64, dtype="f32"),
    "f32-shared-tiles": SHARED["f32-d64"],
    "f32-elements": Step(1, 1, 9, 9, heads=2, dim=37, dtype="f32"),
}


@pytest.mark.parametrize("name", CALLS)
def test_callers_memory(name):
    """Gradients into views of larger tensors, scratch full of NaN: the same bits, nothing else written."""
    c = CALLS[name]
    q, k, v, do, kv_len = tensors(c, seed=9)
    want = run(c, q, k, v, do, kv_len)
    need = describe(c, q, k, v, do)[1][2]
    ws = torch.full((need + 512,), 255, dtype=torch.uint8, device="cuda")
    ws[need:] = 77
    big, views = [], []
    for x in (q, k, v, q):
        b, h, n, d = x.shape
        y = torch.full((b, n + 3, h + 1, -(-(d + 8) // 8) * 8), 3.0, dtype=x.dtype, device="cuda")
        big.append(y)
        views.append(y[:, :n, :h, :d].transpose(1, 2))
    stats = torch.full((q[..., 0].numel() + 32,), 3.0, device="cuda")
    lse = stats[:-32].view(q.shape[:3])
    o, lse2 = pkg.dense_attn_fwd_save(q, k, v, kv_len=kv_len, out=views[3], lse=lse, **c.args)
    assert o is views[3] and lse2 is lse
    grads = pkg.dense_attn_bwd(q, k, v, o, do, lse, kv_len=kv_len, out=tuple(views[:3]), workspace=ws, **c.args)
    torch.cuda.synchronize()
    for n, x in zip(("O", "lse", "dQ", "dK", "dV"), (o, lse, *grads)):
        assert torch.equal(x, want[n]), n
    for y, x in zip(big, views):
        x.fill_(3.0)
        assert (y == 3.0).all(), "written outside of the output"
    assert (stats[-32:] == 3.0).all() and (ws[need:] == 77).all()


@pytest.mark.parametrize("name", CALLS)
def test_streams(name):
    """Another stream than torch's current one; two calls at once on two streams."""
    c = CALLS[name]
    sets = [tensors(c, seed=s) for s in (1, 2)]
    want = [run(c, *x) for x in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = []
        for s, x in zip(streams, sets):
            q, k, v, do, kv_len = x
            o, lse = pkg.dense_attn_fwd_save(q, k, v, kv_len=kv_len, stream=s.cuda_stream, **c.args)
            got.append((o, lse, *pkg.dense_attn_bwd(q, k, v, o, do, lse, kv_len=kv_len, stream=s.cuda_stream, **c.args)))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for n, x in zip(("O", "lse", "dQ", "dK", "dV"), g):
                assert torch.equal(x, w[n]), n
        del got


@pytest.mark.parametrize("name", CALLS)
def test_captured(name):
    """Rotary positions and the step in a captured graph: every replay as the eager calls, on the inputs it finds."""
    c = CALLS[name]
    even = c.dim - c.dim % 2
    split = (even // 2, 0, 0)
    grid = dict(f_q=c.f_q, f_kv=c.f_kv, h=c.h, w=c.w, split=split)
    q, k, v, do, kv_len = tensors(c, seed=3)
    (_, _, nf), (_, _, nb) = describe(c, q, k, v, do)
    own = [torch.empty(max(n, 1), dtype=torch.uint8, device="cuda") for n in (nf, nb)]

    def step(q, k, v, do, scratch):
        a, b = scratch
        qr, kr = pkg.rotary_fwd(q, k, **grid)
        o, lse = pkg.dense_attn_fwd_save(qr, kr, v, workspace=a if nf else None, **c.args)
        dq, dk, dv = pkg.dense_attn_bwd(qr, kr, v, o, do, lse, workspace=b, **c.args)
        return (qr, kr, o, lse, *pkg.rotary_bwd(dq, dk, **grid), dv)
    step(q, k, v, do, own)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(q, k, v, do, own)
    for replay in range(4):
        fresh = tensors(c, seed=20 + replay)
        for x, y in zip((q, k, v, do), fresh):
            x.copy_(y)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = step(*fresh[:4], (torch.empty_like(own[0]), None))
        torch.cuda.synchronize()
        for n, (x, y) in enumerate(zip(out, eager)):
            assert torch.equal(x, y), f"replay {replay}, output {n}"


@pytest.mark.parametrize("name", ["f32-d64", "f32-one-query", "one-head"])
def test_captured_without_scratch(name):
    c = SHARED[name]
    q, k, v, do, kv_len = tensors(c, seed=3)
    run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(c, q, k, v, do, kv_len)
    ref, cost = reference(c, q, k, v, do)
    for _ in range(2):
        for x in got.values():
            x.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        check(c, got, ref, cost)


NOWHERE = {
    "bf16": Step(90, 90, batch=3, heads=2, kv_len=(90, 41, 0)),
    "bf16-d64": Step(200, 200, batch=2, heads=4, kv_heads=2, kv_len=(70, 129), dim=64),
    "bf16-causal": Step(150, 150, batch=2, chunk=1, kv_len=(97, 3)),
    "bf16-shared-tiles": SHARED["padded"],
    "few": Step(2, 400, batch=3, kv_len=(400, 161, 0)),
    "few-d64": Step(9, 130, heads=2, kv_heads=1, batch=2, kv_len=(65, 1), dim=64),
    "f32": Step(75, 75, batch=3, kv_len=(75, 30, 0), dtype="f32"),
    "f32-causal": Step(150, 150, batch=2, chunk=1, kv_len=(97, 3), dtype="f32", dim=64),
    "f32-shared-tiles": SHARED["f32-padded"],
    "f32-full-chip": Step(520, 520, batch=8, heads=16, dim=64, kv_len=(520, 519, 300, 256, 64, 17, 1, 0), dtype="f32"),
}


@pytest.mark.parametrize("name", NOWHERE)
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_padding_holds_anything(name, value):
    c = NOWHERE[name]
    q, k, v, do, kv_len = tensors(c, seed=5)
    want = run(c, q, k, v, do, kv_len)
    for b, n in enumerate(c.kv_len):
        k[b, :, n:], v[b, :, n:] = value, -value
    got = run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    for n in got:
        assert torch.equal(got[n], want[n]), n
    for b, n in enumerate(c.kv_len):
        assert (got["dK"][b, :, n:] == 0).all() and (got["dV"][b, :, n:] == 0).all()


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("f_q,offset", [(3, 1), (1, 0), (2, 2)])
def test_keys_that_no_query_sees(dtype, dim, f_q, offset):
    """Frames behind the last visible one hold NaN: nothing shows, and their gradients are zero."""
    c = Step(f_q, 12, 5, 7, chunk=2, offset=offset, dtype=dtype, dim=dim)
    q, k, v, do, _ = tensors(c, seed=6)
    want = run(c, q, k, v, do, None)
    end = ((offset + f_q - 1) // 2 + 1) * 2 * 35
    k[:, :, end:], v[:, :, end:] = math.nan, math.nan
    got = run(c, q, k, v, do, None)
    torch.cuda.synchronize()
    for n in got:
        assert torch.equal(got[n], want[n]), n
    assert (got["dK"][:, :, end:] == 0).all() and (got["dV"][:, :, end:] == 0).all()


@pytest.mark.parametrize("dtype,far", [("bf16", 1 << 24), ("f32", 1 << 24), ("f32", 1 << 25)])
def test_far_addresses(dtype, far):
    """Rows 2^24 or 2^25 elements apart: tensors that reach past 2^31 elements, all of them in one allocation."""
    n = 70
    c = Step(1, 1, 7, 10, heads=3, batch=2, dim=64, dtype=dtype)
    q, k, v, do, _ = tensors(c, seed=11)
    want = run(c, q, k, v, do, None)
    turned_near = pkg.rotary_fwd(q, k, f_q=1, f_kv=1, h=7, w=10)
    memory = torch.empty(2 * n * far, dtype=q.dtype, device="cuda")
    assert memory.numel() > 1 << 31
    slots = [memory.as_strided((2, 3, n, 64), (n * far, 64, far, 1), i * (far // 16)) for i in range(10)]
    for x, y in zip(slots, (q, k, v, do)):
        x.copy_(y)
    fq, fk, fv, fdo, fo = slots[:5]
    o, lse = pkg.dense_attn_fwd_save(fq, fk, fv, out=fo, **c.args)
    grads = pkg.dense_attn_bwd(fq, fk, fv, o, fdo, lse, out=tuple(slots[5:8]), **c.args)
    both = pkg.rotary_fwd(fq, fk, f_q=1, f_kv=1, h=7, w=10, out=slots[8], k_out=slots[9])
    torch.cuda.synchronize()
    for name, x in zip(("O", "lse", "dQ", "dK", "dV"), (o, lse, *grads)):
        assert torch.equal(x, want[name]), name
    assert all(torch.equal(x, y) for x, y in zip(both, turned_near))


@pytest.mark.parametrize("name", [dict(dim=64), dict(dim=33, chunk=1, kv_heads=1)], ids=["dim-64", "odd-dim-causal-shared"])
def test_gradient_against_differences(name):
    """Central differences of the kernels' own forward pass along the gradients of the formulas, where the slope is steepest.

    They are off by their truncation, which the same differences of the formulas in 64 bits show, and by the roundings of
    two outputs, units() of sum |O| |dO| each, over twice the step; the gradient by its own bound, along the direction."""
    c = Step(40, 40, heads=2, dtype="f32", **name)
    q, k, v, do, _ = tensors(c, seed=12)
    ref, costs = reference(c, q, k, v, do)
    got = run(c, q, k, v, do, None)
    eps, (_, sums) = 2.0 ** -4, units(c)
    for i, grad in enumerate(("dQ", "dK", "dV")):
        inputs = [q, k, v]
        way = (ref[grad] / ref[grad].square().mean().sqrt()).float()
        ends, exact, noise = [], [], 0.0
        for sign in (1, -1):
            moved = list(inputs)
            moved[i] = inputs[i] + sign * eps * way
            o, _ = pkg.dense_attn_fwd_save(*moved, **c.args)
            r, cost = reference(c, *moved, do)
            ends.append(float((o.double() * do.double()).sum()))
            exact.append(float((r["O"] * do.double()).sum()))
            noise += float((cost[0]["O"] * do.double().abs()).sum()) * 2 * sums
        slope, true_slope = (ends[0] - ends[1]) / (2 * eps), (exact[0] - exact[1]) / (2 * eps)
        moved = [(inputs[i] + s * eps * way).double() for s in (1, -1)]
        step = (moved[0] - moved[1]) / (2 * eps)                   # the way taken, after the rounding of the inputs
        along = float((got[grad].double() * step).sum())
        cut = abs(true_slope - float((ref[grad] * step).sum()))
        own = float(((sums * costs[0][grad] + (2.0 ** -24 + sums) * costs[1][grad] + 2.0 ** -24 * ref[grad].abs()) * step.abs()).sum())
        assert abs(slope - along) <= cut + noise / (2 * eps) + own, (grad, slope, along)
        assert cut + noise / (2 * eps) + own <= 0.1 * abs(along), "the bound says nothing"


# ---- rotary positions ----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["adjacent", "halves"])
def test_rotary_in_place_and_into_a_cache(dtype, layout):
    q, k = (torch.randn(2, h, 60, 64, device="cuda").to(dtype) for h in (4, 2))
    args = dict(f_q=2, h=5, w=6, layout=layout, q_frame_offset=3, kv_frame_offset=3)
    want = pkg.rotary_fwd(q, k, **args)
    cache = torch.full((2, 2, 300, 64), 9.0, device="cuda").to(dtype)
    mine = q.clone()
    got = pkg.rotary_fwd(mine, k, out=mine, k_out=cache[:, :, 90:150], **args)
    torch.cuda.synchronize()
    assert got[0] is mine and torch.equal(mine, want[0]) and torch.equal(cache[:, :, 90:150], want[1])
    assert (cache[:, :, :90] == 9).all() and (cache[:, :, 150:] == 9).all()
    packed = torch.randn(2, 60, 3, 4, 64, device="cuda").to(dtype)
    a, b = packed[:, :, 0].transpose(1, 2), packed[:, :, 1].transpose(1, 2)
    want, values = pkg.rotary_fwd(a, b, **args), packed[:, :, 2].clone()
    pkg.rotary_fwd(a, b, out=a, k_out=b, **args)
    torch.cuda.synchronize()
    assert torch.equal(a, want[0]) and torch.equal(b, want[1]) and torch.equal(packed[:, :, 2], values)


def test_rotary_farthest_positions():
    """Positions at both ends of 32 bits.  The angle's 64-bit factor and product are rounded by 2^-53 each, of up to 2^31
    radians: 4.8e-7, and its last turn to 32 bits by 1e-7."""
    at = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 9 + 7, -123456789, 99999999], dtype=torch.int32)
    x = torch.randn(1, 2, 8, 24)
    got = pkg.rotary_fwd(x.cuda(), split=(4, 4, 4), q_positions=at.expand(3, 8).contiguous().cuda())
    torch.cuda.synchronize()
    freq = np.longdouble(10000) ** (-np.arange(4, dtype=np.longdouble) / 4)
    angle = np.tile(at.numpy().astype(np.longdouble)[:, None] * freq, (1, 3))
    turns = angle / (2 * np.longdouble("3.14159265358979323846264338327950288"))
    angle = torch.from_numpy(((turns - np.rint(turns)) * 2 * np.longdouble("3.14159265358979323846264338327950288")).astype(np.float64))
    a, b = x[..., 0::2].double(), x[..., 1::2].double()
    want = torch.stack((a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()), -1).reshape(x.shape)
    off = (got.cpu().double() - want).abs() / (bound(x.double(), torch.float32, (4, 4, 4), "adjacent") * (7e-7 + 8 * 2.0 ** -24) / (1e-7 + 8 * 2.0 ** -24))
    assert off.max() <= 1


def test_rotary_large_batch_of_small_tokens():
    x = torch.randn(5000, 1, 1, 32, device="cuda", dtype=torch.bfloat16)
    at = torch.arange(5000, device="cuda", dtype=torch.int32).view(5000, 1, 1).expand(5000, 3, 1).contiguous()
    got = pkg.rotary_fwd(x, q_positions=at)
    want = pkg.rotary_fwd(x.permute(1, 2, 0, 3), q_positions=at.view(5000, 3).t().contiguous())
    torch.cuda.synchronize()
    assert torch.equal(got, want.permute(2, 0, 1, 3))


# ---- the step as a whole ------------------------------------------------------------------------
def autograd(c, q, k, v, do, split):
    """Rotary positions and the attention in 64 bits on the host: gradients by automatic differentiation."""
    q, k, v = (x.cpu().double().requires_grad_() for x in (q, k, v))

    def turn(x, frames):
        at = positions_of(frames, c.h, c.w, 0).double()
        axis = torch.repeat_interleave(torch.arange(3), torch.tensor(split))
        e = torch.cat([torch.arange(n).double() / max(n, 1) for n in split])
        angle = at[axis].t() * 1e4 ** -e
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()), -1).reshape(x.shape)
    qr, kr = turn(q, c.f_q), turn(k, c.f_kv)
    group = c.heads // (c.kv_heads or c.heads)
    kr, vr = kr.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    s = c.args["scale"] * qr @ kr.transpose(2, 3)
    from dense_training import hidden
    off = torch.stack([hidden(c, b, "cpu") for b in range(c.batch)])[:, None]
    p = torch.softmax(s.masked_fill(off, -1e300), -1).masked_fill(off, 0.0)
    o = p @ vr
    (o * do.cpu().double()).sum().backward()
    return o.detach(), q.grad, k.grad, v.grad


WHOLE = {
    "f32": Step(2, 2, 6, 7, heads=2, dim=64, dtype="f32"),
    "f32-causal-shared": Step(4, 4, 5, 6, heads=4, kv_heads=2, chunk=2, dim=128, dtype="f32"),
    "f32-padded": Step(3, 3, 4, 5, heads=2, batch=3, dim=64, dtype="f32", kv_len=(60, 17, 0)),
    "bf16": Step(2, 2, 6, 7, heads=2),
    "bf16-causal-shared": Step(4, 4, 5, 6, heads=4, kv_heads=2, chunk=2, dim=64),
    "bf16-padded": Step(3, 3, 4, 5, heads=2, batch=3, dim=64, kv_len=(60, 17, 0)),
}


@pytest.mark.parametrize("name", WHOLE)
def test_whole_step(name):
    """Rotary positions, forward, backward, and the turn back of the gradients.

    fp32 against 64-bit automatic differentiation: turned entries are off by 1.2e-6 of their pair (bound()), logits of
    magnitude 4 sqrt(dim) |q| |k| scale < 50 by 2e-6 of it, 1e-4 at the very worst; errors of that kind that all point
    one way do not occur, 2e-5 in the 2-norm is 30 roundings of a typical logit.  bf16: each call against 64 bits on what
    it was given, where the roundings have bounds entry by entry."""
    c = WHOLE[name]
    split = binding.rotary_pairs_split(c.dim)
    grid = dict(f_q=c.f_q, f_kv=c.f_kv, h=c.h, w=c.w)
    q, k, v, do, kv_len = tensors(c, seed=13)
    qr, kr = pkg.rotary_fwd(q, k, **grid)
    got = run(c, qr, kr, v, do, kv_len)
    dq, dk = pkg.rotary_bwd(got["dQ"], got["dK"], **grid)
    torch.cuda.synchronize()
    check(c, got, *reference(c, qr, kr, v, do))
    for x, y, frames, sign in ((q, qr, c.f_q, 1), (k, kr, c.f_kv, 1), (got["dQ"], dq, c.f_q, -1), (got["dK"], dk, c.f_kv, -1)):
        x = x.cpu().double()
        want = turned(x, positions_of(frames, c.h, c.w, 0), split, 1e4, "adjacent", "axis", sign)
        live = slice(0, 2 * sum(split))
        off = (y.cpu().double() - want).abs()[..., live] / bound(x, y.dtype, split, "adjacent")[..., live]
        assert off.max() <= 1
    if c.dtype == "f32":
        for x, want in zip((got["O"], dq, dk, got["dV"]), autograd(c, q, k, v, do, split)):
            assert float((x.cpu().double() - want).norm()) <= 2e-5 * float(want.norm())
