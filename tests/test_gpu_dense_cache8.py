"""GPU: dense attention over a cache of 8 bits.  The cache's values are bf16 numbers, so that the definition and the bounds
of the attention over bf16 keys (dense_training.py) hold as they are."""
import dataclasses
import math

import pytest
import torch

import paper_2602_12271_amd as pkg
from dense_training import Step, check, reference, tensors

pytestmark = pytest.mark.gpu


def cached(c: Step, seed=0, format="e4m3", block=64, extra=0):
    """Q, a cache of K and V (with `extra` tokens of room), its values, kv_len."""
    q, k, v, do, kv_len = tensors(c, seed=seed)
    cache = pkg.cache8(c.batch, k.shape[1], c.nkv + extra, c.dim, format=format, block=block)
    pkg.cache8_write(cache, k.contiguous(), v.contiguous())
    return q, cache, *pkg.cache8_read(cache, c.nkv), do, kv_len


def attend(c: Step, q, cache, kv_len=None, **kw):
    args = {n: x for n, x in c.args.items() if n != "compute"}
    return dict(zip(("O", "lse"), pkg.dense_attn_fwd_cache8(q, cache, kv_len=kv_len, **args, **kw)))


CASES = {
    # one token and a few: their keys shared by workgroups, or few enough for one
    "token": Step(1, 700, heads=4, batch=2),
    "token-shared": Step(1, 1500, heads=32, kv_heads=8),
    "token-shared-d64": Step(1, 2500, heads=8, kv_heads=1, dim=64, batch=2),
    "token-all-share-one": Step(1, 900, heads=40, kv_heads=1),
    "token-one-key": Step(1, 1, heads=5, batch=3),
    "token-two-keys": Step(1, 2, heads=4, kv_heads=2),
    "token-31-keys": Step(1, 31, heads=4, kv_heads=4, dim=64),
    "token-33-keys": Step(1, 33, heads=4, kv_heads=4),
    "token-padded": Step(1, 1000, heads=6, kv_heads=3, batch=5, kv_len=(1000, 1, 0, 517, 64)),
    "token-lengths": Step(1, 4000, heads=2, kv_heads=1, batch=100, dim=64, kv_len=tuple(i * i * 31 % 4001 for i in range(100))),
    "token-fills": Step(1, 600, heads=16, kv_heads=8, batch=40, dim=64, kv_len=tuple(i * 77 % 601 for i in range(40))),
    "token-fills-4-rows": Step(4, 500, heads=16, kv_heads=1, batch=200, dim=64, kv_len=(500,) + (0, 7) * 99 + (499,)),
    "token-fills-parted": Step(1, 600, heads=16, kv_heads=8, batch=40, kv_len=tuple(i * 77 % 601 for i in range(40))),
    "token-fills-4-rows-parted": Step(4, 1100, heads=16, kv_heads=1, batch=200, dim=64, kv_len=(1100,) + (0, 7) * 99 + (1099,)),
    "token-one-long": Step(1, 20000, heads=8, kv_heads=1, batch=16, kv_len=(3, 0, 20000) + (0, 1, 33) * 4 + (0,)),
    "token-long-last": Step(1, 9000, heads=4, kv_heads=2, batch=3, kv_len=(0, 0, 8999)),
    "few-lengths-causal": Step(5, 900, heads=4, kv_heads=1, chunk=1, offset=880, batch=7, kv_len=(884, 1, 0, 881, 64, 900, 300)),
    "token-padded-d64": Step(1, 300, heads=6, kv_heads=6, dim=64, batch=4, kv_len=(-5, 300, 900, 129)),
    "token-long": Step(1, 40000, heads=2, kv_heads=1),
    "few-3": Step(3, 777, heads=4, kv_heads=2),
    "few-7-shared": Step(7, 1025, heads=12, kv_heads=3, batch=2),
    "few-16-d64": Step(16, 640, heads=2, dim=64),
    "few-16-shared": Step(16, 1300, heads=16, kv_heads=2),
    "few-17": Step(17, 400, heads=3),
    "few-24-many": Step(24, 300, heads=140, kv_heads=70),
    "few-20-all-share-one": Step(20, 900, heads=40, kv_heads=1),
    "few-33-shared-d64": Step(33, 500, heads=8, kv_heads=4, dim=64),
    "few-causal": Step(5, 205, heads=4, kv_heads=2, chunk=1, offset=200),
    "few-causal-from-0": Step(9, 9, heads=4, kv_heads=2, chunk=1),
    "few-causal-padded": Step(6, 300, heads=4, kv_heads=1, chunk=1, offset=250, batch=3, kv_len=(300, 252, 0)),
    "few-frames": Step(3, 9, 2, 3, heads=4, chunk=3, offset=3),
    "few-offset-beyond": Step(4, 100, heads=2, chunk=1, offset=5000),
    # many rows
    "frame": Step(1, 5, 13, 17, heads=3),
    "frame-d64": Step(1, 5, 13, 17, heads=3, dim=64),
    "chunk-cache": Step(3, 9, 10, 11, heads=2, chunk=3, offset=6),
    "clip": Step(6, 6, 9, 13, heads=4, kv_heads=1, chunk=2, dim=64),
    "clip-one-frame-chunks": Step(4, 7, 8, 9, heads=2, chunk=1, offset=3),
    "text": Step(400, 400, heads=4, kv_heads=2, chunk=1),
    "text-late": Step(150, 900, heads=2, chunk=1, offset=740),
    "padded": Step(300, 300, batch=3, heads=2, kv_len=(300, 33, 0)),
    "padded-d64": Step(90, 450, batch=4, heads=4, kv_heads=2, dim=64, kv_len=(450, 449, 64, 1)),
    "padded-by-length": Step(700, 700, heads=12, kv_heads=4, batch=5, kv_len=(699, 64, 0, 700, 700)),
    "padded-by-length-d64": Step(2, 2, 17, 23, heads=10, batch=6, dim=64, kv_len=(1, 0, 782, 500, 781, 65)),
    "padded-shared": Step(390, 1500, heads=4, kv_heads=2, batch=4, kv_len=(1500, 40, 0, 700)),
    "padded-64": Step(40, 200, heads=2, batch=64, kv_len=tuple(i * 37 % 201 for i in range(64))),
    "padded-65": Step(40, 200, heads=2, batch=65, kv_len=tuple(i * 37 % 201 for i in range(65))),
    "padded-causal": Step(200, 200, batch=2, heads=1, chunk=1, kv_len=(190, 30)),
    "many-heads": Step(260, 520, heads=48, kv_heads=6, batch=2),
    "tokens-outside": Step(70, 140, heads=4, layout="bnhd"),
    "sharp": Step(40, 300, heads=2, sigma=6.0),
    "sharp-token": Step(1, 600, heads=4, kv_heads=2, sigma=6.0),
    "scale": Step(3, 300, heads=2, scale=0.02),
}


@pytest.mark.parametrize("format,block", [("e4m3", 64), ("int8", 32), ("e4m3", 16), ("int8", 128)])
@pytest.mark.parametrize("name", CASES)
def test_attention(name, format, block):
    c = CASES[name]
    q, cache, k, v, do, kv_len = cached(c, seed=1, format=format, block=block, extra=5)
    got = attend(c, q, cache, kv_len)
    again = attend(c, q, cache, kv_len)
    torch.cuda.synchronize()
    ref, cost = reference(c, q, k, v, do)
    print(f"  {name}: {check(c, got, ref, cost)}", flush=True)
    for n in got:
        assert torch.equal(got[n], again[n]), f"{n}: other bits in a second call"
    # in the 2-norm of a head: two roundings of independent signs, of the weights and of the result, 2^-9 sqrt(4/3) each at
    # the most unlucky mantissas; where few keys weigh they need not average, so that four times that is allowed
    for b in range(c.batch):
        for h in range(c.heads):
            want = ref["O"][b, h]
            assert (got["O"][b, h].double() - want).norm() <= 4 * 2.0 ** -9 * math.sqrt(8 / 3) * want.norm() + 1e-30


@pytest.mark.parametrize("name", ["token", "token-shared", "token-padded", "token-lengths", "token-fills-parted", "token-one-long", "few-7-shared", "few-16-d64", "few-causal-padded", "frame",
                                  "chunk-cache", "padded", "padded-by-length", "padded-by-length-d64", "padded-64", "text-late"])
def test_scratch(name):
    """The caller's scratch, poisoned; too little, or none: the same work with fewer workgroups."""
    c = CASES[name]
    q, cache, k, v, do, kv_len = cached(c, seed=2)
    args = {n: x for n, x in c.args.items() if n != "compute"}
    need = pkg.dense_attn_fwd_cache8_workspace_bytes(q, cache, **args)
    ref, cost = reference(c, q, k, v, do)
    poisoned = torch.full((max(need, 256),), 255, dtype=torch.uint8, device="cuda")
    got = {}
    for way, ws in (("torch's", None), ("own", poisoned), ("too little", poisoned[:max(need - 256, 0)]), ("none", poisoned[:0])):
        got[way] = attend(c, q, cache, kv_len, workspace=ws)
        torch.cuda.synchronize()
        check(c, got[way], ref, cost)
    assert all(torch.equal(got["torch's"][n], got["own"][n]) for n in ("O", "lse"))


@pytest.mark.parametrize("name", ["token-padded", "token-padded-d64", "few-causal-padded", "padded", "padded-d64", "padded-causal"])
@pytest.mark.parametrize("format", ["e4m3", "int8"])
def test_padding_holds_anything(name, format):
    """NaN codes and any scale bytes behind a sequence's end, as memory that nothing was written to holds them; the last
    block's scale belongs to its live rows."""
    c = CASES[name]
    q, cache, k, v, do, kv_len = cached(c, seed=3, format=format, block=32, extra=40)
    want = attend(c, q, cache, kv_len)
    for b, n in enumerate(c.kv_len):
        n = min(max(n, 0), c.nkv)
        for x in cache[:2]:
            x.view(torch.uint8)[b, :, n:] = 0x7f if format == "e4m3" else 0x80
        for x in cache[2:4]:
            x[b, :, -(-n // 32):] = 255
    got = attend(c, q, cache, kv_len)
    torch.cuda.synchronize()
    for n in got:
        assert torch.equal(got[n], want[n]), n


@pytest.mark.parametrize("f_q,offset", [(3, 1), (1, 0), (2, 2)])
@pytest.mark.parametrize("hw", [(5, 7), (1, 1), (2, 2)])
def test_keys_that_no_query_sees(f_q, offset, hw):
    c = Step(f_q, 40, *hw, chunk=2, offset=offset)
    q, cache, *_ = cached(c, seed=4, block=16)
    want = attend(c, q, cache)
    end = ((offset + f_q - 1) // 2 + 1) * 2 * hw[0] * hw[1]
    for x in cache[:2]:
        x.view(torch.uint8)[:, :, end:] = 0x7f
    got = attend(c, q, cache)
    torch.cuda.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in got)


def test_hidden_nan_of_other_rows():
    """A NaN value seen by a later chunk of queries only: earlier ones beyond its run of 256 are as ever."""
    c = Step(2, 2, 16, 40, heads=1, chunk=1)
    q, cache, *_ = cached(c, seed=5)
    want = attend(c, q, cache)
    cache.V.view(torch.uint8)[:, :, 700] = 0x7f
    got = attend(c, q, cache)
    torch.cuda.synchronize()
    assert got["O"][:, :, 640:].isnan().all() and torch.equal(got["O"][:, :, :512], want["O"][:, :, :512])


ROUNDS = {
    # tiles of queries beside the chip's 256 units: a few behind full rounds, which share their keys between many; most of a
    # round, whose second parts the units without a tile take; lengths of their own, an empty one among them
    "few-behind": Step(1, 1, 47, 69, heads=20),
    "few-behind-d64": Step(1, 1, 47, 69, heads=21, dim=64),
    "most-of-a-round": Step(1, 120, 10, 25, heads=234, kv_heads=2),
    "most-of-a-round-d64": Step(1, 120, 10, 25, heads=234, kv_heads=2, dim=64),
    "odd-tiles-padded": Step(1, 1, 41, 77, heads=10, batch=2, kv_len=(3000, 1033)),
    "padded-empty": Step(1, 1, 47, 69, heads=5, kv_heads=1, batch=4, kv_len=(3243, 0, 100, 1)),
    "padded-empty-d64": Step(1, 1, 47, 69, heads=5, kv_heads=1, dim=64, batch=4, kv_len=(3243, 0, 100, 1)),
    "masked-alike": Step(3, 6, 22, 49, heads=20, chunk=3, offset=3),
}


@pytest.mark.parametrize("name", ROUNDS)
@pytest.mark.parametrize("format", ["e4m3", "int8"])
def test_last_round(name, format):
    """Calls whose last round of workgroups is shared: the same as without scratch, up to roundings, everywhere."""
    c = ROUNDS[name]
    q, cache, k, v, do, kv_len = cached(c, seed=13, format=format)
    got = attend(c, q, cache, kv_len)
    again = attend(c, q, cache, kv_len)
    alone = attend(c, q, cache, kv_len, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    ref, cost = reference(c, q, k, v, do)
    print(f"  {name}: {check(c, got, ref, cost)}", flush=True)
    check(c, alone, ref, cost)
    for n in got:
        assert torch.equal(got[n], again[n])


def test_some_calls_share_their_last_round():
    """Scratch of the rows of the tiles behind full rounds, not of all rows."""
    for name in ("few-behind", "few-behind-d64", "masked-alike"):
        c = ROUNDS[name]
        q, cache, *_ = cached(c, seed=13)
        args = {n: x for n, x in c.args.items() if n != "compute"}
        need = pkg.dense_attn_fwd_cache8_workspace_bytes(q, cache, **args)
        row = (c.dim + 2) * 4
        print(f"  {name}: {need / row:.0f} rows of parts", flush=True)
        assert need > 0 and need % (c.heads * c.nq * row) != 0 and need % (64 * row) == 0, name


def test_same_bits_as_over_bf16_keys():
    """Calls under a mask that parts the queries are those of the training step over the cache's values."""
    for c in (Step(6, 6, 9, 13, heads=4, kv_heads=1, chunk=2), Step(700, 700, heads=4, kv_heads=2, chunk=1),
              Step(700, 700, heads=4, kv_heads=2, chunk=1, dim=64)):
        for format in ("e4m3", "int8"):
            q, cache, k, v, *_ = cached(c, seed=6, format=format)
            got = attend(c, q, cache)
            o, lse = pkg.dense_attn_fwd_save(q, k, v, **c.args)
            torch.cuda.synchronize()
            assert torch.equal(got["O"], o) and torch.equal(got["lse"], lse)


@pytest.mark.parametrize("name", ["token-shared", "few-7-shared", "chunk-cache", "padded"])
def test_streams_and_outputs(name):
    c = CASES[name]
    sets = [cached(c, seed=s) for s in (7, 8)]
    want = [attend(c, q, cache, kv_len) for q, cache, _, _, _, kv_len in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        got = [attend(c, x[0], x[1], x[5], stream=s.cuda_stream) for s, x in zip(streams, sets)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            assert all(torch.equal(g[n], w[n]) for n in g)
    q, cache, _, _, _, kv_len = sets[0]
    memory = torch.full((c.batch, c.nq, c.heads, c.dim + 8), 7.0, dtype=q.dtype, device="cuda")
    out = memory.transpose(1, 2)[..., :c.dim]
    lse = torch.empty(q.shape[:3], device="cuda")
    attend(c, q, cache, kv_len, out=out, lse=lse)
    inplace = q.clone()
    attend(c, inplace, cache, kv_len, out=inplace)
    torch.cuda.synchronize()
    assert torch.equal(out, want[0]["O"]) and torch.equal(lse, want[0]["lse"]) and (memory[..., c.dim:] == 7).all()
    assert torch.equal(inplace, want[0]["O"])


def test_views_of_a_cache():
    """The middle of a longer cache's heads and sequences; an interleaved layout; far tokens, past 2^31 bytes."""
    c = Step(2, 300, heads=4, kv_heads=2, batch=2)
    q, cache, k, v, do, _ = cached(c, seed=9, block=32)
    want = attend(c, q, cache)
    wide = [torch.zeros(4, 6, 300, 128, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.zeros(4, 6, 10, dtype=torch.uint8, device="cuda") for _ in range(2)]
    part = [x[1:3, 2:4] for x in (*wide, *scales)]
    far = 1 << 24
    memory = torch.empty(2 * 300 * far // 2, dtype=torch.uint8, device="cuda")
    assert memory.numel() > 1 << 31
    views = [memory.as_strided((2, 2, 300, 128), (150 * far, 128, far // 4, 1), i * 4096).view(torch.int8).view(torch.float8_e4m3fn) for i in range(2)]
    for dst in (part, [*views, cache.K_scale, cache.V_scale]):
        for x, y in zip(dst, cache[:4]):
            x.view(torch.uint8).copy_(y.view(torch.uint8))
        got = attend(c, q, pkg.Cache8(*dst, 32))
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in got)


def test_captured_decoding():
    """A decoding loop in a captured graph: norm and rotary positions, the token's row into the cache at its own place, the
    attention over what there is; every replay as the eager calls and as the definition of the whole."""
    B, H, KH, d, room = 3, 8, 2, 128, 400
    gen = torch.Generator().manual_seed(10)

    def token():
        x = [torch.randn(B, h, 1, d, generator=gen).bfloat16().cuda() for h in (H, KH, KH)]
        return x
    weights = [(1 + 0.2 * torch.randn(d, generator=gen)).cuda() for _ in range(2)]
    caches = [pkg.cache8(B, KH, room, d) for _ in range(2)]
    first = [torch.randn(B, KH, 130, d, generator=gen).bfloat16().cuda() for _ in range(2)]
    for cache in caches:
        pkg.cache8_write(cache, *first)
    at = torch.tensor([5, 63, 128], dtype=torch.int32, device="cuda")
    state = token()
    dims = dict(f_q=1, f_kv=room, h=1, w=1, scale=d ** -0.5)
    need = pkg.dense_attn_fwd_cache8_workspace_bytes(state[0], caches[0], **dims)
    scratch = [torch.full((max(need, 256),), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def step(x, at, cache, scratch):
        q, k, v = x
        where = at[:, None, None].expand(B, 3, 1).contiguous()
        q, k = pkg.norm_rotary_fwd(q, k, *weights, layout="halves", ladder="shared", q_positions=where, k_positions=where)
        pkg.cache8_write(cache, k, v, at=at)
        return pkg.dense_attn_fwd_cache8(q, cache, kv_len=at + 1, workspace=scratch, **dims)
    step(state, at, caches[1], scratch[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(state, at, caches[0], scratch[0])
        at.add_(1)
    for replay in range(8):
        fresh = token()
        for x, y in zip(state, fresh):
            x.copy_(y)
        now = at.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = step(fresh, now, caches[1], scratch[1])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, want)), replay
    k, v = (x.double() for x in pkg.cache8_read(caches[0], room))
    where = now[:, None, None].expand(B, 3, 1).contiguous()
    q = pkg.norm_rotary_fwd(fresh[0], None, weights[0], layout="halves", ladder="shared", q_positions=where).double()
    for b in range(B):
        n = int(now[b]) + 1
        for h in range(H):
            p = torch.softmax(d ** -0.5 * (q[b, h] @ k[b, h // 4, :n].t()), -1)
            want, size = p @ v[b, h // 4, :n], p @ v[b, h // 4, :n].abs()
            # weights and result rounded to bf16, 32-bit sums beside that
            assert ((out[0][b, h].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -12) * (size + want.abs())).all()


def test_video_step():
    """The step of an autoregressive clip: norm and rotary positions of a chunk's queries and keys, its rows into the cache
    behind the earlier chunks, dense attention over the cache, MonarchRT attention over its values.  Each against the
    definition on what the step before it gave."""
    f, h, w, heads, d, chunks = 3, 6, 8, 2, 128, 3
    n = f * h * w
    gen = torch.Generator().manual_seed(12)
    cache = pkg.cache8(1, heads, chunks * n, d)
    weights = [(1 + 0.2 * torch.randn(d, generator=gen)).cuda() for _ in range(2)]
    for i in range(chunks):
        q, k, v = (torch.randn(1, heads, n, d, generator=gen).bfloat16().cuda() for _ in range(3))
        q, k = pkg.norm_rotary_fwd(q, k, *weights, f_q=f, f_kv=f, h=h, w=w, q_frame_offset=f * i, kv_frame_offset=f * i)
        pkg.cache8_write(cache, k, v, at=n * i)
        dims = dict(f_q=f, f_kv=f * (i + 1), h=h, w=w, causal_chunk=f, q_frame_offset=f * i, scale=d ** -0.5)
        o, lse = pkg.dense_attn_fwd_cache8(q, cache, **dims)
        kc, vc = pkg.cache8_read(cache, n * (i + 1))
        m = pkg.monarch_attn_fwd(q, kc, vc, b1=f * h, b2=w, tile=1, iters=2, **dims)
        torch.cuda.synchronize()
        for x, y in ((kc[:, :, n * i:], k), (vc[:, :, n * i:], v)):
            # e4m3: 2^-4 of a value, or 2^-10 of the scale, which is 2^-7 of the block's largest magnitude at most
            most = torch.nn.functional.max_pool1d(y.abs().float().amax(-1), 129, 1, 64)[..., None]
            assert ((x.float() - y.float()).abs() <= (2.0 ** -4 * y.float().abs()).clamp(min=2.0 ** -17) + 2.0 ** -17 * most).all()
        c = Step(f, f * (i + 1), h, w, heads=heads, chunk=f, offset=f * i)
        ref, cost = reference(c, q, kc, vc, torch.zeros_like(q))
        check(c, dict(O=o, lse=lse), ref, cost)
        exact = pkg.monarch_attn_fwd(q, kc, vc, b1=f * h, b2=w, tile=1, iters=2, compute=pkg.MRT_COMPUTE_F32, **dims)
        torch.cuda.synchronize()
        assert (m.float() - exact.float()).abs().max() <= 2e-2
