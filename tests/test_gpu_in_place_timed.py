"""GPU: attention with O in the place of Q while launches are timed: a launch that is repeated between the two events would take its
own result for queries, so such a call runs once and is not recorded."""
import pytest
import torch

import paper_2602_12271_amd as pkg
from paper_2602_12271_amd import binding

pytestmark = pytest.mark.gpu


def check(call, q):
    """call(out) with an O of its own and with q's memory."""
    want = call(torch.empty_like(q)).clone()
    torch.cuda.synchronize()
    binding.profile_enable(3)
    try:
        apart = call(torch.empty_like(q))
        torch.cuda.synchronize()
        recorded = len(binding.profile_read())
        got = call(q)
        torch.cuda.synchronize()
    finally:
        binding.profile_enable(0)
        again = len(binding.profile_read())
    assert got.data_ptr() == q.data_ptr() and recorded > 0 and again == 0
    assert torch.equal(apart, want) and torch.equal(got, want)


@pytest.mark.parametrize("rows", [1, 40, 300])
@pytest.mark.parametrize("op", ["over-a-cache", "plain", "masked"])
def test_dense(op, rows):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    n = 600
    q = torch.randn(2, 4, rows, 128, generator=gen, device="cuda").bfloat16()
    k, v = (torch.randn(2, 4, n, 128, generator=gen, device="cuda").bfloat16() for _ in range(2))
    args = dict(f_q=rows, f_kv=n, h=1, w=1, scale=128 ** -0.5)
    if op == "masked":
        args.update(causal_chunk=8, q_frame_offset=n - rows)
    cache = pkg.cache8(2, 4, n, 128)
    pkg.cache8_write(cache, k, v)
    print(op, rows, flush=True)
    if op == "over-a-cache":
        check(lambda out: pkg.dense_attn_fwd_cache8(q, cache, out=out, **args)[0], q)
    else:
        check(lambda out: pkg.dense_attn_fwd(q, k, v, out=out, **args), q)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("f, h, w, b1, b2, tile, iters, d, heads, chunk", [
    (1, 24, 24, 24, 24, 0, 2, 64, 1, 0), (1, 97, 20, 97, 20, 0, 1, 128, 2, 0), (2, 50, 48, 50, 24, 1, 2, 128, 2, 0),
    (6, 7, 34, 42, 34, 0, 2, 64, 4, 2)])
def test_monarch(f, h, w, b1, b2, tile, iters, d, heads, chunk, dtype):
    gen = torch.Generator(device="cuda").manual_seed(9)
    q, k, v = (torch.randn(1, heads, f * h * w, d, generator=gen, device="cuda").to(dtype) for _ in range(3))
    print(f, h, w, dtype, flush=True)
    check(lambda out: pkg.monarch_attn_fwd(q, k, v, b1=b1, b2=b2, tile=tile, iters=iters, f_q=f, f_kv=f, h=h, w=w, causal_chunk=chunk,
                                           scale=d ** -0.5, out=out), q)


def test_one_token_of_another_layout():
    """O in the place of Q, as [batch, tokens, heads, head_dim]: one token, so that both have the same elements in the same places."""
    q = torch.randn(1, 4, 1, 64, device="cuda").bfloat16()
    cache = pkg.cache8(1, 4, 100, 64)
    rows = torch.randn(1, 4, 100, 64, device="cuda")
    pkg.cache8_write(cache, rows, rows)
    args = dict(f_q=1, f_kv=100, h=1, w=1, scale=0.125)
    want = pkg.dense_attn_fwd_cache8(q, cache, **args)[0]
    out = q.view(1, 1, 4, 64).transpose(1, 2)
    assert out.stride() != q.stride()
    pkg.dense_attn_fwd_cache8(q, cache, out=out, **args)
    assert torch.equal(q, want)
