"""GPU: the dense attention's backward pass where rows see few keys.

delta = dO . O, with O rounded to bf16, is off by up to 2^-8 of sum |dO| |O|, and where a row sees few keys, or keys that
hardly differ, that is more than all of dS = P (dP - delta): over a single key dS is zero.  Such rows form delta from P and
dP, and the gradients are held here to a bound in which O does not occur."""
import dataclasses

import pytest
import torch

from dense_training import Step, hidden, reference, run, tensors, units

pytestmark = pytest.mark.gpu


def alike(c, seed):
    """Values of a head that differ by a thirty-second of their size: what dO . V has in common cancels in dS, and a delta
    that is off does not."""
    q, k, v, do, kv_len = tensors(c, seed=seed)
    common = torch.randn(c.batch, v.shape[1], 1, c.dim, generator=torch.Generator().manual_seed(seed)).to(v.device)
    v.copy_(common + 2.0 ** -5 * v.float())
    return q, k, v, do, kv_len


def by_values(c, q, k, v, do):
    """What a relative error of size 1 of the 32-bit numbers P, dP and delta may cost dQ and dK, entry by entry:
    with A_ij = sum over features of |dO_i| |V_j|, dS_ij is off by P_ij (A_ij + sum_j P_ij A_ij)."""
    scale, group = c.args["scale"], c.heads // (c.kv_heads or c.heads)
    q, k, v, do = (x.double() for x in (q, k, v, do))
    out = dict(dQ=torch.zeros_like(q), dK=torch.zeros_like(k))
    for b in range(c.batch):
        off = hidden(c, b, q.device)
        for h in range(c.heads):
            g = h // group
            s = (scale * (q[b, h] @ k[b, g].t())).masked_fill(off, -torch.inf)
            p = torch.nan_to_num(torch.softmax(s, -1))
            a = do[b, h].abs() @ v[b, g].abs().t()
            ds = p * (a + (p * a).sum(-1, keepdim=True))
            out["dQ"][b, h] = scale * (ds @ k[b, g].abs())
            out["dK"][b, g] += scale * (ds.t() @ q[b, h].abs())
    return out


def check_short(c, got, q, k, v, do, sequences):
    """P, dP and delta are off by units()'s `sums` over the 128 keys that a row sees at most (delta by two, its own sum
    and that of P dP), the sums of dS K and dS^T Q by another: 4 in all; then dS is rounded as an operand, and the result
    to its type."""
    ref, (cost, _) = reference(c, q, k, v, do)
    values = by_values(c, q, k, v, do)
    u, sums = units(dataclasses.replace(c, f_kv=min(c.f_kv, 128)))
    stored = 2.0 ** -8
    for name in ("dQ", "dK"):
        want = ref[name]
        tol = (u * cost[name] + 4 * sums * (1 + u) * values[name]) * (1 + stored) + stored * want.abs() + 1e-30
        off = ((got[name].double() - want).abs() / tol)[list(sequences)]
        print(f"  {name}: {float(off.max()):.2f} of what rounding may cost", flush=True)
        assert off.max() <= 1, name


# (up to 32 queries that share keys, in a tensor of many keys, of which the sequences have few)
CUT = {
    "one-query": Step(1, 3000, heads=30, batch=5, kv_len=(3000, 1, 2, 4, 128)),
    "one-query-d64-shared": Step(1, 500, heads=30, kv_heads=5, batch=4, dim=64, kv_len=(1, 3, 33, 500)),
    "rows": Step(16, 1030, heads=12, batch=4, kv_len=(1, 2, 31, 97)),
    "rows-causal": Step(16, 400, heads=8, kv_heads=4, batch=4, chunk=1, offset=380, kv_len=(1, 64, 100, 390)),
    "rows-of-heads": Step(4, 300, heads=16, kv_heads=2, batch=3, dim=64, kv_len=(1, 0, 65)),
}


@pytest.mark.parametrize("name", CUT)
def test_sequences_cut_to_few_keys(name):
    c = CUT[name]
    q, k, v, do, kv_len = alike(c, seed=31)
    got = run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    check_short(c, got, q, k, v, do, [b for b, n in enumerate(c.kv_len) if n <= 128])


# bf16 tensors, fp32 arithmetic: dS is not rounded, and nothing but the result's rounding and 32-bit sums is left
IN_F32 = {
    "causal-10": Step(10, 10, heads=8, chunk=1, compute=1),
    "causal-100-d64": Step(100, 100, heads=4, chunk=1, dim=64, compute=1),
    "two-keys": Step(3, 2, heads=30, batch=2, compute=1),
    "one-key": Step(40, 1, heads=3, compute=1),
    "queries-50-of-128-shared": Step(50, 128, heads=6, kv_heads=2, dim=64, compute=1),
    "queries-300-of-90": Step(300, 90, heads=2, compute=1),
    "frames-dim-40": Step(4, 4, 3, 7, heads=4, chunk=1, dim=40, compute=1),
    "odd-dim-causal": Step(33, 33, heads=4, chunk=1, dim=37, compute=1),
    "dim-1": Step(20, 30, heads=4, dim=1, compute=1),
    "padded": Step(40, 40, heads=6, batch=5, kv_len=(40, 32, 5, 1, 0), compute=1),
    "cut": Step(17, 2000, heads=4, batch=3, kv_len=(128, 3, 1), compute=1),
    "tokens-outside-heads": Step(2, 3, 4, 9, heads=4, kv_heads=2, batch=2, layout="bnhd", compute=1),
}


@pytest.mark.parametrize("name", IN_F32)
def test_bf16_tensors_in_fp32_arithmetic(name):
    c = IN_F32[name]
    q, k, v, do, kv_len = alike(c, seed=32)
    got = run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    check_short(c, got, q, k, v, do, range(c.batch))


@pytest.mark.parametrize("dim,shift", [(40, 4), (64, 4), (128, 4), (128, 12), (64, 1), (37, 3)])
def test_rows_that_begin_anywhere(dim, shift):
    """Rows of bf16 numbers in fp32 arithmetic that begin at 8 or 2 bytes, the last of them at the end of its memory."""
    c = Step(40, 40, heads=3, kv_heads=1, batch=2, chunk=1, dim=dim, compute=1)
    wide = []
    for x in alike(c, seed=33)[:4]:
        b, h, n, d = x.shape
        memory = torch.full((b, n, h, d + shift), 7.0, dtype=x.dtype, device="cuda")
        memory[..., shift:] = x.transpose(1, 2)
        wide.append(memory[..., shift:].transpose(1, 2))
    q, k, v, do = wide
    assert q.data_ptr() % 16 and q.stride(3) == 1
    got = run(c, q, k, v, do, None)
    torch.cuda.synchronize()
    check_short(c, got, q, k, v, do, range(c.batch))
