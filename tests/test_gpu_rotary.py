"""GPU: rotary positions with three axes, forward and backward, against the definition in 64 bits."""
import itertools
import math

import pytest
import torch

import paper_2602_12271_amd as pkg
from workloads import synthetic as syn

pytestmark = pytest.mark.gpu


def positions_of(f, h, w, first):
    at = torch.cartesian_prod(first + torch.arange(f), torch.arange(h), torch.arange(w)).reshape(-1, 3)
    return at.t()


def turned(x, positions, split, theta, layout, ladder, sign):
    """x [batch, heads, tokens, dim] (64 bits, on the host); positions [3, tokens] or [batch, 3, tokens]."""
    x, total = x.clone(), sum(split)
    positions = positions.double() if positions.dim() == 3 else positions.double()[None]
    p = 0
    for axis, count in enumerate(split):
        for i in range(count):
            angle = positions[:, axis] * theta ** -(p / total if ladder == "shared" else i / count)
            c, s = torch.cos(angle)[:, None], sign * torch.sin(angle)[:, None]
            u, v = (2 * p, 2 * p + 1) if layout == "adjacent" else (p, p + total)
            a, b = x[..., u].clone(), x[..., v].clone()
            x[..., u], x[..., v] = a * c - b * s, a * s + b * c
            p += 1
    return x


def bound(x, out_dtype, split, layout):
    """Entries are off by the rounding of the result, and by that of cos and sin (2 ulp each at most, plus 1e-7 for
    the angle) and of two products in 32 bits: 8 x 2^-24 of the pair's magnitudes."""
    total = sum(split)
    pair = torch.zeros_like(x)
    u = [2 * p if layout == "adjacent" else p for p in range(total)]
    v = [2 * p + 1 if layout == "adjacent" else p + total for p in range(total)]
    size = x[..., u].abs() + x[..., v].abs()
    pair[..., u], pair[..., v] = size, size
    step = 2.0 ** -8 if out_dtype == torch.bfloat16 else 2.0 ** -24
    return (8 * 2.0 ** -24 + 1e-7 + step * math.sqrt(2)) * pair + 1e-30


SHAPES = {
    # dim, split, tokens as (f, h, w) or n, heads, kv_heads, batch
    "chunk": (128, None, (3, 5, 7), 12, 12, 1),
    "one-token": (128, (16, 24, 24), 1, 32, 8, 1),
    "dim-64": (64, None, (2, 3, 5), 5, 1, 3),
    "dim-72": (72, (18, 9, 9), 33, 3, 3, 2),
    "dim-80": (80, (10, 10, 20), 33, 4, 2, 2),
    "partial": (128, (8, 8, 8), (1, 6, 6), 4, 2, 1),
    "one-axis": (96, (0, 0, 48), 70, 2, 1, 1),
    "odd-pairs": (30, (3, 5, 6), 41, 3, 1, 2),
    "odd-dim": (31, (4, 4, 4), 41, 3, 1, 1),
    "dim-2": (2, (0, 1, 0), 300, 1, 1, 1),
    "dim-256": (256, (40, 44, 44), 19, 2, 2, 1),
    "many-heads": (64, None, 3, 200, 40, 1),
    "long": (64, None, 5000, 2, 1, 1),
}
TYPES = {"bf16": (torch.bfloat16, torch.bfloat16), "f32": (torch.float32, torch.float32),
         "f32-bf16": (torch.float32, torch.bfloat16), "bf16-f32": (torch.bfloat16, torch.float32)}


@pytest.mark.parametrize("layout,ladder", itertools.product(("adjacent", "halves"), ("axis", "shared")))
@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_rotary(shape, types, layout, ladder):
    dim, split, tokens, heads, kv_heads, batch = SHAPES[shape]
    tin, tout = TYPES[types]
    gen = torch.Generator().manual_seed(3)
    n = tokens if isinstance(tokens, int) else math.prod(tokens)
    q, k = (torch.randn(batch, x, n, dim, generator=gen).to(tin) for x in (heads, kv_heads))
    args = dict(theta=1e4, split=split, layout=layout, ladder=ladder, dtype=tout)
    if isinstance(tokens, int):
        where = torch.randint(-50, 1 << 20, (batch, 3, n), generator=gen).to(torch.int32)
        args.update(q_positions=where.cuda(), k_positions=where.cuda())
        at = (where, where)
    else:
        f, h, w = tokens
        args.update(f_q=f, h=h, w=w, q_frame_offset=18, kv_frame_offset=4)
        at = (positions_of(f, h, w, 18), positions_of(f, h, w, 4))
    split = split or pkg.binding.rotary_pairs_split(dim)
    for call, sign in ((pkg.rotary_fwd, 1), (pkg.rotary_bwd, -1)):
        got = call(q.cuda(), k.cuda(), **args)
        torch.cuda.synchronize()
        for x, y, positions in zip((q, k), got, at):
            assert y.dtype == tout and y.shape == x.shape
            want = turned(x.double(), positions, split, 1e4, layout, ladder, sign)
            off = (y.cpu().double() - want).abs() / bound(x.double(), tout, split, layout)
            rest = y.cpu()[..., 2 * sum(split):]
            assert torch.equal(rest, x[..., 2 * sum(split):].to(tout))
            off = off[..., :2 * sum(split)]
            assert off.max() <= 1, f"{off.max():.2f} of the bound"


def test_rotary_is_the_workloads_rotation():
    # the encoding of the named workloads' inputs (numpy, 32-bit tables) within its own roundings
    wl = syn.WORKLOADS["C3"]
    rng = torch.Generator().manual_seed(0)
    x = torch.randn(1, 2, wl.n_q, wl.head_dim, generator=rng)
    ang = syn.rope_angles(wl.q_frame_offset + syn.np.arange(wl.f_q), wl.h, wl.w, wl.head_dim)
    want = torch.from_numpy(syn.apply_rope(x.numpy(), ang))
    got = pkg.rotary_fwd(x.cuda(), f_q=wl.f_q, h=wl.h, w=wl.w, q_frame_offset=wl.q_frame_offset)
    torch.cuda.synchronize()
    assert pkg.binding.rotary_pairs_split(wl.head_dim) == syn.rope_pairs_split(wl.head_dim)
    assert (got.cpu() - want).abs().max() <= 16 * 2.0 ** -24 * x.abs().max()
