"""The dense attention's forward and backward pass in 64 bits, written from the formulas, with bounds on what a
rounding of the kernels may cost an entry; shared by the GPU tests of the training step."""
from __future__ import annotations

import math
from dataclasses import dataclass

import torch

import paper_2602_12271_amd as pkg


@dataclass(frozen=True)
class Step:
    f_q: int
    f_kv: int
    h: int = 1
    w: int = 1
    heads: int = 2
    kv_heads: int = 0
    batch: int = 1
    dim: int = 128
    chunk: int = 0
    offset: int = 0
    dtype: str = "bf16"
    kv_len: tuple = ()
    layout: str = "bhnd"        # "bnhd": tokens outside of heads, as a projection leaves them; "packed": Q, K, V in one
    scale: float = 0.0          # 0: 1 / sqrt(dim)
    sigma: float = 1.0          # of Q and K
    compute: int = 0

    @property
    def nq(self):
        return self.f_q * self.h * self.w

    @property
    def nkv(self):
        return self.f_kv * self.h * self.w

    @property
    def args(self):
        return dict(f_q=self.f_q, f_kv=self.f_kv, h=self.h, w=self.w, causal_chunk=self.chunk, q_frame_offset=self.offset,
                    scale=self.scale or self.dim ** -0.5, compute=self.compute)


def tensors(c: Step, seed=0, device="cuda"):
    """Q, K, V, dO in the layout of the case, and kv_len."""
    gen = torch.Generator().manual_seed(seed)
    dt = torch.float32 if c.dtype == "f32" else torch.bfloat16
    kvh = c.kv_heads or c.heads

    def one(n, heads, sigma=1.0):
        x = (sigma * torch.randn(c.batch, heads, n, c.dim, generator=gen)).to(dt).to(device)
        return x.transpose(1, 2).contiguous().transpose(1, 2) if c.layout == "bnhd" else x
    if c.layout == "packed":
        assert c.nq == c.nkv and kvh == c.heads
        x = torch.randn(c.batch, c.nq, 3, c.heads, c.dim, generator=gen).to(dt).to(device)
        q, k, v = (x[:, :, i].transpose(1, 2) for i in range(3))
        do = torch.randn(c.batch, c.nq, c.heads, c.dim, generator=gen).to(dt).to(device).transpose(1, 2)
    else:
        q, k, v, do = one(c.nq, c.heads, c.sigma), one(c.nkv, kvh, c.sigma), one(c.nkv, kvh), one(c.nq, c.heads)
    kv_len = torch.tensor(c.kv_len, dtype=torch.int32, device=device) if c.kv_len else None
    return q, k, v, do, kv_len


def hidden(c: Step, b, device):
    """[queries, keys]: pairs that take no part."""
    hw = c.h * c.w
    key = torch.arange(c.nkv, device=device)[None]
    out = torch.zeros(c.nq, c.nkv, dtype=torch.bool, device=device)
    if c.chunk:
        query_chunk = (torch.arange(c.nq, device=device) // hw + c.offset) // c.chunk
        out |= key // hw // c.chunk > query_chunk[:, None]
    if c.kv_len:
        out |= key >= min(max(c.kv_len[b], 0), c.nkv)
    return out


def reference(c: Step, q, k, v, do, dtype=torch.float64):
    """{name: value}, and two {name: what relative roundings of size 1 may cost}, entry by entry: of the weights P and
    the logits' gradients dS, operands of the second products; and of O, whose product with dO is subtracted in dS."""
    scale, group = c.args["scale"], c.heads // (c.kv_heads or c.heads)
    q, k, v, do = (x.to(dtype) for x in (q, k, v, do))
    shapes = dict(O=q, lse=q[..., 0], dQ=q, dK=k, dV=v)
    out = {n: torch.zeros(x.shape, dtype=dtype, device=x.device) for n, x in shapes.items()}
    cost, cost_o = ({n: torch.zeros_like(x) for n, x in out.items()} for _ in range(2))
    for b in range(c.batch):
        off = hidden(c, b, q.device)
        for h in range(c.heads):
            g = h // group
            qh, kh, vh, doh = q[b, h], k[b, g], v[b, g], do[b, h]
            s = scale * (qh @ kh.t())
            s = s.masked_fill(off, -math.inf)
            lse = torch.logsumexp(s, -1)
            p = torch.where(off, torch.zeros_like(s), torch.exp(s - torch.where(lse.isinf(), torch.zeros_like(lse), lse)[:, None]))
            vh, kh = torch.nan_to_num(vh), torch.nan_to_num(kh)
            o = p @ vh
            ds = p * (doh @ vh.t() - (o * doh).sum(-1, keepdim=True))
            out["O"][b, h], out["lse"][b, h] = o, lse
            out["dQ"][b, h] = scale * (ds @ kh)
            out["dK"][b, g] += scale * (ds.t() @ qh)
            out["dV"][b, g] += p.t() @ doh
            by_o = p * (o.abs() * doh.abs()).sum(-1, keepdim=True)
            cost["O"][b, h] = p @ vh.abs()
            cost["dV"][b, g] += p.t() @ doh.abs()
            for part, size in ((cost, ds.abs()), (cost_o, by_o)):
                part["dQ"][b, h] = scale * (size @ kh.abs())
                part["dK"][b, g] += scale * (size.t() @ qh.abs())
    return out, (cost, cost_o)


def run(c: Step, q, k, v, do, kv_len, **kw):
    o, lse = pkg.dense_attn_fwd_save(q, k, v, kv_len=kv_len, **c.args)
    grads = pkg.dense_attn_bwd(q, k, v, o, do, lse, kv_len=kv_len, **c.args, **kw)
    return dict(zip(("O", "lse", "dQ", "dK", "dV"), (o, lse, *grads)))


def units(c: Step):
    """(relative rounding of the operands and results, relative error of 32-bit sums and exponents).

    32 bits: a sum of n terms is off by at most n 2^-24 of the sum of their magnitudes; logits of magnitude up to
    sigma^2 sqrt(dim) 4 and their log-sum-exp are rounded by 2^-24 each, twice, and the exponential turns that into a
    relative error of the weight."""
    n = max(c.nq * (c.heads // (c.kv_heads or c.heads)), c.nkv) + 2 * c.dim
    logit = 8 * c.sigma ** 2 * c.dim * c.args["scale"] + math.log(c.nkv + 1)
    sums = (n + 4 * logit + 16) * 2.0 ** -24
    return (0.0 if c.dtype == "f32" or c.compute else 2.0 ** -8), sums


def check(c: Step, got, ref, costs):
    """O reaches the backward pass in its storage type, also where the arithmetic is 32 bits: the products of its
    rounding, 2^-8 |O| in bf16, with dO enter every dS of the row times P, which is what cost_o sums up."""
    u, sums = units(c)
    stored = 2.0 ** -8 if c.dtype == "bf16" else 2.0 ** -24
    cost, cost_o = costs
    worst = {}
    for name, x in got.items():
        want = ref[name]
        x = x.double()
        if name == "lse":
            same = torch.equal(x == -math.inf, want == -math.inf)
            assert same, "rows that see no key"
            live = want != -math.inf
            tol = sums * (1 + want[live].abs())
            err = (x[live] - want[live]).abs()
        else:
            # (second order: roundings of what is rounded already)
            tol = (u * (1 + u) + sums) * cost[name] + (stored * (1 + u) ** 2 + sums) * cost_o[name]
            tol = tol * (1 + stored) + stored * want.abs() + 1e-30
            err = (x - want).abs()
        assert torch.isfinite(err).all(), name
        if err.numel():
            worst[name] = float((err / tol).max())
            assert worst[name] <= 1, f"{name}: {worst[name]:.2f} of what rounding may cost"
    return worst
