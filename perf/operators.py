"""The operators of a training step of a dense attention layer: rotary positions over (frame, height, width),
the attention that keeps its row statistics, its backward pass, and the rotation of the gradients.

Every case is one pass through the public binding on device tensors.  With `own` false the same results
are formed from elementary torch operations in 32 bits (angles in 64), rounded once at the end.  Shapes are
those of a video diffusion transformer's self-attention (latent grids of 30 x 52 and 45 x 80, chunks of three
frames, 21 latent frames, heads of 128 or 64), of sequences of text and images, and of a query that pools a clip.

`exact` states the results in 64 bits, one head at a time.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _attn(op, grid, heads, *, f_kv=None, kv_heads=None, chunk=0, offset=0, dtype="bf16", dim=128, batch=1, padded=False,
          **named):
    f, h, w = grid
    return dict(named, op=op, batch=batch, heads=heads, kv_heads=kv_heads or heads, dim=dim, f_q=f,
                f_kv=f if f_kv is None else f_kv, h=h, w=w, chunk=chunk, offset=offset, dtype=dtype, padded=padded)


def _rotary(op, grid, heads, *, kv_heads=None, offset=0, dtype="bf16", out="bf16", dim=128, batch=1, layout="adjacent",
            ladder="axis", split="", theta=10000.0, **named):
    # grid (f, h, w): tokens of a grid; (0, 0, n): n tokens of text and images at positions of their own
    f, h, w = grid
    return dict(named, op=op, batch=batch, heads=heads, kv_heads=kv_heads or heads, dim=dim, f=f, h=h, w=w, offset=offset,
                dtype=dtype, out=out, layout=layout, ladder=ladder, split=split, theta=theta)


def listed():
    return [
        # the smallest training step: one head of one small frame in fp32; latency is all there is
        _attn("step", (1, 24, 24), 1, dtype="f32", dim=64, name="step-tiny-f32"),
        # a small model's layer on an odd grid, a padded batch: one clip whole, one cut short, one empty
        _attn("step", (2, 17, 23), 4, dim=64, batch=3, padded=True, name="step-padded-odd-d64"),
        # text under a causal mask, queries of eight heads sharing one head of keys
        _attn("step", (1531, 1, 1), 16, kv_heads=2, chunk=1, batch=2, name="step-text-shared-heads"),
        # one query that pools a whole cached clip (a reward or class head), its step
        _attn("step", (1, 1, 1), 12, f_kv=32760, batch=4, name="step-pool-clip"),
        # one frame in fp32 storage and arithmetic, as quality studies train it
        _attn("step", (1, 30, 52), 12, dtype="f32", name="step-frame-480p-f32"),
        # a layer kept dense, on one chunk: the ordinary training step
        _attn("step", (3, 30, 52), 12, name="step-chunk-480p"),
        # backward pass of the last chunk against the cached keys of the whole clip
        _attn("bwd", (3, 30, 52), 12, f_kv=21, chunk=3, offset=18, name="bwd-cache-480p"),
        # the largest step: three chunks of a clip under the block-causal mask
        _attn("step", (9, 30, 52), 12, chunk=3, name="step-clip-480p"),
        # decoding: one token's query and key at positions of its own, far into a session
        _rotary("fwd", (0, 0, 1), 32, kv_heads=8, layout="halves", ladder="shared", split="16,24,24", theta=1e6,
                name="rotary-token"),
        # queries and keys of one autoregressive chunk late in a clip: the ordinary call
        _rotary("fwd", (3, 30, 52), 12, offset=18, name="rotary-chunk-480p"),
        # gradients in fp32 of a batch of text and images, back to bf16 leaves
        _rotary("bwd", (0, 0, 4099), 32, kv_heads=8, batch=2, dtype="f32", layout="halves", ladder="shared",
                split="16,24,24", theta=1e6, name="rotary-bwd-text-image"),
        # the largest: gradients of a whole 720p clip of a 40-head model
        _rotary("bwd", (21, 45, 80), 40, name="rotary-bwd-clip-720p"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _candidate(rng):
    kind = rng.choice(["chunk", "cache", "clip", "text", "pool", "padded", "f32", "rotary", "rotary", "rotary-text"])
    dim, batch = rng.choice([64, 128, 128]), rng.choice([1, 1, 2, 3])
    h, w, heads = _log_int(rng, 3, 45), _log_int(rng, 3, 80), _log_int(rng, 1, 40)
    kv = heads // rng.choice([n for n in (1, 1, 2, 3, 4, 5, 8) if heads % n == 0])
    op = rng.choice(["step", "step", "bwd"])
    if kind == "chunk":
        return _attn(op, (rng.randint(1, 3), h, w), heads, dim=dim, batch=batch)
    if kind == "cache":
        n = 3 * rng.randint(2, 7)
        return _attn(op, (3, h, w), heads, kv_heads=kv, f_kv=n, chunk=3, offset=n - 3, dim=dim, batch=batch)
    if kind == "clip":
        return _attn(op, (3 * rng.randint(2, 4), h, w), heads, chunk=rng.choice([1, 3]), dim=dim, batch=batch)
    if kind == "text":
        # (from two tokens on: over a single key dQ and dK are zero, and what is left is rounding alone)
        return _attn(op, (_log_int(rng, 2, 8192), 1, 1), heads, kv_heads=kv, chunk=1, dim=dim, batch=batch)
    if kind == "pool":
        n = _log_int(rng, 2, 75600)
        return _attn(op, (rng.randint(1, 16), 1, 1), heads, kv_heads=kv, f_kv=n, dim=dim, batch=batch)
    if kind == "padded":
        return _attn(op, (rng.randint(1, 3), h, w), heads, kv_heads=kv, dim=dim, batch=rng.randint(2, 4), padded=True,
                     chunk=rng.choice([0, 1]))
    if kind == "f32":
        return _attn(op, (rng.randint(1, 2), h, w), min(heads, 16), dtype="f32", dim=rng.choice([40, 64, 96, 128]),
                     chunk=rng.choice([0, 1]))
    op = rng.choice(["fwd", "bwd"])
    dtype, out = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "f32")] + [("f32", "bf16")] * (op == "bwd"))
    layout, ladder = rng.choice([("adjacent", "axis"), ("adjacent", "shared"), ("halves", "axis"), ("halves", "shared")])
    if kind == "rotary":
        return _rotary(op, (rng.randint(1, 21), h, w), heads, kv_heads=kv, offset=rng.choice([0, 18, 5000]), dtype=dtype,
                       out=out, dim=dim, batch=batch, layout=layout, ladder=ladder)
    dim = rng.choice([64, 72, 80, 96, 128])
    axes = [dim // 8, dim // 8, dim // 4]
    rng.shuffle(axes)
    return _rotary(op, (0, 0, _log_int(rng, 1, 32768)), heads, kv_heads=kv, dtype=dtype, out=out, dim=dim, batch=batch,
                   layout=layout, ladder=ladder, split=",".join(map(str, axes)), theta=rng.choice([1e4, 1e6]))


def _cost(c):
    """A rough time of the plain form in seconds, to keep drawn cases below the largest listed one of their kind."""
    if c["op"] in ("fwd", "bwd") and "split" in c:
        return work(c)["bytes"] / 1e12
    return c["batch"] * c["heads"] * c["f_q"] * c["f_kv"] * (c["h"] * c["w"]) ** 2 * (14 * c["dim"] + 4000) / 6e13


def draw(rng):
    most = {}
    for c in listed():
        most["split" in c] = max(most.get("split" in c, 0), _cost(c))
    while True:
        c = _candidate(rng)
        if _cost(c) <= 0.9 * most["split" in c]:
            return c


# ---- inputs --------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _clip_positions(frames, h, w, first):
    """[3, tokens]: frame, row and column of every token of a grid."""
    at = torch.cartesian_prod(first + torch.arange(frames, device="cuda"), torch.arange(h, device="cuda"),
                              torch.arange(w, device="cuda"))
    return at.reshape(-1, 3).t().contiguous()


def _text_positions(case, gen):
    """[batch, 3, tokens] int32: text (the same position on every axis) around an image of 24 columns."""
    n, batch = case["w"], case["batch"]
    start = torch.randint(0, 1 << 20, (batch, 1, 1), generator=gen, device="cuda")
    i = torch.arange(n, device="cuda")
    lo, hi = n // 4, n - n // 4
    image = (i >= lo) & (i < hi)
    rows = torch.stack([torch.full_like(i, lo), lo + (i - lo) // 24, lo + (i - lo) % 24])
    after = torch.where(i >= hi, lo + (hi - lo + 23) // 24 + i - hi, i)
    return (start + torch.where(image[None], rows, after[None].expand(3, n))[None]).to(torch.int32).contiguous()


def _pairs(case):
    """Rotary pairs of every axis."""
    if case.get("split"):
        return [int(x) for x in case["split"].split(",")]
    pairs = case["dim"] // 2
    return [pairs - 2 * (pairs // 3), pairs // 3, pairs // 3]


def _angles(pairs, ladder, theta, positions):
    """[..., tokens, pairs] in 64 bits for positions [..., 3, tokens]."""
    total = sum(pairs)
    if ladder == "shared":
        exponent = torch.arange(total, dtype=torch.float64, device="cuda") / total
    else:
        exponent = torch.cat([torch.arange(n, dtype=torch.float64, device="cuda") / n for n in pairs])
    axis = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(pairs, device="cuda"))
    return positions.double()[..., axis, :].transpose(-1, -2) * theta ** -exponent


def _rotate(x, angles, layout, sign):
    """x [batch, heads, tokens, dim] in its type; angles [(batch,) tokens, pairs]."""
    angles = angles if angles.dim() == 2 else angles[:, None]
    cos, sin = angles.cos().to(x.dtype), (sign * angles.sin()).to(x.dtype)
    n = angles.shape[-1]
    if layout == "halves":
        a, b, rest = x[..., :n], x[..., n:2 * n], x[..., 2 * n:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], -1)
    a, b, rest = x[..., 0:2 * n:2], x[..., 1:2 * n:2], x[..., 2 * n:]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), rest], -1)


def _attn_tensors(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    hw, dt = c["h"] * c["w"], _DTYPES[c["dtype"]]
    split = _pairs({"dim": c["dim"]})

    def rotated(heads, frames, first):
        x = _normal(gen, c["batch"], heads, frames * hw, c["dim"])
        return _rotate(x, _angles(split, "axis", 1e4, _clip_positions(frames, c["h"], c["w"], first)), "adjacent", 1).to(dt)

    q = rotated(c["heads"], c["f_q"], c["offset"])
    k = rotated(c["kv_heads"], c["f_kv"], 0)
    v = _normal(gen, *k.shape).to(dt)
    do = _normal(gen, *q.shape).to(dt)
    kv_len = None
    if c["padded"]:      # one clip whole, the others cut short, the last one empty
        cut = torch.rand(c["batch"], generator=gen, device="cuda")
        cut[0], cut[-1] = 1.0, 0.0
        kv_len = (cut * k.shape[2]).to(torch.int32)
    return q, k, v, do, kv_len


def _rotary_tensors(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = c["w"] if c["f"] == 0 else c["f"] * c["h"] * c["w"]
    positions = _text_positions(c, gen) if c["f"] == 0 else None
    dt = _DTYPES[c["dtype"]]
    q, k = (torch.empty(c["batch"], heads, n, c["dim"], dtype=dt, device="cuda") for heads in (c["heads"], c["kv_heads"]))
    q.normal_(generator=gen)
    k.normal_(generator=gen)
    return q, k, positions


def prepare(case, seed):
    if "split" in case:
        return {"case": case, "tensors": _rotary_tensors(case, seed)}
    q, k, v, do, kv_len = _attn_tensors(case, seed)
    state = {"case": case, "tensors": (q, k, v, do, kv_len)}
    if case["op"] == "bwd":      # the forward call's results, which the program kept
        o, lse = _plain_forward(case, q.float(), k.float(), v.float(), kv_len)[:2]
        state["kept"] = (o.to(q.dtype), lse)
    return state


# ---- one pass ------------------------------------------------------------------------------------
def _hidden(c, nq, nkv, kv_len, device):
    """[batch or 1, 1, 1, queries, keys] truth values, or None."""
    hidden = None
    if c["chunk"]:
        hw = c["h"] * c["w"]
        chunk_q = torch.div(c["offset"] + torch.arange(nq, device=device) // hw, c["chunk"], rounding_mode="floor")
        chunk_k = torch.div(torch.arange(nkv, device=device) // hw, c["chunk"], rounding_mode="floor")
        hidden = (chunk_k[None, :] > chunk_q[:, None])[None, None, None]
    if kv_len is not None:
        past = (torch.arange(nkv, device=device)[None] >= kv_len[:, None])[:, None, None, None]
        hidden = past if hidden is None else hidden | past
    return hidden


def _grouped(c, x):
    """[batch, heads, tokens, dim] -> [batch, kv heads, group, tokens, dim]."""
    return x.unflatten(1, (c["kv_heads"], c["heads"] // c["kv_heads"]))


def _logits(c, q, k, kv_len):
    s = torch.matmul(_grouped(c, q), k[:, :, None].transpose(-1, -2)).mul_(1 / math.sqrt(c["dim"]))
    hidden = _hidden(c, q.shape[2], k.shape[2], kv_len, q.device)
    return s if hidden is None else s.masked_fill_(hidden, -math.inf)


def _plain_forward(c, q, k, v, kv_len):
    s = _logits(c, q, k, kv_len)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p /= torch.where(total == 0, torch.ones_like(total), total)
    o = torch.matmul(p, v[:, :, None])
    return o.flatten(1, 2), (total.log() + top).flatten(1, 2).squeeze(-1), p


def _plain_probabilities(c, q, k, kv_len, lse):
    lse = _grouped(c, lse[..., None])
    return (_logits(c, q, k, kv_len) - torch.where(lse == -math.inf, torch.zeros_like(lse), lse)).exp_()


def _plain_backward(c, q, k, v, o, do, p):
    do, delta = _grouped(c, do), _grouped(c, (o * do).sum(-1, keepdim=True))
    dv = torch.matmul(p.transpose(-1, -2), do).sum(2)
    ds = torch.matmul(do, v[:, :, None].transpose(-1, -2)).sub_(delta).mul_(p).mul_(1 / math.sqrt(c["dim"]))
    dq = torch.matmul(ds, k[:, :, None]).flatten(1, 2)
    dk = torch.matmul(ds.transpose(-1, -2), _grouped(c, q)).sum(2)
    return dq, dk, dv


def _run_rotary(c, q, k, positions):
    if own:
        import paper_2602_12271_amd as mrt
        args = dict(theta=c["theta"], layout=c["layout"], ladder=c["ladder"], split=_pairs(c))
        if positions is not None:
            args.update(q_positions=positions, k_positions=positions)
        else:
            args.update(f_q=c["f"], f_kv=c["f"], h=c["h"], w=c["w"], q_frame_offset=c["offset"], kv_frame_offset=c["offset"])
        return mrt.rotary_fwd(q, k, **args) if c["op"] == "fwd" else mrt.rotary_bwd(q, k, dtype=_DTYPES[c["out"]], **args)
    positions = _clip_positions(c["f"], c["h"], c["w"], c["offset"]) if positions is None else positions
    angles = _angles(_pairs(c), c["ladder"], c["theta"], positions)
    return tuple(_rotate(x.float(), angles, c["layout"], 1 if c["op"] == "fwd" else -1).to(_DTYPES[c["out"]]) for x in (q, k))


def run(state):
    c = state["case"]
    if "split" in c:
        return dict(zip(("Q", "K"), _run_rotary(c, *state["tensors"])))
    q, k, v, do, kv_len = state["tensors"]
    if own:
        import paper_2602_12271_amd as mrt
        args = dict(f_q=c["f_q"], f_kv=c["f_kv"], h=c["h"], w=c["w"], causal_chunk=c["chunk"], q_frame_offset=c["offset"],
                    scale=1 / math.sqrt(c["dim"]), kv_len=kv_len)
        o, lse = mrt.dense_attn_fwd_save(q, k, v, **args) if c["op"] == "step" else state["kept"]
        grads = mrt.dense_attn_bwd(q, k, v, o, do, lse, **args)
    else:
        wide = [x.float() for x in (q, k, v)]
        if c["op"] == "step":
            o, lse, p = _plain_forward(c, *wide, kv_len)
        else:
            o, lse = state["kept"]
            p = _plain_probabilities(c, *wide[:2], kv_len, lse)
        grads = [g.to(q.dtype) for g in _plain_backward(c, *wide, o.float(), do.float(), p)]
        o = o.to(q.dtype)
    grads = dict(zip(("dQ", "dK", "dV"), grads))
    return dict(grads, O=o, lse=lse) if c["op"] == "step" else grads


def _seen(c):
    """(query, key) pairs of one head that take part, without what padding hides."""
    hw, frames = c["h"] * c["w"], c["f_kv"]
    if c["chunk"] == 0:
        return c["f_q"] * frames * hw * hw
    return sum(min(frames, ((f + c["offset"]) // c["chunk"] + 1) * c["chunk"]) for f in range(c["f_q"])) * hw * hw


def work(case):
    c = case
    size, to = ({"bf16": 2, "f32": 4}[c.get(x, c["dtype"])] for x in ("dtype", "out"))
    if "split" in c:
        n = (c["w"] if c["f"] == 0 else c["f"] * c["h"] * c["w"]) * c["batch"]
        elements = n * (c["heads"] + c["kv_heads"]) * c["dim"]
        return {"bytes": elements * (size + to) + (12 * n if c["f"] == 0 else 0), "flops": 3 * elements}
    hw = c["h"] * c["w"]
    q, k = (c["batch"] * c[n] * c[f] * hw for n, f in (("heads", "f_q"), ("kv_heads", "f_kv")))
    pairs = c["batch"] * c["heads"] * _seen(c) * c["dim"]
    # Q, O, dO, dQ and the row statistics; K, V, dK, dV.  Two products forward, five backward
    return {"bytes": (4 * q + 4 * k) * c["dim"] * size + 4 * q, "flops": (14 if c["op"] == "step" else 10) * pairs}


# ---- the same results in 64 bits -----------------------------------------------------------------
def _exact_rotary(c, seed):
    q, k, positions = _rotary_tensors(c, seed)
    n = q.shape[2]
    if positions is None:
        token = torch.arange(n, device="cuda")
        column, row, frame = token % c["w"], token // c["w"] % c["h"], token // (c["w"] * c["h"]) + c["offset"]
        axes = [x[None].double() for x in (frame, row, column)]
    else:
        axes = [positions[:, i].double() for i in range(3)]
    pairs, done = _pairs(c), []
    for x in (q, k):
        out = torch.empty_like(x, dtype=torch.float64) if x.numel() < 1 << 30 else None
        if out is None:
            return None
        out.copy_(x)
        p, total = 0, sum(pairs)
        for axis, count in zip(axes, pairs):
            for i in range(count):
                power = p / total if c["ladder"] == "shared" else i / count
                turn = torch.polar(torch.ones_like(axis), axis * c["theta"] ** -power)[:, None]
                turn = turn if c["op"] == "fwd" else turn.conj()
                u, v = (p, p + total) if c["layout"] == "halves" else (2 * p, 2 * p + 1)
                z = torch.complex(out[..., u], out[..., v]) * turn
                out[..., u], out[..., v] = z.real, z.imag
                p += 1
        done.append(out)
    return {"Q": done[0], "K": done[1]}


def exact(case, seed):
    c = case
    if "split" in c:
        return _exact_rotary(c, seed)
    state = prepare(dict(c), seed)
    q, k, v, do, kv_len = state["tensors"]
    hw, scale, group = c["h"] * c["w"], 1 / math.sqrt(c["dim"]), c["heads"] // c["kv_heads"]
    out = {name: torch.zeros(x.shape, dtype=torch.float64, device="cuda") for name, x in
           (("dQ", q), ("dK", k), ("dV", v), ("O", q), ("lse", q[..., 0]))}
    for b in range(c["batch"]):
        most = k.shape[2] if kv_len is None else int(kv_len[b])
        for head in range(c["heads"]):
            qh, doh = q[b, head].double(), do[b, head].double()
            kh, vh = (x[b, head // group].double() for x in (k, v))
            step = hw if c["chunk"] and hw > 1 else max(1, min(q.shape[2], (1 << 28) // max(1, k.shape[2])))
            for at in range(0, q.shape[2], step):
                rows = slice(at, min(at + step, q.shape[2]))
                z = scale * (qh[rows] @ kh[:most].t())
                if c["chunk"]:
                    frame = torch.arange(rows.start, rows.stop, device="cuda") // hw + c["offset"]
                    last = (frame // c["chunk"] + 1) * c["chunk"] * hw
                    z = z.masked_fill(torch.arange(most, device="cuda")[None] >= last[:, None], -math.inf)
                lse = torch.logsumexp(z, -1) if most else torch.full((z.shape[0],), -math.inf, dtype=torch.float64, device="cuda")
                w = torch.softmax(z, -1) if most else z
                o = w @ vh[:most]
                kept = state["kept"][0][b, head, rows].double() if c["op"] == "bwd" else o
                g = doh[rows] @ vh[:most].t() - (kept * doh[rows]).sum(-1, keepdim=True)
                g = scale * w * g
                out["O"][b, head, rows], out["lse"][b, head, rows] = o, lse
                out["dQ"][b, head, rows] = g @ kh[:most]
                out["dK"][b, head // group, :most] += g.t() @ qh[rows]
                out["dV"][b, head // group, :most] += w.t() @ doh[rows]
    return out if c["op"] == "step" else {n: out[n] for n in ("dQ", "dK", "dV")}
