"""The operators of a decoding step against a cache held in 8 bits, and the norm that precedes them: norms of queries
and keys with the position rotation in the same pass, forward and backward; rows written to and read from the cache; the
attention over it.

Every case is one pass through the public binding on device tensors.  With `own` false the same results are formed
from elementary torch operations in 32 bits (angles and long sums in 64), rounded once at the end.  Shapes are those of
a video diffusion transformer (latent grids of 30 x 52 and 45 x 80, chunks of three frames, 21 latent frames, heads of 128
or 64), of sequences of text and images, and of single tokens.

The cache: codes [batch, heads, tokens, head_dim], e4m3 or whole numbers of -127 .. 127, and one power of two for every
`block` tokens of a (batch, head), held as its exponent + 127.  A block's scale is the smallest that brings the block's largest
value to 448 (127) or below; the rows before a written one keep their values, rounded again where the scale grows.

`exact` states the results in 64 bits.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
_LARGEST = {"e4m3": 448.0, "int8": 127.0}


def _norm(op, grid, heads, *, kv_heads=None, offset=0, dtype="bf16", out="bf16", dim=128, batch=1, layout="adjacent",
          ladder="axis", split="", theta=10000.0, weight="f32", each=False, **named):
    # grid (f, h, w): tokens of a grid; (0, 0, n): n tokens of text and images at positions of their own.
    # each: a weight for every head, not one that the heads share
    f, h, w = grid
    return dict(named, op=op, batch=batch, heads=heads, kv_heads=kv_heads or heads, dim=dim, f=f, h=h, w=w, offset=offset,
                dtype=dtype, out=out, layout=layout, ladder=ladder, split=split, theta=theta, weight=weight, each=each)


def _cache(tokens, at, read, heads, *, room, batch=1, dim=128, format="e4m3", block=64, dtype="bf16", ragged=False, **named):
    # writes `tokens` rows at `at` (ragged: sequences are up to half as long), then reads the last `read` rows
    return dict(named, op="cache", tokens=tokens, at=at, read=read, heads=heads, room=room, batch=batch, dim=dim, format=format,
                block=block, dtype=dtype, ragged=ragged)


def _attn(grid, heads, *, f_kv, kv_heads=None, chunk=0, offset=0, dim=128, batch=1, format="e4m3", block=64, lengths="whole",
          **named):
    f, h, w = grid
    return dict(named, op="attn", f_q=f, f_kv=f_kv, h=h, w=w, heads=heads, kv_heads=kv_heads or heads, chunk=chunk, offset=offset,
                dim=dim, batch=batch, format=format, block=block, lengths=lengths)


def listed():
    return [
        # decoding: one token's query and key, far into a session; latency is all there is
        _norm("fwd", (0, 0, 1), 32, kv_heads=8, layout="halves", ladder="shared", split="16,24,24", theta=1e6, weight="bf16",
              name="norm-token"),
        # queries and keys of one autoregressive chunk late in a clip: the ordinary call
        _norm("fwd", (3, 30, 52), 12, offset=18, name="norm-chunk-480p"),
        # training on text and images in fp32, a weight for every head
        _norm("bwd", (0, 0, 4099), 32, kv_heads=8, batch=2, dtype="f32", out="f32", layout="halves", ladder="shared",
              split="16,24,24", theta=1e6, each=True, name="norm-bwd-text-image-f32"),
        # the largest: gradients of a whole 720p clip of a 40-head model
        _norm("bwd", (21, 45, 80), 40, name="norm-bwd-clip-720p"),
        # decoding: a token of each of eight sequences is appended, inside a block
        _cache(1, 4096, 64, 8, room=8192, batch=8, ragged=True, name="cache-token"),
        # the last chunk of a clip is written, and handed on in 16 bits as the cache holds it
        _cache(4680, 28080, 4680, 12, room=32760, name="cache-chunk-480p"),
        # the same, and the whole clip is read for an attention that takes 16 bits
        _cache(4680, 28080, 32760, 12, room=32760, format="int8", block=32, name="cache-clip-480p-int8"),
        # decoding: one token's queries, eight to a key head, sequences of unequal lengths
        _attn((1, 1, 1), 32, f_kv=32760, kv_heads=8, batch=4, lengths="spread", name="attn-token"),
        # a small model's layer on an odd grid, a padded batch: one clip whole, one cut short, one empty
        _attn((2, 17, 23), 4, f_kv=6, dim=64, batch=3, format="int8", block=32, lengths="padded", name="attn-padded-odd-d64"),
        # one frame against the clip
        _attn((1, 30, 52), 12, f_kv=21, format="int8", name="attn-frame-480p-int8"),
        # the ordinary call: the last chunk against the cached clip
        _attn((3, 30, 52), 12, f_kv=21, chunk=3, offset=18, name="attn-chunk-480p"),
        # the largest: the same at 720p
        _attn((3, 45, 80), 12, f_kv=21, chunk=3, offset=18, name="attn-chunk-720p"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def _candidate(rng):
    kind = rng.choice(["norm", "norm", "norm-text", "cache", "cache", "token", "pool", "frames", "clip", "text", "padded"])
    dim, batch = rng.choice([64, 128, 128]), rng.choice([1, 1, 2, 3])
    h, w, heads = _log_int(rng, 3, 45), _log_int(rng, 3, 80), _log_int(rng, 1, 40)
    kv = heads // rng.choice([n for n in (1, 1, 2, 3, 4, 5, 8) if heads % n == 0])
    if kind in ("norm", "norm-text"):
        op, each = rng.choice(["fwd", "bwd"]), rng.random() < 0.25
        dtype, out = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"), ("bf16", "f32")])
        layout, ladder = rng.choice([("adjacent", "axis"), ("adjacent", "shared"), ("halves", "axis"), ("halves", "shared")])
        weight = rng.choice(["f32", "bf16"])
        if kind == "norm":
            return _norm(op, (rng.randint(1, 21), h, w), heads, kv_heads=kv, offset=rng.choice([0, 18, 5000]), dtype=dtype, out=out,
                         dim=dim, batch=batch, layout=layout, ladder=ladder, weight=weight, each=each)
        dim = rng.choice([64, 72, 80, 96, 128, 256])
        part = rng.choice([8, 8, 16])      # the whole head, or half of it
        axes = [dim // part, dim // part, dim // (part // 2)]
        rng.shuffle(axes)
        return _norm(op, (0, 0, _log_int(rng, 1, 32768)), heads, kv_heads=kv, dtype=dtype, out=out, dim=dim, batch=batch,
                     layout=layout, ladder=ladder, split=",".join(map(str, axes)), theta=rng.choice([1e4, 1e6]), weight=weight,
                     each=each)
    form = dict(format=rng.choice(["e4m3", "e4m3", "int8"]), block=rng.choice([16, 32, 64, 128]), dim=dim)
    if kind == "cache":
        tokens, at = _log_int(rng, 1, 10800), rng.randint(0, 32768)
        read = min(at // 2 + tokens, _log_int(rng, 1, 32768))
        return _cache(tokens, at, read, kv, room=at + tokens + rng.randint(0, 200), batch=rng.choice([1, 1, 2, 5]),
                      dtype=rng.choice(["bf16", "bf16", "f32"]), ragged=rng.random() < 0.5, **form)
    if kind in ("token", "pool"):
        n = _log_int(rng, 1, 75600)
        return _attn((1 if kind == "token" else rng.randint(2, 16), 1, 1), heads, f_kv=n, kv_heads=kv, batch=rng.choice([1, 2, 4, 8]),
                     lengths=rng.choice(["whole", "spread"]), **form)
    if kind == "frames":
        n = rng.randint(1, 21)
        f = rng.randint(1, min(3, n))
        return _attn((f, h, w), heads, f_kv=n, kv_heads=kv, batch=batch, **form)
    if kind == "clip":
        f, before = 3 * rng.randint(1, 4), 3 * rng.randint(0, 3)
        return _attn((f, h, w), heads, f_kv=f + before, kv_heads=kv, chunk=rng.choice([1, 3]), offset=before, batch=batch, **form)
    if kind == "text":
        n, before = _log_int(rng, 1, 4096), rng.choice([0, _log_int(rng, 1, 16384)])
        return _attn((n, 1, 1), heads, f_kv=n + before, kv_heads=kv, chunk=1, offset=before, batch=batch, **form)
    return _attn((rng.randint(1, 3), h, w), heads, f_kv=rng.randint(3, 9), kv_heads=kv, batch=rng.randint(2, 4), lengths="padded", **form)


def _kind(c):
    return c["op"] if c["op"] in ("cache", "attn") else "norm"


def _cost(c):
    """A rough time of the plain form in seconds, to keep drawn cases below the largest listed one of their kind."""
    if _kind(c) == "attn":
        return c["batch"] * c["heads"] * c["f_q"] * c["f_kv"] * (c["h"] * c["w"]) ** 2 * (4 * c["dim"] + 1500) / 6e13
    return work(c)["bytes"] / 1e12


def draw(rng):
    most = {}
    for c in listed():
        most[_kind(c)] = max(most.get(_kind(c), 0), _cost(c))
    while True:
        c = _candidate(rng)
        if _cost(c) <= 0.9 * most[_kind(c)]:
            return c


# ---- inputs --------------------------------------------------------------------------------------
def _normal(gen, *shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="cuda").normal_(generator=gen)


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
    """x [batch, heads, tokens, dim]; angles [(batch,) tokens, pairs]."""
    angles = angles if angles.dim() == 2 else angles[:, None]
    cos, sin = angles.cos().to(x.dtype), (sign * angles.sin()).to(x.dtype)
    n = angles.shape[-1]
    if layout == "halves":
        a, b, rest = x[..., :n], x[..., n:2 * n], x[..., 2 * n:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], -1)
    a, b, rest = x[..., 0:2 * n:2], x[..., 1:2 * n:2], x[..., 2 * n:]
    return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), rest], -1)


def _norm_tensors(c, seed):
    """[(rows, gradients of the results or None, weight)] of queries and keys, positions or None."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = c["w"] if c["f"] == 0 else c["f"] * c["h"] * c["w"]
    positions = _text_positions(c, gen) if c["f"] == 0 else None
    sides = []
    for heads, spread in ((c["heads"], 1.5), (c["kv_heads"], 0.5)):      # (queries and keys leave their products at unlike scales)
        shape = (c["batch"], heads, n, c["dim"])
        x = _normal(gen, *shape, dtype=_DTYPES[c["dtype"]]).mul_(spread)
        g = _normal(gen, *shape, dtype=_DTYPES[c["out"]]) if c["op"] == "bwd" else None
        weight = 1 + 0.2 * _normal(gen, *((heads, c["dim"]) if c["each"] else (c["dim"],)))
        sides.append((x, g, weight.to(_DTYPES[c["weight"]])))
    return sides, positions


def _rows(c, gen, heads, tokens, dtype=torch.float32):
    """Rows as a layer's keys or values: features of unlike size, a few large ones."""
    size = torch.exp(0.5 * _normal(gen, 1, heads, 1, c["dim"]))
    return (_normal(gen, c["batch"], heads, tokens, c["dim"]) * size).to(dtype)


def _code_values(codes):
    return codes.float()


def _scale_of(exponents):
    return torch.ldexp(torch.ones_like(exponents, dtype=torch.float32), exponents.int() - 127)


def _exponents(largest, format):
    """Exponent bytes of blocks whose largest magnitudes are `largest`."""
    fraction, power = torch.frexp(largest)
    top, bits = math.frexp(_LARGEST[format])
    power = power - bits + (fraction > top).int()
    return torch.where(largest == 0, torch.full_like(power, 3), (power + 127).clamp(3, 246)).to(torch.uint8)


def _encode(x, exponents, format):
    x = (x / _scale_of(exponents)).clamp(-_LARGEST[format], _LARGEST[format])
    return (x.round() if format == "int8" else x).to(_CODES[format])


def _new_cache(c, gen, heads, tokens):
    """(codes, exponents) of a tensor [batch, heads, tokens, dim], and its float values' maker's shape."""
    blocks, block = -(-tokens // c["block"]), c["block"]
    x = _rows(c, gen, heads, blocks * block).unflatten(2, (blocks, block))
    exponents = _exponents(x.abs().amax((-1, -2)), c["format"])
    codes = _encode(x, exponents[..., None, None], c["format"]).flatten(2, 3)
    return codes[:, :, :tokens].contiguous(), exponents


def _lengths(c):
    """Keys of every sequence."""
    n = c["f_kv"] * c["h"] * c["w"]
    if c["lengths"] == "whole":
        return None
    if c["lengths"] == "spread":      # from a part of the longest to the longest
        return [max(1, n * (i + 1) // c["batch"]) for i in range(c["batch"])]
    return [n] + [(3 * n) // (4 + i) for i in range(c["batch"] - 2)] + [0]      # whole, cut short, empty


def _whole_numbers(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    c = case
    if _kind(c) == "norm":
        sides, positions = _norm_tensors(c, seed)
        return {"case": c, "sides": sides, "positions": positions}
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if c["op"] == "cache":
        cache = [_new_cache(c, gen, c["heads"], c["room"]) for _ in range(2)]
        rows = [_rows(c, gen, c["heads"], c["tokens"], _DTYPES[c["dtype"]]) for _ in range(2)]
        at = read_at = None
        if c["ragged"]:
            lo = max(c["at"] // 2, c["read"] - c["tokens"])
            at = torch.randint(lo, max(lo, c["at"]) + 1, (c["batch"],), generator=gen, device="cuda").int()
            read_at = at + (c["tokens"] - c["read"])
        return {"case": c, "cache": cache, "rows": rows, "at": at, "read_at": read_at}
    nq, nkv = c["f_q"] * c["h"] * c["w"], c["f_kv"] * c["h"] * c["w"]
    cache = [_new_cache(c, gen, c["kv_heads"], nkv) for _ in range(2)]
    q = _normal(gen, c["batch"], c["heads"], nq, c["dim"]).mul_(1.5).bfloat16()
    lengths = _lengths(c)
    return {"case": c, "cache": cache, "q": q, "lengths": None if lengths is None else _whole_numbers(lengths)}


# ---- one pass ------------------------------------------------------------------------------------
def _run_norm(c, sides, positions):
    eps = 1e-6
    if own:
        import paper_2602_12271_amd as mrt
        args = dict(eps=eps, theta=c["theta"], layout=c["layout"], ladder=c["ladder"], split=_pairs(c))
        if positions is not None:
            args.update(q_positions=positions, k_positions=positions)
        else:
            args.update(f_q=c["f"], f_kv=c["f"], h=c["h"], w=c["w"], q_frame_offset=c["offset"], kv_frame_offset=c["offset"])
        (q, dq, qw), (k, dk, kw) = sides
        if c["op"] == "fwd":
            return dict(zip(("Q", "K"), mrt.norm_rotary_fwd(q, k, qw, kw, dtype=_DTYPES[c["out"]], **args)))
        return dict(zip(("dQ", "dK", "dqw", "dkw"), mrt.norm_rotary_bwd(q, k, qw, kw, dq, dk, **args)))
    positions = _clip_positions(c["f"], c["h"], c["w"], c["offset"]) if positions is None else positions
    angles = _angles(_pairs(c), c["ladder"], c["theta"], positions)
    out = {}
    for name, (x, g, weight) in zip("QK", sides):
        dtype = x.dtype
        x = x.float()
        weight = weight.float()[:, None] if c["each"] else weight.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
        if c["op"] == "fwd":
            out[name] = _rotate(x * r * weight, angles, c["layout"], 1).to(_DTYPES[c["out"]])
            continue
        g = _rotate(g.float(), angles, c["layout"], -1)
        x = x * r
        h = g * x
        # (a sum over up to millions of rows)
        out["d" + name.lower() + "w"] = h.double().sum((0, 2) if c["each"] else (0, 1, 2)).float()
        h = (h * weight).mean(-1, keepdim=True)
        out["d" + name] = ((g * weight - x * h) * r).to(dtype)
    return out


def _plain_write(c, codes, exponents, rows, at):
    """Writes the rows at `at` ([batch], whole numbers) in place."""
    block, format = c["block"], c["format"]
    blocks = exponents.shape[2]
    n = rows.shape[2]
    b = torch.arange(c["batch"], device="cuda")
    first = torch.div(at, block, rounding_mode="floor")
    span = (n + block - 2) // block + 1                                  # blocks a run may touch
    index = first[:, None] + torch.arange(span, device="cuda")           # [batch, span]
    there = (index <= torch.div(at + n - 1, block, rounding_mode="floor")[:, None]) & (index < blocks)
    held = index.clamp(max=blocks - 1)
    token = index[:, :, None] * block + torch.arange(block, device="cuda")
    token = token.flatten(1)                                             # [batch, span * block]
    inside = token.clamp(max=codes.shape[2] - 1)
    old = codes.view(torch.uint8)[b[:, None], :, inside].view(codes.dtype)            # [batch, tokens, heads, dim]
    scale = _scale_of(exponents[b[:, None], :, held]).repeat_interleave(block, 1)     # [batch, tokens, heads]
    old = _code_values(old) * scale[..., None]
    new = token - at[:, None]
    fresh = (new >= 0) & (new < n)
    kept = (new < 0) & (token < codes.shape[2])
    picked = rows.float().transpose(1, 2)[b[:, None], new.clamp(0, n - 1)]
    x = torch.where(fresh[:, :, None, None], picked, torch.where(kept[:, :, None, None], old, torch.zeros_like(old)))
    x = x.unflatten(1, (span, block))
    power = _exponents(x.abs().amax((2, 4)), format)                     # [batch, span, heads]
    x = _encode(x, power[:, :, None, :, None], format).flatten(1, 2)
    write = (fresh | kept) & there.repeat_interleave(block, 1)
    bi, ti = torch.nonzero(write, as_tuple=True)
    codes.view(torch.uint8)[bi, :, token[bi, ti]] = x.view(torch.uint8)[bi, ti]
    bi, ti = torch.nonzero(there, as_tuple=True)
    exponents[bi, :, index[bi, ti]] = power[bi, ti]


def _run_cache(state):
    c = state["case"]
    (k8, ks), (v8, vs) = state["cache"]
    read_at = c["at"] + c["tokens"] - c["read"]
    if own:
        import paper_2602_12271_amd as mrt
        cache = mrt.Cache8(k8, v8, ks, vs, c["block"])
        mrt.cache8_write(cache, *state["rows"], at=c["at"] if state["at"] is None else state["at"])
        k, v = mrt.cache8_read(cache, c["read"], at=read_at if state["read_at"] is None else state["read_at"])
        return {"K": k, "V": v}
    at = state["at"].long() if state["at"] is not None else torch.full((c["batch"],), c["at"], device="cuda")
    read_at = at + c["tokens"] - c["read"]
    out = {}
    for name, (codes, exponents), rows in zip("KV", state["cache"], state["rows"]):
        _plain_write(c, codes, exponents, rows, at)
        b = torch.arange(c["batch"], device="cuda")[:, None]
        token = read_at[:, None] + torch.arange(c["read"], device="cuda")
        x = _code_values(codes.view(torch.uint8)[b, :, token].view(codes.dtype))
        scale = _scale_of(exponents[b, :, torch.div(token, c["block"], rounding_mode="floor")])
        out[name] = (x * scale[..., None]).bfloat16().transpose(1, 2).contiguous()
    return out


def _values(c, codes, exponents):
    return _code_values(codes) * _scale_of(exponents).repeat_interleave(c["block"], 2)[:, :, :codes.shape[2], None]


def _hidden(c, nq, nkv, lengths, device):
    """[batch or 1, 1, 1, queries, keys] truth values, or None."""
    hidden = None
    if c["chunk"]:
        hw = c["h"] * c["w"]
        chunk_q = torch.div(c["offset"] + torch.arange(nq, device=device) // hw, c["chunk"], rounding_mode="floor")
        chunk_k = torch.div(torch.arange(nkv, device=device) // hw, c["chunk"], rounding_mode="floor")
        hidden = (chunk_k[None, :] > chunk_q[:, None])[None, None, None]
    if lengths is not None:
        past = (torch.arange(nkv, device=device)[None] >= lengths[:, None])[:, None, None, None]
        hidden = past if hidden is None else hidden | past
    return hidden


def _run_attn(state):
    c, q, lengths = state["case"], state["q"], state["lengths"]
    (k8, ks), (v8, vs) = state["cache"]
    if own:
        import paper_2602_12271_amd as mrt
        o, lse = mrt.dense_attn_fwd_cache8(q, mrt.Cache8(k8, v8, ks, vs, c["block"]), f_q=c["f_q"], f_kv=c["f_kv"], h=c["h"], w=c["w"],
                                           causal_chunk=c["chunk"], q_frame_offset=c["offset"], scale=1 / math.sqrt(c["dim"]),
                                           kv_len=lengths)
        return {"O": o, "lse": lse}
    k, v = _values(c, k8, ks), _values(c, v8, vs)
    nq, nkv = q.shape[2], k.shape[2]
    hidden = _hidden(c, nq, nkv, lengths, q.device)
    group = c["heads"] // c["kv_heads"]
    qs = q.float().unflatten(1, (c["kv_heads"], group))
    o, lse = torch.empty_like(qs), torch.empty_like(qs[..., 0])
    step = max(1, (1 << 30) // (c["batch"] * group * nq * nkv))
    for at in range(0, c["kv_heads"], step):
        s = torch.matmul(qs[:, at:at + step], k[:, at:at + step, None].transpose(-1, -2)).mul_(1 / math.sqrt(c["dim"]))
        if hidden is not None:
            s.masked_fill_(hidden, -math.inf)
        top = s.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        s = s.sub_(top).exp_()
        total = s.sum(-1, keepdim=True)
        o[:, at:at + step] = torch.matmul(s, v[:, at:at + step, None]) / torch.where(total == 0, torch.ones_like(total), total)
        lse[:, at:at + step] = (total.log() + top).squeeze(-1)
    return {"O": o.flatten(1, 2).bfloat16(), "lse": lse.flatten(1, 2)}


def run(state):
    c = state["case"]
    if c["op"] == "cache":
        return _run_cache(state)
    if c["op"] == "attn":
        return _run_attn(state)
    return _run_norm(c, state["sides"], state["positions"])


def _seen(c):
    """(query, key) pairs of one query head that take part, over the batch, and keys that some query sees."""
    hw = c["h"] * c["w"]
    pairs = keys = 0
    for n in _lengths(c) or [c["f_kv"] * hw] * c["batch"]:
        last = 0
        for f in range(c["f_q"]):
            last = min(n, ((f + c["offset"]) // c["chunk"] + 1) * c["chunk"] * hw) if c["chunk"] else n
            pairs += hw * last
        keys += last
    return pairs, keys


def work(case):
    c = case
    if c["op"] == "attn":
        pairs, keys = _seen(c)
        rows = c["batch"] * c["heads"] * c["f_q"] * c["h"] * c["w"]
        return {"bytes": rows * (4 * c["dim"] + 4) + 2 * keys * c["kv_heads"] * c["dim"], "flops": 4 * c["heads"] * pairs * c["dim"]}
    if c["op"] == "cache":
        size = {"bf16": 2, "f32": 4}[c["dtype"]]
        row = 2 * c["batch"] * c["heads"] * c["dim"]
        # rows in, their codes; codes of the rows that are read, their values
        return {"bytes": row * (c["tokens"] * (size + 1) + c["read"] * (1 + 2)), "flops": row * (3 * c["tokens"] + c["read"])}
    x, y = ({"bf16": 2, "f32": 4}[c[n]] for n in ("dtype", "out"))
    n = (c["w"] if c["f"] == 0 else c["f"] * c["h"] * c["w"]) * c["batch"]
    elements = n * (c["heads"] + c["kv_heads"]) * c["dim"]
    return {"bytes": elements * (x + y if c["op"] == "fwd" else 2 * x + y) + (12 * n if c["f"] == 0 else 0),
            "flops": elements * (7 if c["op"] == "fwd" else 14)}


# ---- the same results in 64 bits -----------------------------------------------------------------
def _turns(c, positions):
    """[batch or 1, tokens, pairs], complex: the turn of every pair."""
    n = c["w"] if c["f"] == 0 else c["f"] * c["h"] * c["w"]
    if positions is None:
        token = torch.arange(n, device="cuda")
        axes = [x[None].double() for x in (token // (c["w"] * c["h"]) + c["offset"], token // c["w"] % c["h"], token % c["w"])]
    else:
        axes = [positions[:, i].double() for i in range(3)]
    pairs, columns, p = _pairs(c), [], 0
    for axis, count in zip(axes, pairs):
        for i in range(count):
            columns.append(axis * c["theta"] ** -(p / sum(pairs) if c["ladder"] == "shared" else i / count))
            p += 1
    angle = torch.stack(columns, -1)
    return torch.polar(torch.ones_like(angle), angle)


def _exact_norm(c, seed):
    sides, positions = _norm_tensors(c, seed)
    turns, out = _turns(c, positions), {}
    pairs = turns.shape[-1]
    first = torch.arange(pairs, device="cuda") * (1 if c["layout"] == "halves" else 2)
    second = first + (pairs if c["layout"] == "halves" else 1)

    def turned(x, by):
        x = x.clone()
        z = torch.complex(x[:, first], x[:, second]) * by
        x[:, first], x[:, second] = z.real, z.imag
        return x
    for name, (x, g, weight) in zip("QK", sides):
        backward = c["op"] == "bwd"
        result = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        grad = torch.zeros(weight.shape, dtype=torch.float64, device="cuda")
        for b in range(x.shape[0]):
            turn = turns[b if turns.shape[0] > 1 else 0]
            for head in range(x.shape[1]):
                row = x[b, head].double()
                w = (weight[head] if c["each"] else weight).double()
                size = (row.square().sum(-1, keepdim=True) / c["dim"] + 1e-6).sqrt()
                unit = row / size
                if not backward:
                    result[b, head] = turned(unit * w, turn)
                    continue
                back = turned(g[b, head].double(), turn.conj())
                part = (back * unit).sum(0)
                if c["each"]:
                    grad[head] += part
                else:
                    grad += part
                back = back * w
                result[b, head] = (back - unit * (back * unit).sum(-1, keepdim=True) / c["dim"]) / size
        out[("d" if backward else "") + name] = result
        if backward:
            out["d" + name.lower() + "w"] = grad
    return out


def _table(format):
    """The value of every code, by its bits."""
    if format == "int8":
        return torch.tensor([i - 256 if i > 127 else i for i in range(256)], dtype=torch.float64, device="cuda")
    values = []
    for i in range(256):
        power, rest = i >> 3 & 15, i & 7
        x = math.nan if i & 127 == 127 else rest / 8 * 2.0 ** -6 if power == 0 else (1 + rest / 8) * 2.0 ** (power - 7)
        values.append(-x if i & 128 else x)
    return torch.tensor(values, dtype=torch.float64, device="cuda")


def _exact_values(c, codes, exponents):
    x = _table(c["format"])[codes.view(torch.uint8).long()]
    power = exponents.double().sub(127).exp2()
    at = torch.arange(codes.shape[-2], device="cuda") // c["block"]
    return x * power[..., at, None]


def _nearest(x, format):
    """x, already divided by its scale, as the nearest code's value."""
    if format == "int8":
        return x.round()
    power = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -9))).clamp(min=-6)
    step = torch.exp2(power - 3)
    return (x / step).round() * step


def _exact_cache(c, seed):
    state = prepare(dict(c), seed)
    out, block = {}, c["block"]
    for name, (codes, exponents), rows in zip("KV", state["cache"], state["rows"]):
        result = torch.empty(c["batch"], c["heads"], c["read"], c["dim"], dtype=torch.float64, device="cuda")
        for b in range(c["batch"]):
            at = c["at"] if state["at"] is None else int(state["at"][b])
            end = at + c["tokens"]
            lo, start = end - c["read"], at - at % block
            if lo < at:
                result[b, :, :at - lo] = _exact_values(c, codes[b], exponents[b])[:, lo:at]
            x = torch.cat([_exact_values(c, codes[b], exponents[b])[:, start:at], rows[b].double()], 1)
            x = torch.nn.functional.pad(x, (0, 0, 0, -x.shape[1] % block)).unflatten(1, (-1, block))
            scale = x.abs().amax((-1, -2), keepdim=True) / _LARGEST[c["format"]]
            fraction, power = torch.frexp(scale.clamp(min=2.0 ** -124))
            scale = torch.exp2((power - (fraction == 0.5).int()).double())
            x = (_nearest(x / scale, c["format"]) * scale).flatten(1, 2)[:, :end - start]
            keep = min(c["read"], end - start)
            result[b, :, c["read"] - keep:] = x[:, x.shape[1] - keep:]
        out[name] = result
    return out


def exact(case, seed):
    c = case
    if _kind(c) == "norm":
        return _exact_norm(c, seed)
    if c["op"] == "cache":
        return _exact_cache(c, seed)
    state = prepare(dict(c), seed)
    q, lengths = state["q"], _lengths(c)
    k, v = (_exact_values(c, *x) for x in state["cache"])
    hw, group = c["h"] * c["w"], c["heads"] // c["kv_heads"]
    out = {"O": torch.zeros(q.shape, dtype=torch.float64, device="cuda"),
           "lse": torch.full(q.shape[:3], -math.inf, dtype=torch.float64, device="cuda")}
    for b in range(c["batch"]):
        most = k.shape[2] if lengths is None else lengths[b]
        if most == 0:
            continue
        for head in range(c["heads"]):
            kh, vh = k[b, head // group, :most], v[b, head // group, :most]
            step = max(1, min(q.shape[2], (1 << 28) // most))
            for at in range(0, q.shape[2], step):
                rows = slice(at, min(at + step, q.shape[2]))
                z = (q[b, head, rows].double() @ kh.t()) / math.sqrt(c["dim"])
                if c["chunk"]:
                    frame = torch.arange(rows.start, rows.stop, device="cuda") // hw + c["offset"]
                    last = (frame // c["chunk"] + 1) * c["chunk"] * hw
                    z = z.masked_fill(torch.arange(most, device="cuda")[None] >= last[:, None], -math.inf)
                out["lse"][b, head, rows] = torch.logsumexp(z, -1)
                out["O"][b, head, rows] = torch.softmax(z, -1) @ vh
    return out
