"""The norm with rotary positions and the 8-bit cache in 64 bits on the host, written from the formulas; shared by the tests
of the decoding step."""
from __future__ import annotations

import math

import torch

LARGEST = {"e4m3": 448.0, "int8": 127.0}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


# ---- norms with rotary positions -------------------------------------------------------------------
def pair_index(dim, split, layout):
    """Features of the first and of the second half of every pair."""
    total = sum(split)
    first = torch.arange(total) * (2 if layout == "adjacent" else 1)
    return first, first + (1 if layout == "adjacent" else total)


def angles(positions, split, theta, ladder):
    """[batch or 1, tokens, pairs] for positions [3, tokens] or [batch, 3, tokens]."""
    positions = (positions if positions.dim() == 3 else positions[None]).double()
    columns = []
    for axis, count in enumerate(split):
        for i in range(count):
            columns.append(positions[:, axis] * theta ** -(len(columns) / sum(split) if ladder == "shared" else i / count))
    return torch.stack(columns, -1)


def turned(x, angle, split, layout, sign=1):
    """x [batch, heads, tokens, dim]."""
    first, second = pair_index(x.shape[-1], split, layout)
    c, s = torch.cos(angle)[:, None], sign * torch.sin(angle)[:, None]
    y = x.clone()
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., first] * s + x[..., second] * c
    return y


def pair_size(x, split, layout):
    """The sum of magnitudes of an entry's pair, of an entry itself where it has none."""
    first, second = pair_index(x.shape[-1], split, layout)
    y = x.abs().clone()
    y[..., first] = y[..., second] = x[..., first].abs() + x[..., second].abs()
    return y


def weight_rows(weight, heads, dim):
    """[1, heads or 1, 1, dim] in 64 bits."""
    if weight is None:
        return torch.ones(1, 1, 1, dim, dtype=torch.float64)
    return weight.double().reshape(1, -1, 1, dim)


def norm_forward(x, weight, eps, angle, split, layout):
    x = x.double()
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    return turned(x * r * weight_rows(weight, x.shape[1], x.shape[-1]), angle, split, layout)


def norm_backward(x, weight, eps, angle, split, layout, dy):
    """dx, dw (in the weight's shape, or None)."""
    x, w = x.double(), weight_rows(weight, x.shape[1], x.shape[-1])
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    n, g = x * r, turned(dy.double(), angle, split, layout, -1)
    dx = r * (g * w - n * (g * w * n).mean(-1, keepdim=True))
    dw = None if weight is None else (g * n).sum((0, 2) if weight.dim() == 2 else (0, 1, 2))
    return dx, dw


# ---- the cache -------------------------------------------------------------------------------------
def code_values(format):
    """The value of each of the 256 codes, by its bits."""
    if format == "int8":
        return torch.tensor([float(i - 256 if i > 127 else i) for i in range(256)], dtype=torch.float64)
    values = []
    for i in range(256):
        power, rest = i >> 3 & 15, i & 7
        x = math.nan if i & 127 == 127 else rest / 8 * 2.0 ** -6 if power == 0 else (1 + rest / 8) * 2.0 ** (power - 7)
        values.append(-x if i & 128 else x)
    return torch.tensor(values, dtype=torch.float64)


def nearest(x, format):
    """The value of the nearest code, ties to even, of x within the codes' range."""
    if format == "int8":
        return x.round()
    _, power = torch.frexp(x)                       # x = f 2^power, f in 1/2 .. 1: four significant bits are steps of 2^(power - 4)
    step = torch.exp2((power - 4).clamp(min=-9).double())
    return (x / step).round() * step


def scale_byte(x, format):
    """The byte of a block of numbers."""
    finite = x[torch.isfinite(x)].abs()
    most = math.inf if torch.isinf(x).any() else float(finite.max()) if finite.numel() else 0.0
    if most == math.inf:
        return 246
    byte = 3
    while byte < 246 and most > LARGEST[format] * 2.0 ** (byte - 127):
        byte += 1
    return byte


def quantised(x, format, byte):
    """Values of the codes of x (64 bits) under a scale, divided by it."""
    z = x / 2.0 ** (byte - 127)
    z = z.clamp(-LARGEST[format], LARGEST[format])          # (keeps NaN)
    y = nearest(torch.nan_to_num(z), format)
    return torch.where(torch.isnan(x), torch.full_like(y, math.nan if format == "e4m3" else 0.0), y)


class HostCache:
    """One (batch, head) of K or V."""

    def __init__(self, capacity, dim, block, format):
        self.block, self.format = block, format
        self.codes = torch.zeros(capacity, dim, dtype=torch.float64)            # the codes' values
        self.bytes = torch.full((-(-capacity // block),), 3, dtype=torch.int64)

    def write(self, rows, at):
        rows = rows.double()
        if at < 0:
            rows, at = rows[-at:], 0
        end = min(at + rows.shape[0], self.codes.shape[0])
        for j in range(at // self.block, -(-end // self.block)):
            first, last = j * self.block, min((j + 1) * self.block, end)
            if last <= at:
                continue
            kept = self.codes[first:max(first, at)] * 2.0 ** (int(self.bytes[j]) - 127)
            new = torch.cat([kept, rows[max(first, at) - at:last - at]])
            self.bytes[j] = scale_byte(new, self.format)
            self.codes[first:last] = quantised(new, self.format, int(self.bytes[j]))

    def values(self, tokens):
        scale = 2.0 ** (self.bytes[tokens // self.block] - 127).double()
        return self.codes[tokens] * scale[:, None]
