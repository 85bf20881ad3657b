"""How far a value of a cache of 8 bits may be off: rows written once, kernels and definition.  A whole number by half the scale, which
is less than 1/127 of the block's largest magnitude, since half of the smallest power of two that holds it would not; 2^-7 of that
magnitude is not enough where it lies just above 127 times a power of two."""
import pytest
import torch

import paper_2602_12271_amd as pkg
from decoding import LARGEST, HostCache


def blocks():
    """16 x 16 entries each: one of many sizes, and largest magnitudes at, just above and well above 127 and 448 times a power of two."""
    gen = torch.Generator().manual_seed(11)
    x = torch.randn(12, 256, generator=gen, dtype=torch.float64)
    tops = [127.0, 127.25, 127.5, 128.0, 200.0, 253.0, 254.5, 448.0, 449.0, 600.0, 127.25 * 2.0 ** -20, 449.0 * 2.0 ** 30]
    for i, top in enumerate(tops):
        x[i] *= top / 2 / x[i].abs().max()
        x[i, 0], x[i, 1] = top, 65.0 / 127.25 * top
    return x.float()


def check(x, values, scales, format):
    x, values = x.double(), values.double()
    top = x.abs().amax(1, keepdim=True)
    assert (top <= LARGEST[format] * scales).all() and (top > LARGEST[format] * scales / 2).all()
    off = (values - x).abs()
    if format == "e4m3":
        # four significant bits: half a step is 2^-4 of the value at most, subnormal steps are 2^-9 of the scale
        assert (off <= (2.0 ** -4 * x.abs()).maximum(2.0 ** -10 * scales)).all()
    else:
        assert (off <= scales / 2).all() and (scales / 2 < top / 127).all()
        assert off[1, 1] == 1.0 and off[1, 1] > 2.0 ** -7 * 127.25                 # 65 under a scale of 2


@pytest.mark.parametrize("format", ["e4m3", "int8"])
def test_definition(format):
    x = blocks()
    host = HostCache(16 * x.shape[0], 16, 16, format)
    host.write(x.reshape(-1, 16), 0)
    check(x, host.values(torch.arange(16 * x.shape[0])).view(x.shape), 2.0 ** (host.bytes[:, None] - 127).double(), format)


@pytest.mark.gpu
@pytest.mark.parametrize("format", ["e4m3", "int8"])
def test_kernels(format):
    x = blocks()
    rows = x.reshape(1, 1, -1, 16).cuda()
    cache = pkg.cache8(1, 1, rows.shape[2], 16, format=format, block=16)
    pkg.cache8_write(cache, rows, rows.flip(3).contiguous())
    for values, scales, flip in zip(pkg.cache8_read(cache, rows.shape[2], dtype=torch.float32), (cache.K_scale, cache.V_scale), (False, True)):
        values = values.cpu()[0, 0]
        values = (values.flip(1) if flip else values).reshape(x.shape)
        check(x, values, 2.0 ** (scales.cpu()[0, 0, :, None].double() - 127), format)


@pytest.mark.gpu
@pytest.mark.parametrize("format", ["e4m3", "int8"])
def test_rows_behind_are_replaced(format):
    """A block's last rows written again and again, larger and smaller: the rows before them are off by what the largest scale costs."""
    gen = torch.Generator().manual_seed(5)
    block, n, first = 32, 8, 20
    kept = torch.randn(1, 1, first, 64, generator=gen)
    cache, host = pkg.cache8(1, 1, block, 64, format=format, block=block), HostCache(block, 64, block, format)
    pkg.cache8_write(cache, kept.cuda(), kept.cuda())
    host.write(kept[0, 0], 0)
    largest = int(host.bytes[0])
    for size in (1.0, 40.0, 3.0, 11.0, 0.01):
        rows = size * torch.randn(1, 1, n, 64, generator=gen)
        pkg.cache8_write(cache, rows.cuda(), rows.cuda(), at=first)
        host.write(rows[0, 0], first)
        largest = max(largest, int(host.bytes[0]))
        values = pkg.cache8_read(cache, first, dtype=torch.float32)[0][0, 0].cpu().double()
        assert torch.equal(values, host.values(torch.arange(first)))
        off, unit = (values - kept[0, 0].double()).abs(), 2.0 ** (largest - 127)
        # an e4m3 code: rounded once as a normal one, 2^-4 of it; where growing scales make it subnormal, by 2^-10 of each, 2^-9 of the
        # largest in all; a whole number by half of each, one unit of the largest in all
        assert (off <= (2.0 ** -4 * kept[0, 0].double().abs() + 2.0 ** -9 * unit if format == "e4m3" else unit)).all()
    assert int(host.bytes[0]) < largest
    if format == "int8":
        assert off.max() > 2.0 ** (int(host.bytes[0]) - 127)          # more than one unit of the last scale
