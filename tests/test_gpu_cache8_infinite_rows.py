"""GPU: infinite entries in rows for a cache of 8 bits.  They do not cost rows that are there: a block that keeps some has the scale
of its finite magnitudes, under which an infinity is the largest code."""
import math

import pytest
import torch

import paper_2602_12271_amd as pkg
from decoding import LARGEST, code_values, quantised, scale_byte

pytestmark = pytest.mark.gpu

INF, NAN = math.inf, math.nan


def held(cache, b, head, first, n):
    """Codes' values and scale byte of n tokens of one block, of K and of V."""
    format = "e4m3" if cache.K.dtype == torch.float8_e4m3fn else "int8"
    for codes, scales in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)):
        yield code_values(format)[codes[b, head, first:first + n].view(torch.uint8).cpu().long()], int(scales[b, head, first // cache.block])


def same(x, y):
    return torch.equal(x.isnan(), y.isnan()) and torch.equal(x.nan_to_num(), y.nan_to_num())


# tokens of a block times features: a block of a wave and of a workgroup, one and several accesses a thread
@pytest.mark.parametrize("block, dim", [(16, 16), (32, 64), (64, 128), (128, 256)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("format", ["e4m3", "int8"])
def test_kept_rows_stay(format, dtype, block, dim):
    gen = torch.Generator().manual_seed(block + dim)
    kept, new = block // 2 + 1, 3
    first = block                                  # the second of three blocks
    k, v = (torch.randn(1, 2, first + kept, dim, generator=gen).to(dtype) for _ in range(2))
    cache = pkg.cache8(1, 2, 3 * block, dim, format=format, block=block)
    pkg.cache8_write(cache, k.cuda(), v.cuda())
    before = [list(held(cache, 0, h, first, kept)) for h in range(2)]
    rows = [torch.randn(1, 2, new, dim, generator=gen).to(dtype) * 3 for _ in range(2)]
    rows[0][0, 0, 0, 1], rows[0][0, 0, 2, dim - 1], rows[0][0, 0, 1, 3] = INF, -INF, NAN      # (V, and the other head, have none)
    print(format, dtype, block, dim, flush=True)
    pkg.cache8_write(cache, *(x.cuda() for x in rows), at=first + kept)
    for h in range(2):
        for side, ((codes, byte), (old, was), x) in enumerate(zip(held(cache, 0, h, first, kept + new), before[h], rows)):
            values = torch.cat([old * 2.0 ** (was - 127), x[0, h].double()])
            want = scale_byte(values[torch.isfinite(values)], format)
            assert byte == want, (h, side, byte, want)
            assert same(codes, quantised(values, format, want)), (h, side)
    got = pkg.cache8_read(cache, kept, at=first, dtype=torch.float32)[0][0, 0].cpu()
    x = k[0, 0, first:].float()
    # two roundings of a kept entry: of e4m3 2^-4 of it each, or 2^-10 of the scale; of whole numbers half of the first scale and of the last
    scales = [2.0 ** (byte - 127) for byte in (before[0][0][1], next(held(cache, 0, 0, first, 1))[1])]
    bound = sum((x.abs() * 2.0 ** -4).clamp(min=2.0 ** -10 * s) if format == "e4m3" else torch.full_like(x, s / 2) for s in scales)
    assert ((got - x).abs() <= bound * (1 + 2.0 ** -3)).all()


@pytest.mark.parametrize("format", ["e4m3", "int8"])
def test_places_of_their_own(format):
    """A token of every sequence, inside a block and at the beginning of one."""
    cache = pkg.cache8(3, 1, 32, 16, format=format, block=16)
    ones = torch.ones(3, 1, 20, 16, device="cuda")
    pkg.cache8_write(cache, ones, ones)
    row = torch.full((3, 1, 1, 16), 2.0, device="cuda")
    row[:, :, :, 5] = -INF
    at = torch.tensor([20, 16, 7], dtype=torch.int32, device="cuda")
    pkg.cache8_write(cache, row, row, at=at)
    K, V = (x.cpu() for x in pkg.cache8_read(cache, 32, dtype=torch.float32))
    most = LARGEST[format]
    for x in (K, V):
        assert (x[0, 0, :20] == 1).all() and (x[1, 0, :16] == 1).all() and (x[2, 0, :7] == 1).all()
        for b, t in ((0, 20), (2, 7)):
            scale = 2.0 ** (scale_byte(torch.tensor([1.0, 2.0]), format) - 127)
            want = torch.full((16,), 2.0)
            want[5] = -most * scale
            assert torch.equal(x[b, 0, t], want)
        # no row is kept: the largest scale, under which the row's other entries are zero
        want = torch.zeros(16)
        want[5] = -most * 2.0 ** 119
        assert torch.equal(x[1, 0, 16], want)


@pytest.mark.parametrize("format", ["e4m3", "int8"])
def test_the_same_call_again(format):
    """Rows written twice over leave the same bytes: a repeated launch changes nothing."""
    gen = torch.Generator().manual_seed(3)
    rows = torch.randn(1, 1, 40, 64, generator=gen).cuda()
    cache = pkg.cache8(1, 1, 64, 64, format=format, block=32)
    pkg.cache8_write(cache, rows[:, :, :20], rows[:, :, :20])
    x = rows[:, :, 20:].clone() * 5
    x[0, 0, 3, 9] = INF
    seen = []
    for _ in range(3):
        pkg.cache8_write(cache, x, x, at=20)
        seen.append([t.view(torch.uint8).clone() for t in cache[:4]])
    for later in seen[1:]:
        assert all(torch.equal(a, b) for a, b in zip(later, seen[0]))
