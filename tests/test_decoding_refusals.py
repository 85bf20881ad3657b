"""CPU-only checks of the norms with rotary positions, of the 8-bit cache and of the attention over it: structures, what the entry
points refuse and with which status, and the definitions that the GPU tests compare with.  No kernel is launched here."""
import ctypes
import math

import pytest
import torch

import paper_2602_12271_amd as pkg
from paper_2602_12271_amd import binding as B
from decoding import LARGEST, HostCache, angles, code_values, norm_backward, norm_forward, quantised, scale_byte

SHAPE, UNSUPPORTED, NULL, WORKSPACE = B.MRT_ERR_SHAPE, B.MRT_ERR_UNSUPPORTED, B.MRT_ERR_NULL, B.MRT_ERR_WORKSPACE
S = B.MrtStrides
A = [0x10000 * (i + 1) for i in range(12)]       # addresses that no launch sees: every call is refused before


def test_structures_match_the_header():
    assert B.MrtNormTensor.weight.offset == 104 and B.MrtNormTensor.weight_head.offset == 120
    assert B.MrtNormTensor.dweight.offset == 152 and ctypes.sizeof(B.MrtNormTensor) == 160
    assert B.MrtCache8.k.offset == 24 and B.MrtCache8.k_codes.offset == 104 and ctypes.sizeof(B.MrtCache8) == 136
    assert B.MrtCache8Rows.k.offset == 24 and B.MrtCache8Rows.dtype.offset == 72 and ctypes.sizeof(B.MrtCache8Rows) == 80


# ---- norms -------------------------------------------------------------------------------------------
def rotary(dim=128, pairs=(22, 21, 21), layout=0, ladder=0, theta=1e4):
    return B.MrtRotary(dim, (ctypes.c_int * 3)(*pairs), layout, ladder, theta)


def norm(heads=4, dim=128, xd=1, yd=1, weight=A[8], wd=0, apart=0, dweight=None, dx=None, **kw):
    st = S(heads * 30 * dim, 30 * dim, dim)
    t = dict(batch=2, heads=heads, f=2, h=3, w=5, frame_offset=0, x=st, y=st, positions=None)
    t.update(kw)
    t = B.MrtRotaryTensor(t["batch"], t["heads"], t["f"], t["h"], t["w"], t["frame_offset"], t["x"], t["y"], xd, yd, t["positions"], 0, 0)
    return B.MrtNormTensor(t, weight, wd, apart, dx or st, dweight)


def norm_check(r, x, eps=1e-6, backward=0, n=None):
    return pkg.load_library().mrt_norm_rotary_check(ctypes.byref(r) if r else None, eps, (B.MrtNormTensor * len(x))(*x), len(x) if n is None else n, backward)


NORMS = {
    "good": (dict(), dict(), dict(), 0),
    "no-weight": (dict(), dict(weight=None), dict(), 0),
    "each": (dict(), dict(apart=128), dict(), 0),
    "pairs-none": (dict(pairs=(0, 0, 0)), dict(), dict(), SHAPE),
    "pairs-too-many": (dict(dim=64), dict(dim=64), dict(), SHAPE),
    "dim-257": (dict(dim=257), dict(dim=257), dict(), SHAPE),
    "eps-zero": (dict(), dict(), dict(eps=0.0), SHAPE),
    "eps-negative": (dict(), dict(), dict(eps=-1e-6), SHAPE),
    "eps-nan": (dict(), dict(), dict(eps=math.nan), SHAPE),
    "eps-inf": (dict(), dict(), dict(eps=math.inf), SHAPE),
    "eps-tiny": (dict(), dict(), dict(eps=1e-31), SHAPE),
    "heads-65536": (dict(), dict(heads=65536), dict(), SHAPE),
    "heads-0": (dict(), dict(heads=0), dict(), SHAPE),
    "weight-type": (dict(), dict(wd=2), dict(), SHAPE),
    "weight-apart-100": (dict(), dict(apart=100), dict(), SHAPE),
    "weight-apart-negative": (dict(), dict(apart=-128), dict(), SHAPE),
    "token-stride": (dict(), dict(x=S(1 << 20, 1 << 14, 127)), dict(), SHAPE),
    "dx-token-stride": (dict(), dict(dx=S(1 << 20, 1 << 14, 127)), dict(backward=1), SHAPE),
    "dx-not-looked-at": (dict(), dict(dx=S(0, 0, 0)), dict(), 0),
    "dx-expanded": (dict(), dict(dx=S(0, 0, 0)), dict(backward=1), SHAPE),
    "gradient-of-no-weight": (dict(), dict(weight=None, dweight=A[9]), dict(backward=1), SHAPE),
    "three-tensors": (dict(), dict(), dict(n=3), SHAPE),
    "no-tensors": (dict(), dict(), dict(n=0), SHAPE),
}


@pytest.mark.parametrize("name", NORMS)
def test_norm_descriptions(name):
    r, x, kw, status = NORMS[name]
    for others in ([], [norm()]):
        if others and (x.get("dim") or "n" in kw):
            continue
        st = norm_check(rotary(**r), [*others, norm(**x)], **kw)
        assert st == status, B.last_error()
        assert st == 0 or B.last_error()


def norm_run(x, X, out, dY=None, ws=A[11], nbytes=1 << 30):
    lib, r = pkg.load_library(), rotary()
    t, p = (B.MrtNormTensor * len(x))(*x), ctypes.c_void_p * len(x)
    if dY is None:
        return lib.mrt_norm_rotary_fwd(ctypes.byref(r), 1e-6, t, len(x), p(*X), p(*out), None)
    return lib.mrt_norm_rotary_bwd(ctypes.byref(r), 1e-6, t, len(x), p(*X), p(*dY), p(*out), ws, nbytes, None)


def test_norm_call_refusals():
    two = [norm(dweight=A[6]), norm(weight=A[9], dweight=A[7])]
    good = dict(X=A[:2], dY=A[2:4], out=A[4:6])
    for part in good:
        for i in (0, 1):
            for address, status in ((None, NULL), (A[10] + 1, SHAPE)):
                at = {n: list(v) for n, v in good.items()}
                at[part][i] = address
                assert norm_run(two, **at) == status, (part, i)
                if part != "dY":
                    at.pop("dY")
                    assert norm_run(two, **at) == status, (part, i)
    # a gradient in the place of another tensor; a result in that of the other input
    for i in (0, 1):
        for other in (*A[:4], A[5 - i], A[6], A[7], A[8], A[9]):
            out = list(A[4:6])
            out[i] = other
            assert norm_run(two, A[:2], out, A[2:4]) == SHAPE, (i, other)
        for other in (A[1 - i], A[5 - i], A[8], A[9]):
            out = list(A[4:6])
            out[i] = other
            assert norm_run(two, A[:2], out) == SHAPE, (i, other)
    for other in (*A[:4], A[7], A[8], A[9]):
        assert norm_run([norm(dweight=other), two[1]], A[:2], A[4:6], A[2:4]) == SHAPE, other
    # in place with other types or strides
    assert norm_run([norm(yd=0)], A[:1], A[:1]) == SHAPE
    assert norm_run([norm(y=S(1 << 20, 1 << 14, 136))], A[:1], A[:1]) == SHAPE
    lib = pkg.load_library()
    r, t = rotary(), (B.MrtNormTensor * 2)(*two)
    need = lib.mrt_norm_rotary_bwd_workspace_bytes(ctypes.byref(r), t, 2)
    assert 0 < need <= 4 << 20
    for ws, nbytes in ((None, need), (A[11] + 128, need), (A[11], need - 1)):
        assert norm_run(two, A[:2], A[4:6], A[2:4], ws, nbytes) == WORKSPACE
    assert lib.mrt_norm_rotary_bwd_workspace_bytes(ctypes.byref(r), (B.MrtNormTensor * 1)(norm()), 1) == 0
    assert lib.mrt_norm_rotary_bwd_workspace_bytes(None, t, 2) == 0
    assert lib.mrt_norm_rotary_bwd(ctypes.byref(r), 1e-6, t, 2, (ctypes.c_void_p * 2)(*A[:2]), None, (ctypes.c_void_p * 2)(*A[4:6]), A[11], need, None) == NULL


def test_norm_binding_refusals():
    q, w = torch.zeros(1, 2, 6, 64), torch.ones(64)
    for call in (lambda: pkg.norm_rotary_fwd(q, f_q=1, h=2, w=3), lambda: pkg.norm_rotary_bwd(q, None, w, None, q, f_q=1, h=2, w=3)):
        with pytest.raises(pkg.MrtError, match="GPU"):
            call()
    with pytest.raises(pkg.MrtError, match="k_weight"):
        pkg.norm_rotary_fwd(q, None, w, w, f_q=1, h=2, w=3)
    with pytest.raises(pkg.MrtError, match="together"):
        pkg.norm_rotary_bwd(q, q, w, w, q, f_q=1, h=2, w=3)
    for shape in ((63,), (3, 64), (64, 1), (2, 2, 64)):
        with pytest.raises(pkg.MrtError, match="weight"):
            B._norm_problem([q], [q], (), (torch.ones(shape), None), 1, None, 2, 3, 0, 0, 1e4, None, "adjacent", "axis", (None, None))
    with pytest.raises(pkg.MrtError, match="type"):
        B._norm_problem([q], [q], [q.bfloat16()], (w, None), 1, None, 2, 3, 0, 0, 1e4, None, "adjacent", "axis", (None, None))
    a = B._norm_problem([q], [q], (), (torch.ones(2, 64), None), 1, None, 2, 3, 0, 0, 1e4, None, "adjacent", "axis", (None, None))
    b = B._norm_problem([q], [q], (), (w, None), 1, None, 2, 3, 0, 0, 1e4, None, "adjacent", "axis", (None, None))
    assert a[1][0].weight_head == 64 and b[1][0].weight_head == 0


# ---- the cache ---------------------------------------------------------------------------------------
def cache(batch=2, heads=3, dim=128, capacity=200, block=64, format=0, **kw):
    st = S(heads * capacity * dim, capacity * dim, dim)
    blocks = -(-capacity // max(block, 1))
    c = dict(k=st, v=st, ksb=heads * blocks, ksh=blocks, vsb=heads * blocks, vsh=blocks, at=A[:4])
    c.update(kw)
    return B.MrtCache8(batch, heads, dim, capacity, block, format, c["k"], c["v"], c["ksb"], c["ksh"], c["vsb"], c["vsh"], *c["at"])


def rows(tokens=20, at=0, dtype=1, dim=128, heads=3, at_each=None, tokens_each=None, **kw):
    st = S(heads * tokens * dim, tokens * dim, dim) if tokens > 0 else S(dim, dim, dim)
    c = dict(k=st, v=st)
    c.update(kw)
    return B.MrtCache8Rows(tokens, at, at_each, tokens_each, c["k"], c["v"], dtype)


CACHES = {
    "good": (dict(), dict(), 0),
    "int8": (dict(format=1, block=16), dict(), 0),
    "last-row": (dict(), dict(at=180), 0),
    "device-places": (dict(), dict(at=-7, at_each=A[5]), 0),
    "f32": (dict(), dict(dtype=0, k=S(1 << 20, 1 << 14, 132)), 0),
    "beyond": (dict(), dict(at=181), SHAPE),
    "before": (dict(), dict(at=-1), SHAPE),
    "far": (dict(), dict(at=0x7fffffff), SHAPE),
    "no-rows": (dict(), dict(tokens=0), SHAPE),
    "rows-negative": (dict(), dict(tokens=-1), SHAPE),
    "rows-type": (dict(), dict(dtype=2), SHAPE),
    "rows-stride-not-8": (dict(), dict(v=S(1 << 20, 1 << 14, 132)), SHAPE),
    "rows-token-stride": (dict(), dict(k=S(1 << 20, 1 << 14, 120)), SHAPE),
    "rows-expanded": (dict(), dict(k=S(1 << 20, 0, 128)), SHAPE),
    "block-48": (dict(block=48), dict(), SHAPE),
    "block-0": (dict(block=0), dict(), SHAPE),
    "block-256": (dict(block=256), dict(), SHAPE),
    "format": (dict(format=2), dict(), SHAPE),
    "dim-72": (dict(dim=72), dict(dim=72), SHAPE),
    "dim-272": (dict(dim=272), dict(dim=272), SHAPE),
    "dim-0": (dict(dim=0), dict(), SHAPE),
    "heads-0": (dict(heads=0), dict(), SHAPE),
    "heads-65536": (dict(heads=65536, batch=1), dict(), SHAPE),
    "capacity-0": (dict(capacity=0), dict(), SHAPE),
    "capacity-2^24+1": (dict(capacity=(1 << 24) + 1), dict(), SHAPE),
    "codes-token-stride": (dict(k=S(1 << 20, 1 << 16, 112)), dict(), SHAPE),
    "codes-stride-not-16": (dict(v=S(1 << 20, 1 << 16, 136)), dict(), SHAPE),
    "codes-head-stride-0": (dict(v=S(1 << 20, 0, 128)), dict(), SHAPE),
    "scales-stride-0": (dict(ksh=0), dict(), SHAPE),
    "codes-NULL": (dict(at=(None, A[1], A[2], A[3])), dict(), NULL),
    "scales-NULL": (dict(at=(A[0], A[1], None, A[3])), dict(), NULL),
    "codes-unaligned": (dict(at=(A[0], A[1] + 8, A[2], A[3])), dict(), SHAPE),
    "keys-are-values": (dict(at=(A[0], A[0], A[2], A[3])), dict(), SHAPE),
    "scales-are-scales": (dict(at=(A[0], A[1], A[2], A[2])), dict(), SHAPE),
}


@pytest.mark.parametrize("name", CACHES)
def test_cache_descriptions(name):
    c, r, status = CACHES[name]
    lib, c, r = pkg.load_library(), cache(**c), rows(**r)
    assert lib.mrt_cache8_check(ctypes.byref(c), ctypes.byref(r)) == status, B.last_error()
    if status:
        assert B.last_error()
        assert lib.mrt_cache8_write(ctypes.byref(c), ctypes.byref(r), A[6], A[7], None) == status
        assert lib.mrt_cache8_read(ctypes.byref(c), ctypes.byref(r), A[6], A[7], None) == status


def test_cache_call_refusals():
    lib, c, r = pkg.load_library(), cache(), rows()
    for f in (lib.mrt_cache8_write, lib.mrt_cache8_read):
        assert f(None, ctypes.byref(r), A[6], A[7], None) == NULL
        assert f(ctypes.byref(c), None, A[6], A[7], None) == NULL
        for at, status in (((None, A[7]), NULL), ((A[6], None), NULL), ((A[6] + 8, A[7]), SHAPE), ((A[6], A[7] + 2), SHAPE),
                           ((A[0], A[7]), SHAPE), ((A[6], A[3]), SHAPE)):
            assert f(ctypes.byref(c), ctypes.byref(r), *at, None) == status, at
    assert lib.mrt_cache8_read(ctypes.byref(c), ctypes.byref(r), A[6], A[6], None) == SHAPE
    r = rows(tokens_each=A[5])
    assert lib.mrt_cache8_read(ctypes.byref(c), ctypes.byref(r), A[6], A[7], None) == SHAPE
    assert lib.mrt_cache8_check(None, None) == NULL


def problem(**kw):
    base = dict(batch=2, heads=6, head_dim=128, f_q=1, f_kv=4, h=5, w=10, scale=0.1)
    base.update(kw)
    return pkg.make_problem(**base)


ATTENTION = {
    "good": (dict(), dict(), 0, 0),
    "masked": (dict(q_frame_offset=3), dict(), 1, 0),
    "one-head": (dict(heads=3), dict(), 0, 0),
    "heads-4-of-3": (dict(heads=4), dict(), 0, SHAPE),
    "batch": (dict(batch=1), dict(), 0, SHAPE),
    "dim": (dict(head_dim=64), dict(), 0, SHAPE),
    "dim-96": (dict(head_dim=96), dict(dim=96), 0, SHAPE),
    "dim-64": (dict(head_dim=64), dict(dim=64), 0, 0),
    "more-keys": (dict(f_kv=5), dict(), 0, SHAPE),
    "f32": (dict(dtype=B.MRT_F32), dict(), 0, UNSUPPORTED),
    "f32-arithmetic": (dict(compute=1), dict(), 0, UNSUPPORTED),
    "scale": (dict(scale=1e-31), dict(), 0, UNSUPPORTED),
    "chunk-negative": (dict(), dict(), -1, SHAPE),
    "far-frames": (dict(q_frame_offset=0x7fffffff), dict(), 1, SHAPE),
    "cache-block": (dict(), dict(block=10), 0, SHAPE),
    "cache-NULL": (dict(), dict(at=(A[0], None, A[2], A[3])), 0, NULL),
    "far-codes": (dict(), dict(k=S(1 << 40, 1 << 36, 1 << 24)), 0, UNSUPPORTED),
}


@pytest.mark.parametrize("name", ATTENTION)
def test_attention_descriptions(name):
    p, c, chunk, status = ATTENTION[name]
    lib, p, c = pkg.load_library(), problem(**p), cache(**c)
    assert lib.dense_attn_cache8_check(ctypes.byref(p), ctypes.byref(c), chunk) == status, B.last_error()
    if status:
        assert lib.dense_attn_fwd_cache8_workspace_bytes(ctypes.byref(p), ctypes.byref(c), chunk) == 0
        assert lib.dense_attn_fwd_cache8(A[4], ctypes.byref(c), A[5], A[6], ctypes.byref(p), None, chunk, None, 0, None) == status


def test_attention_call_refusals():
    lib, p, c = pkg.load_library(), problem(), cache()

    def run(q=A[4], o=A[5], lse=A[6], ws=A[7], cache=c, prob=p):
        return lib.dense_attn_fwd_cache8(q, ctypes.byref(cache) if cache else None, o, lse, ctypes.byref(prob) if prob else None, None, 0, ws, 1 << 30, None)
    for kw in (dict(q=None), dict(o=None), dict(lse=None), dict(cache=None), dict(prob=None)):
        assert run(**kw) == NULL, kw
    for kw in (dict(q=A[4] + 8), dict(o=A[5] + 8), dict(o=A[0]), dict(o=A[1]), dict(lse=A[2]), dict(lse=A[5]), dict(lse=A[4])):
        assert run(**kw) == SHAPE, kw
    assert run(ws=A[7] + 128) == WORKSPACE


def test_cache_binding_refusals():
    c = pkg.cache8(2, 3, 40, 32, device="cpu")
    k = torch.zeros(2, 3, 5, 32)
    with pytest.raises(pkg.MrtError, match="GPU"):
        pkg.cache8_write(c, k, k)
    with pytest.raises(pkg.MrtError, match="GPU"):
        pkg.cache8_read(c, 5)
    with pytest.raises(pkg.MrtError, match="GPU"):
        pkg.dense_attn_fwd_cache8(k, c, f_q=1, f_kv=1, h=1, w=5)
    assert B._cache8_of(c).capacity == 40 and B._cache8_of(c).format == 0 and B._cache8_of(c).k_codes == c.K.data_ptr()
    for bad in (c._replace(K=c.K.view(torch.uint8)), c._replace(V=c.V[:, :, :39]), c._replace(K_scale=c.K_scale.int()),
                c._replace(V_scale=c.V_scale[:, :1]), c._replace(block=32), c._replace(block=64.0), c._replace(K=c.K[0]),
                c._replace(V=torch.zeros(2, 3, 40, 32, dtype=torch.int8)), c._replace(K=c.K.transpose(2, 3), V=c.V.transpose(2, 3))):
        with pytest.raises(pkg.MrtError):
            B._cache8_of(bad)
    for bad in (dict(K=k[:, :2]), dict(V=k.bfloat16()), dict(K=k[..., :16], V=k[..., :16]), dict(at=torch.zeros(2)), dict(at=1.0), dict(at=-1), dict(at=1 << 32), dict(at=None),
                dict(at=torch.zeros(3, dtype=torch.int32)), dict(lengths=torch.zeros(2, dtype=torch.int64)), dict(lengths=5),
                dict(K=k.half(), V=k.half())):
        args = dict(K=k, V=k, at=0, lengths=None)
        args.update(bad)
        for _ in range(2):       # (refused again where a description is kept)
            with pytest.raises(pkg.MrtError):
                B._require_places(args["at"], args["lengths"])
                B._cache8_rows(c, **args)
            B._cache8_rows(c, k, k, 0, None)
    for bad in (dict(format="e5m2"), dict(block=48)):
        with pytest.raises(pkg.MrtError):
            pkg.cache8(1, 1, 8, 32, device="cpu", **bad)


# ---- the definitions ---------------------------------------------------------------------------------
@pytest.mark.parametrize("layout", ["adjacent", "halves"])
def test_norm_gradients_against_differences(layout):
    gen = torch.Generator().manual_seed(0)
    x, dy = (torch.randn(2, 3, 5, 14, generator=gen, dtype=torch.float64) for _ in range(2))
    w, split = torch.randn(3, 14, generator=gen, dtype=torch.float64), (2, 3, 1)
    angle = angles(torch.randint(0, 50, (2, 3, 5), generator=gen), split, 100.0, "axis")
    dx, dw = norm_backward(x, w, 0.1, angle, split, layout, dy)
    h = 1e-5
    for i in (0, 17, 101, 400):
        d = torch.zeros_like(x).view(-1)
        d[i] = h
        d = d.view_as(x)
        slope = ((norm_forward(x + d, w, 0.1, angle, split, layout) - norm_forward(x - d, w, 0.1, angle, split, layout)) * dy).sum() / (2 * h)
        assert abs(slope - dx.view(-1)[i]) < 1e-8
    d = torch.zeros_like(w)
    d[1, 4] = h
    slope = ((norm_forward(x, w + d, 0.1, angle, split, layout) - norm_forward(x, w - d, 0.1, angle, split, layout)) * dy).sum() / (2 * h)
    assert abs(slope - dw[1, 4]) < 1e-8


@pytest.mark.parametrize("format", ["e4m3", "int8"])
def test_host_cache(format):
    table = code_values(format)
    table = table[torch.isfinite(table) & (table.abs() <= LARGEST[format])].sort().values.unique()
    x = torch.randn(4000, generator=torch.Generator().manual_seed(1), dtype=torch.float64) * 100
    byte = scale_byte(x, format)
    top = float(x.abs().max())
    assert top <= LARGEST[format] * 2.0 ** (byte - 127) < 2 * top * (1 + 1e-12)
    z = x / 2.0 ** (byte - 127)
    best = (z[:, None] - table).abs().min(1).values
    assert torch.equal((quantised(x, format, byte) - z).abs(), best)          # the nearest code
    if format == "e4m3":       # torch's conversion is to the nearest, ties to even, too
        assert torch.equal(z.float().to(torch.float8_e4m3fn).double(), quantised(z.float().double(), format, 127))
    # a block that is appended to keeps what it holds, up to the header's bound
    cache = HostCache(64, 4, 32, format)
    for t in range(64):
        cache.write(torch.full((1, 4), 1.3 ** (t % 32)), t)
    got = cache.values(torch.arange(64))[:, 0]
    want = 1.3 ** (torch.arange(64, dtype=torch.float64) % 32)
    scale = 2.0 ** (cache.bytes[torch.arange(64) // 32] - 127).double()
    bound = scale if format == "int8" else (want * 2.0 ** -4).clamp(min=2.0 ** -9) * torch.ones_like(scale)
    assert ((got - want).abs() <= bound).all()
