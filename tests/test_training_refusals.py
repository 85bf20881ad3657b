"""CPU-only checks of the training step's entry points and of rotary positions: structures, what they refuse and with
which status, scratch sizes.  No kernel is launched here."""
import ctypes

import pytest
import torch

import paper_2602_12271_amd as pkg
from paper_2602_12271_amd import binding as B
from test_problem_cache import Tensor

SHAPE, UNSUPPORTED, NULL, WORKSPACE = B.MRT_ERR_SHAPE, B.MRT_ERR_UNSUPPORTED, B.MRT_ERR_NULL, B.MRT_ERR_WORKSPACE


def test_structures_match_the_header():
    # int, pointer, 4 stride sets
    assert B.MrtDenseTrain.kv_len.offset == 8 and B.MrtDenseTrain.dout.offset == 16
    assert ctypes.sizeof(B.MrtDenseTrain) == 16 + 4 * 24
    # 4 ints, 2 enums, double
    assert B.MrtRotary.layout.offset == 16 and B.MrtRotary.theta.offset == 24 and ctypes.sizeof(B.MrtRotary) == 32
    # 6 ints, 2 stride sets, 2 enums, pointer, 2 long long
    assert B.MrtRotaryTensor.x.offset == 24 and B.MrtRotaryTensor.x_dtype.offset == 72
    assert B.MrtRotaryTensor.positions.offset == 80 and ctypes.sizeof(B.MrtRotaryTensor) == 104


def problem(**kw):
    base = dict(batch=2, heads=6, head_dim=128, f_q=2, f_kv=3, h=5, w=7, scale=0.1)
    base.update(kw)
    return pkg.make_problem(**base)


def train(prob, kv_heads=0, **kw):
    strides = dict(dout=prob.o, dq=prob.q, dk=prob.k, dv=prob.v)
    strides.update(kw)
    return B.MrtDenseTrain(kv_heads, None, strides["dout"], strides["dq"], strides["dk"], strides["dv"])


BF16, F32 = B.MRT_BF16, B.MRT_F32
S = B.MrtStrides
DESCRIPTIONS = {
    "good": (dict(), dict(), 0),
    "shared": (dict(), dict(kv_heads=2), 0),
    "f32-odd-dim": (dict(dtype=F32, head_dim=37), dict(), 0),
    "bf16-in-f32-odd-dim": (dict(head_dim=37, compute=1), dict(), 0),
    "kv-heads-4-of-6": (dict(), dict(kv_heads=4), SHAPE),
    "kv-heads-12-of-6": (dict(), dict(kv_heads=12), SHAPE),
    "kv-heads-negative": (dict(), dict(kv_heads=-1), SHAPE),
    "scale-zero": (dict(scale=0.0), dict(), None),
    "scale-negative": (dict(scale=-1.0), dict(), None),
    "scale-tiny": (dict(scale=1e-31), dict(), UNSUPPORTED),
    "scale-nan": (dict(scale=float("nan")), dict(), None),
    "scale-inf": (dict(scale=float("inf")), dict(), None),
    "no-keys": (dict(f_kv=0), dict(), SHAPE),
    "no-queries": (dict(f_q=0), dict(), SHAPE),
    "bf16-odd-dim": (dict(head_dim=96), dict(), None),
    "dq-token-stride": (dict(), dict(dq=S(1 << 20, 1 << 14, 127)), SHAPE),
    "dk-head-stride-0": (dict(), dict(dk=S(1 << 20, 0, 128)), SHAPE),
    "dv-batch-stride-negative": (dict(), dict(dv=S(-(1 << 20), 1 << 14, 128)), SHAPE),
    "dout-expanded": (dict(), dict(dout=S(0, 0, 0)), SHAPE),
    "dout-stride-not-8": (dict(), dict(dout=S(1 << 20, 1 << 14, 132)), SHAPE),
    "f32-stride-not-8": (dict(dtype=F32), dict(dout=S(1 << 20, 1 << 14, 133)), 0),
    "dq-token-stride-far": (dict(), dict(dq=S(1 << 50, 1 << 40, (1 << 25) + 8)), UNSUPPORTED),
    "f32-token-stride-far": (dict(dtype=F32), dict(dq=S(1 << 50, 1 << 40, (1 << 25) + 8)), 0),
}


@pytest.mark.parametrize("name", DESCRIPTIONS)
def test_backward_descriptions(name):
    kw, tr, status = DESCRIPTIONS[name]
    lib, p = pkg.load_library(), problem(**kw)
    t = train(p, **tr)
    st = lib.dense_attn_bwd_check(ctypes.byref(p), ctypes.byref(t), 0)
    assert st == status if status is not None else st != 0
    assert (B.dense_attn_bwd_workspace_bytes(p, t) > 0) == (st == 0)
    if st:
        assert B.last_error()


def test_backward_needs_a_description():
    lib, p = pkg.load_library(), problem()
    assert lib.dense_attn_bwd_check(ctypes.byref(p), None, 0) == NULL
    assert lib.dense_attn_bwd_check(None, None, 0) != 0
    assert lib.dense_attn_bwd_workspace_bytes(ctypes.byref(p), None, 0) == 0
    assert lib.dense_attn_fwd_save_workspace_bytes(None, None, 0) == 0


# addresses that no launch sees: every call below is refused before
A = [0x10000 * (i + 1) for i in range(10)]


def fwd(p, t, q=A[0], k=A[1], v=A[2], o=A[3], lse=A[4], ws=A[9], nbytes=1 << 40):
    return pkg.load_library().dense_attn_fwd_save(q, k, v, o, lse, ctypes.byref(p), None if t is None else ctypes.byref(t), 0, ws, nbytes, None)


def bwd(p, t, at=A[:9], ws=A[9], nbytes=1 << 40):
    q, k, v, o, do, lse, dq, dk, dv = at
    return pkg.load_library().dense_attn_bwd(q, k, v, o, do, lse, dq, dk, dv, ctypes.byref(p), ctypes.byref(t), 0, ws, nbytes, None)


def test_forward_call_refusals():
    p = problem()
    for name in ("q", "k", "v", "o", "lse"):
        assert fwd(p, None, **{name: None}) == NULL, name
    for name in ("q", "k", "v", "o"):
        assert fwd(p, None, **{name: A[5] + 8}) == SHAPE, name
    assert fwd(p, None, ws=A[9] + 128) == WORKSPACE
    assert fwd(p, None, o=A[1]) == SHAPE and fwd(p, None, o=A[2]) == SHAPE
    assert fwd(p, train(p, kv_heads=5)) == SHAPE
    assert fwd(problem(scale=1e-31), None) == UNSUPPORTED


def test_backward_call_refusals():
    p = problem()
    t = train(p)
    need = B.dense_attn_bwd_workspace_bytes(p, t)
    for i in range(9):
        at = list(A[:9])
        at[i] = None
        assert bwd(p, t, at) == NULL, i
        if i != 5:
            at[i] = A[i] + 8
            assert bwd(p, t, at) == SHAPE, i
    for i in (6, 7, 8):                          # a gradient in the place of another tensor
        for j in (0, 1, 2, 3, 4, 6, 7, 8):
            if i != j:
                at = list(A[:9])
                at[i] = at[j]
                assert bwd(p, t, at) == SHAPE, (i, j)
    assert bwd(p, t, ws=None) == WORKSPACE
    assert bwd(p, t, ws=A[9] + 128) == WORKSPACE
    assert bwd(p, t, nbytes=need - 1) == WORKSPACE
    assert str(need) in B.last_error()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scratch_stays_small(dtype):
    # the parts of dK and dV, or of dQ, together at most 2^27 elements, and 2 numbers a row in tiles of 32
    for f, h, w, heads, batch, kvh in ((1, 1, 1, 1, 1, 1), (1, 24, 24, 1, 1, 1), (3, 30, 52, 12, 1, 12), (21, 45, 80, 12, 1, 12),
                                       (1, 1, 1, 40, 4, 40), (1531, 1, 1, 16, 2, 2), (1, 3, 3, 2, 500, 1)):
        p = problem(f_q=f, f_kv=f, h=h, w=w, heads=heads, batch=batch, dtype=dtype)
        rows = batch * heads * ((f * h * w + 31) // 32) * 32
        for chunk in (0, 1):
            own = B.dense_attn_bwd_workspace_bytes(p, train(p, kvh), chunk)
            grads = 4 * 128 * f * h * w * batch * max(heads, 2 * kvh)
            assert 8 * rows <= own <= 8 * rows + max(4 << 27, grads) + 512
            more = B.dense_attn_fwd_save_workspace_bytes(p, train(p, kvh), chunk)
            assert 0 <= more <= (4 << 27) * 130 // 128 + 512


# ---- rotary positions ----------------------------------------------------------------------------
def rotary(head_dim=128, pairs=(22, 21, 21), layout=0, ladder=0, theta=1e4):
    return B.MrtRotary(head_dim, (ctypes.c_int * 3)(*pairs), layout, ladder, theta)


def tensor(batch=2, heads=3, f=2, h=3, w=5, frame_offset=0, x=None, y=None, x_dtype=BF16, y_dtype=BF16, positions=None,
           position_batch=0, position_axis=30, dim=128):
    s = S(heads * f * h * w * dim, f * h * w * dim, dim)
    return B.MrtRotaryTensor(batch, heads, f, h, w, frame_offset, x or s, y or s, x_dtype, y_dtype, positions, position_batch, position_axis)


ROTARY = {
    "good": (dict(), dict(), 0),
    "two-features": (dict(head_dim=2, pairs=(0, 1, 0)), dict(dim=2), 0),
    "odd-dim": (dict(head_dim=31, pairs=(4, 4, 4)), dict(dim=31), 0),
    "head-dim-0": (dict(head_dim=0, pairs=(0, 0, 0)), dict(), SHAPE),
    "head-dim-258": (dict(head_dim=258), dict(dim=258), SHAPE),
    "no-pairs": (dict(pairs=(0, 0, 0)), dict(), SHAPE),
    "too-many-pairs": (dict(pairs=(22, 22, 21)), dict(), SHAPE),
    "negative-pairs": (dict(pairs=(-1, 22, 21)), dict(), SHAPE),
    "pairs-that-wrap": (dict(pairs=((1 << 31) - 1, (1 << 31) - 1, 10)), dict(), SHAPE),
    "layout-2": (dict(layout=2), dict(), SHAPE),
    "ladder-2": (dict(ladder=2), dict(), SHAPE),
    "theta-0": (dict(theta=0.0), dict(), SHAPE),
    "theta-nan": (dict(theta=float("nan")), dict(), SHAPE),
    "theta-inf": (dict(theta=float("inf")), dict(), SHAPE),
    "batch-0": (dict(), dict(batch=0), SHAPE),
    "heads-0": (dict(), dict(heads=0), SHAPE),
    "heads-that-wrap": (dict(), dict(batch=1 << 16, heads=1 << 16), SHAPE),
    "no-frames": (dict(), dict(f=0), SHAPE),
    "tokens-that-wrap": (dict(), dict(f=1 << 16, h=1 << 16, w=1), SHAPE),
    "offset-negative": (dict(), dict(frame_offset=-1), SHAPE),
    "offset-that-wraps": (dict(), dict(frame_offset=(1 << 31) - 2), SHAPE),
    "x-dtype": (dict(), dict(x_dtype=7), SHAPE),
    "y-dtype": (dict(), dict(y_dtype=7), SHAPE),
    "x-token-stride": (dict(), dict(x=S(1 << 20, 1 << 14, 120)), SHAPE),
    "y-token-stride": (dict(), dict(y=S(1 << 20, 1 << 14, 0)), SHAPE),
    "y-head-stride": (dict(), dict(y=S(1 << 20, 0, 128)), SHAPE),
    "x-batch-stride": (dict(), dict(x=S(0, 1 << 14, 128)), SHAPE),
    "position-axis-negative": (dict(), dict(positions=A[0], position_axis=-30), SHAPE),
    "position-axis-0": (dict(), dict(positions=A[0], position_axis=0), 0),
}


@pytest.mark.parametrize("name", ROTARY)
def test_rotary_descriptions(name):
    kw, tk, status = ROTARY[name]
    lib = pkg.load_library()
    r, good, bad = rotary(**kw), tensor(), tensor(**tk)
    assert lib.mrt_rotary_check(ctypes.byref(r), (B.MrtRotaryTensor * 1)(bad), 1) == status
    if not kw:                                   # also as the second tensor
        assert lib.mrt_rotary_check(ctypes.byref(r), (B.MrtRotaryTensor * 2)(good, bad), 2) == status
    if status:
        assert B.last_error()


@pytest.mark.parametrize("entry", ["mrt_rotary_fwd", "mrt_rotary_bwd"])
def test_rotary_call_refusals(entry):
    lib, r = pkg.load_library(), rotary()

    def call(tensors, x, y, n=None):
        n = len(tensors) if n is None else n
        return getattr(lib, entry)(ctypes.byref(r), (B.MrtRotaryTensor * len(tensors))(*tensors), n,
                                   (ctypes.c_void_p * len(x))(*x), (ctypes.c_void_p * len(y))(*y), None)
    one, f32 = tensor(), tensor(y_dtype=F32)
    other = tensor(y=S(1 << 20, 1 << 14, 128))
    assert call([one], A[:1], A[1:2], 0) == SHAPE and call([one], A[:1], A[1:2], 3) == SHAPE
    assert call([one], [None], A[1:2]) == NULL and call([one], A[:1], [None]) == NULL
    assert call([one, one], A[:2], [A[2], None]) == NULL
    assert call([one], [A[0] + 1], A[1:2]) == SHAPE
    assert call([f32], A[:1], [A[1] + 2]) == SHAPE
    assert call([f32], A[:1], A[:1]) == SHAPE                   # in place with another type
    assert call([other], A[:1], A[:1]) == SHAPE                 # ... and with other strides
    assert call([one, one], A[:2], [A[2], A[2]]) == SHAPE       # one output twice
    assert call([one, one], A[:2], [A[1], A[2]]) == SHAPE       # an output in the other tensor
    assert call([one, one], A[:2], [A[2], A[0]]) == SHAPE
    assert call([one, one], [A[0], A[0]], [A[0], A[0]]) == SHAPE
    assert getattr(lib, entry)(None, (B.MrtRotaryTensor * 1)(one), 1, None, None, None) == NULL
    assert getattr(lib, entry)(ctypes.byref(r), (B.MrtRotaryTensor * 1)(one), 1, None, None, None) == NULL


# ---- the binding ---------------------------------------------------------------------------------
def step_problem(q=(2, 6, 30, 64), k=(2, 2, 60, 64), f_q=1, f_kv=2, h=5, w=6, grads=True, dtype=torch.bfloat16, o=None, **kw):
    Q, K, V = Tensor(q, dtype), Tensor(k, dtype), kw.pop("V", Tensor(k, dtype))
    O = o or Tensor(q, dtype)
    g = (kw.pop("dO", Tensor(q, dtype)), Tensor(q, dtype), kw.pop("dK", Tensor(k, dtype)), Tensor(k, dtype)) if grads else ()
    return B._train_problem(Q, K, V, O, g, f_q, f_kv, h, w, kw.get("chunk", 0), 0, kw.get("scale", 0.1), 0)


STEPS = {
    "three-dims": dict(q=(6, 30, 64)),
    "query-tokens": dict(f_q=2),
    "key-tokens": dict(f_kv=1),
    "key-batch": dict(k=(1, 2, 60, 64)),
    "key-dim": dict(k=(2, 2, 60, 128)),
    "value-shape": dict(V=Tensor((2, 2, 59, 64))),
    "value-type": dict(V=Tensor((2, 2, 60, 64), torch.float32)),
    "output-shape": dict(o=Tensor((2, 6, 31, 64))),
    "output-type": dict(o=Tensor((2, 6, 30, 64), torch.float32)),
    "gradient-shape": dict(dK=Tensor((2, 6, 60, 64))),
    "gradient-type": dict(dO=Tensor((2, 6, 30, 64), torch.float32)),
    "gradient-last-stride": dict(dO=Tensor((2, 6, 30, 64), strides=(23040, 3840, 128, 2))),
    "gradient-expanded": dict(dO=Tensor((2, 6, 30, 64), strides=(0, 0, 0, 1))),
    "half": dict(dtype=torch.float16),
    "kv-heads": dict(k=(2, 4, 60, 64)),
    "scale": dict(scale=0.0),
    "bf16-dim": dict(q=(2, 6, 30, 96), k=(2, 2, 60, 96)),
}


@pytest.mark.parametrize("name", STEPS)
def test_binding_refuses_training_steps(name):
    for _ in range(2):
        step_problem()                           # a cached description lets nothing else through
        with pytest.raises(pkg.MrtError) as e:
            step_problem(**STEPS[name])
        assert str(e.value)


def test_training_descriptions_are_by_value():
    B._train_problems.clear()
    a, b = step_problem(), step_problem()
    assert a is b
    assert bytes(step_problem(grads=False)[0]) == bytes(a[0])
    assert step_problem(scale=0.2)[0].scale != a[0].scale
    assert step_problem(k=(2, 6, 60, 64))[1].kv_heads == 6 and a[1].kv_heads == 2
    for n in range(2 * B._MAX_PROBLEMS):
        step_problem(scale=0.5 + n)
    assert len(B._train_problems) <= B._MAX_PROBLEMS


def test_binding_wants_device_tensors():
    x = torch.zeros(1, 2, 30, 64, dtype=torch.bfloat16)
    grid = dict(f_q=1, f_kv=1, h=5, w=6)
    lse = torch.zeros(1, 2, 30)
    for call in (lambda: pkg.dense_attn_fwd_save(x, x, x, **grid), lambda: pkg.dense_attn_bwd(x, x, x, x, x, lse, **grid),
                 lambda: pkg.rotary_fwd(x, x, **grid), lambda: pkg.rotary_bwd(x, **grid)):
        with pytest.raises(pkg.MrtError, match="GPU"):
            call()


def test_row_statistics_and_lengths():
    Q = Tensor((2, 6, 30, 64))
    B._require_lse(torch.zeros(2, 6, 30), Q)
    for bad in (torch.zeros(2, 6, 31), torch.zeros(2, 6, 30, dtype=torch.float64), torch.zeros(2, 30, 6).transpose(1, 2)):
        with pytest.raises(pkg.MrtError, match="lse"):
            B._require_lse(bad, Q)
    t = step_problem()[1]
    n = torch.zeros(2, dtype=torch.int32)
    assert B._with_lengths(t, None, 2) is t
    own = B._with_lengths(t, n, 2)
    assert own.kv_len == n.data_ptr() and own.kv_heads == t.kv_heads and t.kv_len is None
    for bad in (torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int64), torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises(pkg.MrtError, match="kv_len"):
            B._with_lengths(t, bad, 2)


ROTARY_TENSORS = {
    "no-grid": dict(f=None),
    "tokens": dict(f=3),
    "three-dims": dict(x=Tensor((6, 30, 64))),
    "last-stride": dict(x=Tensor((2, 6, 30, 64), strides=(23040, 3840, 128, 2))),
    "output-shape": dict(y=Tensor((2, 6, 31, 64))),
    "half": dict(x=Tensor((2, 6, 30, 64), torch.float16)),
    "output-half": dict(y=Tensor((2, 6, 30, 64), torch.float16)),
    "positions-type": dict(positions=Tensor((3, 30), torch.int64)),
    "positions-two-axes": dict(positions=Tensor((2, 30), torch.int32)),
    "positions-tokens": dict(positions=Tensor((3, 31), torch.int32)),
    "positions-batch": dict(positions=Tensor((3, 3, 30), torch.int32)),
    "positions-stride": dict(positions=Tensor((3, 30), torch.int32, strides=(1, 3))),
}


@pytest.mark.parametrize("name", ROTARY_TENSORS)
def test_binding_refuses_rotary_tensors(name):
    args = dict(x=Tensor((2, 6, 30, 64)), y=Tensor((2, 6, 30, 64)), f=1, h=5, w=6, offset=0, positions=None, name="Q")
    B._rotary_tensor(**args)
    with pytest.raises(pkg.MrtError):
        B._rotary_tensor(**{**args, **ROTARY_TENSORS[name]})


def test_rotary_split():
    for dim in range(2, 257):
        split = pkg.binding.rotary_pairs_split(dim)
        assert sum(split) == dim // 2 and min(split) >= 0 and split[0] - split[2] in (0, 1, 2)


def test_rotary_arguments_that_contradict():
    x = torch.zeros(1, 2, 30, 64)
    at = torch.zeros(3, 30, dtype=torch.int32)
    for kw in (dict(k_out=x), dict(k_positions=at), dict(dtype=torch.bfloat16, out=x), dict(K=x, dtype=torch.bfloat16, k_out=x)):
        with pytest.raises(pkg.MrtError, match="k_out|dtype"):
            pkg.rotary_fwd(x, f_q=1, h=5, w=6, **kw)
