"""The training step's promise in the 2-norm, head by head, on the GPU; and on the host, that the check finds what an entry's
bound does not: keys that are missing from long rows."""
import dataclasses

import pytest
import torch

from dense_training import Step, reference, run, tensors
from test_gpu_dense_training import CASES, FEW
from test_gpu_training_calls import CALLS, FEW_KEYS, FULL, NOWHERE, SHARED, SHARP
from training_norms import check_norms

ALL = {f"{group}-{name}": c for group, cases in (("case", CASES), ("few", FEW), ("shared", SHARED), ("full", FULL), ("few-keys", FEW_KEYS),
                                                 ("call", CALLS), ("padded", NOWHERE)) for name, c in cases.items()}
# logits of hundreds: dS is what is left of a difference that cancels, and each entry has its bound only
ALL = {name: c for name, c in ALL.items() if c.sigma < 6}


@pytest.mark.gpu
@pytest.mark.parametrize("name", ALL)
def test_norms(name):
    c = ALL[name]
    q, k, v, do, kv_len = tensors(c, seed=41)
    ref, _ = reference(c, q, k, v, do)
    got = run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    print(f"  {name}: {check_norms(c, got, ref)}", flush=True)


@pytest.mark.gpu
@pytest.mark.parametrize("name", [n for n in SHARP if n.startswith("bf16")])
def test_norms_of_sharp_rows(name):
    """dS cancels where a row's weight lies on one key; the rounding of O, by 2^-8 of sum |dO| |O| in delta, does not.  In the
    norm it is drawn: 2^-9 sqrt(4/3) of what the entries' bound has for it, beside the promise for the rest."""
    c = SHARP[name]
    q, k, v, do, kv_len = tensors(c, seed=41)
    ref, (_, cost_o) = reference(c, q, k, v, do)
    got = run(c, q, k, v, do, kv_len)
    torch.cuda.synchronize()
    for n in ("dQ", "dK"):
        off, most = (got[n].double() - ref[n]).norm(), 1e-2 * ref[n].norm() + 2.0 ** -9 * (4 / 3) ** 0.5 * cost_o[n].norm()
        print(f"  {name} {n}: {float(off / ref[n].norm()):.1e} of the norm, {float(off / most):.2f} of the bound", flush=True)
        assert off <= most, n


# exact steps and the number of keys that the planted one has
LOST = {"bf16-11-of-20011": (FEW["long"], 20000), "bf16-32-of-1023": (Step(200, 1023, heads=1), 991),
        "f32-1-of-2011": (Step(16, 2011, heads=2, kv_heads=1, dim=64, dtype="f32"), 2010)}


@pytest.mark.parametrize("name", LOST)
def test_keys_that_are_lost_show(name):
    """The formulas without the last few keys, rounded as the library's results are, in the place of its results."""
    c, keys = LOST[name]
    q, k, v, do, _ = tensors(c, seed=42, device="cpu")
    whole = reference(c, q, k, v, do)[0]
    lost = reference(dataclasses.replace(c, kv_len=(keys,)), q, k, v, do)[0]

    def stored(x):
        return {n: y if n == "lse" else y.to(q.dtype) for n, y in x.items()}
    check_norms(c, stored(whole), whole)
    for n in ("O", "lse", "dQ"):
        with pytest.raises(AssertionError, match=n):
            check_norms(c, {n: stored(lost)[n]}, whole)
