"""What the training step promises in the 2-norm, head by head; shared by its GPU tests.  (check() of dense_training.py
holds every entry to what its roundings may cost if all of them point one way, which on long rows is more than a tile of
keys gives; roundings do not point one way, and a head's norm sees what is missing.)"""
import math

import torch

from dense_training import Step


def limits(c: Step):
    """(of O, of the gradients).  O: its own rounding and that of the weights, 2^-9 sqrt(4/3) of the norm each at the most
    unlucky mantissas, 3.2e-3 together (drawn values of mean zero); a half more for heads of few entries."""
    if c.dtype == "f32":
        return 1e-5, 1e-5
    return 5e-3, 5e-3 if c.compute else 1e-2


def check_norms(c: Step, got, ref):
    """Heads whose exact gradient is zero, as over a single key, are left out: check() has them.

    lse: logits are sums of head_dim products, and so is what they are off by: a few roundings of their size, drawn, and
    the sum over the keys as many as its square root."""
    of_o, of_grads = limits(c)
    worst = {}
    for name, x in got.items():
        want, x = ref[name], x.double()
        if name == "lse":
            live = want != -math.inf
            logit = 8 * c.sigma ** 2 * c.dim * c.args["scale"] + math.log(c.nkv + 1)
            tol = 2.0 ** -24 * (8 * (1 + want[live].abs() + logit) + 4 * math.sqrt(c.nkv))
            off = ((x[live] - want[live]).abs() / tol).flatten()
            limit = 1.0
        else:
            size = want.flatten(0, 1).flatten(1).norm(dim=1)
            off = (x - want).flatten(0, 1).flatten(1).norm(dim=1)[size > 1e-9] / size[size > 1e-9]
            limit = of_o if name == "O" else of_grads
        if off.numel():
            worst[name] = float(off.max())
            assert torch.isfinite(off).all() and worst[name] <= limit, f"{name}: {worst[name]:.1e} of the norm of a head"
    return worst
