"""What the training step takes for scratch memory: the binding tells the library how many bytes there are, so that a tensor
which names more elements than it has, or elements apart, is refused.  No kernel is launched here."""
import pytest
import torch

import paper_2602_12271_amd as pkg
from paper_2602_12271_amd import binding as B


class OnGpu:
    """A tensor on the host that says it is on the GPU."""

    def __init__(self, x):
        self._x = x

    def get_device(self):
        return 0

    def __getattr__(self, name):
        return getattr(self._x, name)


BAD = {"expanded": torch.zeros(1, dtype=torch.uint8).expand(1 << 20), "apart": torch.zeros(64, 64, dtype=torch.uint8)[:, ::2]}


@pytest.mark.parametrize("name", BAD)
def test_scratch_that_is_not_there(name):
    x, lse, ws = (OnGpu(y) for y in (torch.zeros(1, 2, 30, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 30), BAD[name]))
    grid = dict(f_q=1, f_kv=1, h=5, w=6, workspace=ws)
    for call in (lambda: pkg.dense_attn_fwd_save(x, x, x, **grid), lambda: pkg.dense_attn_bwd(x, x, x, x, x, lse, **grid)):
        with pytest.raises(pkg.MrtError, match="workspace") as e:
            call()
        assert e.value.status == B.MRT_ERR_WORKSPACE


def test_scratch_of_any_type():
    for ws in (None, torch.zeros(256, dtype=torch.uint8), torch.zeros(8, 8), torch.zeros(0), torch.zeros(4, 64)[1:3]):
        B._require_scratch(ws)
