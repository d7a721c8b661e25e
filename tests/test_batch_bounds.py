"""CPU-only checks of a batch's bounds: what 32 bits do not hold is refused, not cut to
what they do."""
import pytest
import torch

import grow_ref as R
from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError

BAD = [dict(max_new=1 << 32), dict(max_new=(1 << 32) + 4), dict(max_new=-1), dict(num_tokens=1 << 31),
       dict(num_tokens=(1 << 32) + 8), dict(max_kv=0), dict(max_kv=1 << 31), dict(max_kv=(1 << 32) + 50)]
OK = dict(num_tokens=8, max_new=4, max_kv=50)


class Vector:
    """An int32 vector on a GPU, as far as a batch looks before it takes memory there."""
    dtype, device = torch.int32, torch.device("cuda", 0)
    dim = staticmethod(lambda: 1)
    is_contiguous = staticmethod(lambda: True)

    def __init__(self, n):
        self.numel = lambda: n


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_batches(bad):
    with pytest.raises(MoriError, match="bounds") as e:
        A.TokenBatch(R.Geom(16, 30), *(Vector(n) for n in (5, 20, 4, 3)), **{**OK, **bad})
    assert e.value.code == M.MORI_EINVAL


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_growths(bad):
    z = lambda n, dt=torch.int32: torch.zeros(n, dtype=dt)
    with pytest.raises(MoriError, match="bounds") as e:
        A.TokenGrowth(R.Geom(16, 30), z(5), z(20), z(30, torch.uint8), z(4), z(3), z(3), **{**OK, **bad})
    assert e.value.code == M.MORI_EINVAL
