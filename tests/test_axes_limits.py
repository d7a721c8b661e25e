"""CPU-only checks of numbers of pairs that are none: refused like others that do not fit."""
import pytest
import torch

from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError


@pytest.mark.parametrize("order", ["blocks", "turns"])
@pytest.mark.parametrize("sections", [(float("nan"), 4), (float("inf"),), (2049,), (1 << 22, 1), (4, -float("inf"))], ids=str)
def test_sections(sections, order):
    """Before a list of as many pairs is made."""
    with pytest.raises(MoriError) as e:
        A.pair_axes(sections, order)
    assert e.value.code == M.MORI_EINVAL


def test_the_widest_head():
    assert A.pair_axes((2000, 48)) == [0] * 2000 + [1] * 48


@pytest.mark.parametrize("restart,rot", [((), 0), ((), 32), ((20, -4), 32), ((-1, 1), 0)])
def test_parts_of_a_table(restart, rot):
    with pytest.raises(MoriError) as e:
        A.rope_table(4, rot, device="cpu", restart=restart)
    assert e.value.code == M.MORI_EINVAL


def test_empty_parts_have_no_pairs():
    assert torch.equal(A.rope_table(5, 32, device="cpu", restart=(0, 16)), A.rope_table(5, 32, device="cpu"))
