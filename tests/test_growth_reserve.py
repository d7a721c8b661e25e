"""CPU-only checks of a table that moves: what is under way is waited for, and growths over
the old table are refused, whoever made them."""
import pytest
import torch

from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError, TierPool


def tier_pool():
    tp = object.__new__(TierPool)
    tp.device, tp.tbl_len, tp.ctx = torch.device("cpu"), 3, 77
    tp.tbl = torch.tensor([4, 5, 6], dtype=torch.int32)
    return tp


def test_a_plan_under_way_is_waited_for(monkeypatch):
    """The plan's kernels rewrite the table that is about to move."""
    tp = tier_pool()

    def wait(ctx):
        assert ctx == 77
        tp.tbl[1] = 9  # what the plan writes last
        return M.MORI_OK, None

    monkeypatch.setattr(M, "mori_plan_wait", wait)
    tp.reserve(5)
    assert tp.tbl.tolist() == [4, 9, 6, -1, -1]


def test_no_plan_yet(monkeypatch):
    tp = tier_pool()
    monkeypatch.setattr(M, "mori_plan_wait", lambda ctx: (M.MORI_ESTATE, None))
    tp.reserve(4)
    assert tp.tbl.tolist() == [4, 5, 6, -1]


@pytest.mark.parametrize("into", [False, True])
def test_growths_over_the_old_table_are_refused(monkeypatch, into):
    tp = tier_pool()
    monkeypatch.setattr(M, "mori_plan_wait", lambda ctx: (M.MORI_OK, None))
    ran = []
    monkeypatch.setattr(M, "mori_tables_grow", lambda *a: ran.append(a) or M.MORI_OK)
    monkeypatch.setattr(A, "_stream_of", lambda *a: 0)
    monkeypatch.setattr(A, "_current_device", lambda: 0)
    g = object.__new__(A.TokenGrowth)
    g.batch = object.__new__(A.TokenBatch)
    g.batch.index, g.batch.error = 0, torch.zeros(1, dtype=torch.int32)
    g._pool = g.desc = None
    g._workspace = torch.zeros(1, dtype=torch.uint8)
    other = torch.zeros(3, dtype=torch.int32)
    g._tables, g._written = (other, tp.tbl) if into else (tp.tbl, tp.tbl), ()
    g.run()
    tp.reserve(3)  # there is room: nothing moves
    g.run()
    assert len(ran) == 2
    tp.reserve(8)
    with pytest.raises(MoriError) as e:
        g.run()
    assert e.value.code == M.MORI_EINVAL and len(ran) == 2
