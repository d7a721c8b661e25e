"""CPU-only checks of tables that grow: what the library refuses before anything is
enqueued, what the Python entry point refuses, and the plain definition on a worked case."""
import ctypes as C

import numpy as np
import pytest
import torch

import grow_ref as R
from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError, TierPool

POOL = dict(layers=1, planes=2, block_tokens=16, row_bytes=256, num_blocks=5000, base=256)
OK = dict(num_seqs=3, num_tokens=9, max_new=4, max_kv=100, new_tokens=4096, num_programs=5, tbl_len=70, tbl_off=4096,
          tbl=4096, free_map=4096, held=4096, tbl_off_to=4096, tbl_to=8192, free_to=4096, held_to=4096, seq_off=4096,
          kv_len=4096)


def test_workspace():
    rc, n = M.mori_tables_grow_workspace(M.mori_pool(**POOL), M.mori_growth(**OK))
    assert rc == M.MORI_OK and n > 0
    rc, more = M.mori_tables_grow_workspace(M.mori_pool(**POOL), M.mori_growth(**{**OK, "tbl_to": OK["tbl"]}))
    assert rc == M.MORI_OK and more >= n + 4 * OK["tbl_len"]


@pytest.mark.parametrize("bad", [
    dict(num_seqs=0), dict(num_seqs=M.MORI_MAX_PROGRAMS + 1), dict(num_programs=0),
    dict(num_programs=M.MORI_MAX_PROGRAMS + 1), dict(max_kv=0), dict(max_kv=(1 << 31) - 16), dict(num_tokens=1 << 31),
    dict(tbl_len=0), dict(free_map=4097), dict(free_to=4104)] + [{n: None} for n in (
        "new_tokens", "tbl_off", "tbl", "free_map", "held", "tbl_off_to", "tbl_to", "free_to", "held_to", "seq_off",
        "kv_len")], ids=str)
def test_refused_by_the_library(bad):
    g = M.mori_growth(**{**OK, **bad})
    assert M.mori_tables_grow_workspace(M.mori_pool(**POOL), g)[0] == M.MORI_EINVAL
    assert M.mori_tables_grow(M.mori_pool(**POOL), g, 4096, 1 << 30) == M.MORI_EINVAL


@pytest.mark.parametrize("bad", [dict(block_tokens=0), dict(num_blocks=0), dict(num_blocks=0xFFFFFFFF),
                                 dict(block_tokens=(1 << 18) + 1)], ids=str)
def test_pools_refused(bad):
    assert M.mori_tables_grow_workspace(M.mori_pool(**{**POOL, **bad}), M.mori_growth(**OK))[0] == M.MORI_EINVAL


def test_workspace_refused():
    pool, g = M.mori_pool(**POOL), M.mori_growth(**OK)
    n = M.mori_tables_grow_workspace(pool, g)[1]
    for ws, size in ((0, n), (4096 + 16, n), (4096, n - 1)):
        assert M.mori_tables_grow(pool, g, ws, size) == M.MORI_EINVAL
    assert M.lib().mori_tables_grow(None, C.byref(g), 4096, n, None, None) == M.MORI_EINVAL
    assert M.lib().mori_tables_grow(C.byref(pool), None, 4096, n, None, None) == M.MORI_EINVAL
    assert M.lib().mori_tables_grow_workspace(C.byref(pool), C.byref(g), None) == M.MORI_EINVAL


def tensors(P=4, B=3, entries=20, pages=30):
    z = lambda n, dt=torch.int32: torch.zeros(n, dtype=dt)
    return dict(tbl_off=z(P + 1), tbl=z(entries), free_map=z(pages, torch.uint8), held=z(P), new_tokens=z(B),
                program=z(B), tier=z(P, torch.uint8), num_tokens=8, max_new=4, max_kv=50)


@pytest.mark.parametrize("bad", [
    dict(tbl_off=torch.zeros(5)), dict(held=torch.zeros(5, dtype=torch.int32)),
    dict(free_map=torch.zeros(29, dtype=torch.uint8)), dict(free_map=torch.zeros(30, dtype=torch.int32)),
    dict(tier=torch.zeros(3, dtype=torch.uint8)), dict(program=torch.zeros(4, dtype=torch.int32)),
    dict(new_tokens=torch.zeros(0, dtype=torch.int32), program=None), dict(tbl=torch.zeros(40, dtype=torch.int32)[::2]),
    dict(new_tokens=torch.zeros(5, dtype=torch.int32), program=None), dict(num_tokens=-1), dict(num_tokens=1 << 31),
    dict(held=torch.zeros(4, dtype=torch.int32, device="meta"))], ids=str)
def test_refused_by_the_class(bad):
    with pytest.raises(MoriError) as e:
        A.TokenGrowth(R.Geom(16, 30), **{**tensors(), **bad})
    assert e.value.code == M.MORI_EINVAL


def test_into():
    t = tensors()
    before = [t[k] for k in ("tbl_off", "tbl", "free_map", "held")]
    other = [torch.empty_like(x) for x in before]
    apart = lambda to: A._apart(tuple(to), tuple(before), [t["new_tokens"], t["program"], t["tier"]])
    assert apart(before) and apart(other) and apart([before[0], other[1], before[2], other[3]])
    big = torch.zeros(64, dtype=torch.int32)
    t["tbl"] = before[1] = big[:20]
    assert apart(before) and apart([before[0], big[20:40], before[2], before[3]])
    assert not apart([before[0], big[1:21], before[2], before[3]])
    assert not apart([other[0], other[1], other[2], t["new_tokens"]])
    assert not apart([other[0], other[0], other[2], other[3]])
    for into in (other[:3], [torch.empty(3, dtype=torch.int32), *other[1:]], [other[0], other[1][:9], *other[2:]]):
        with pytest.raises(MoriError):
            A.TokenGrowth(R.Geom(16, 30), **t, into=into)


def test_worked_case():
    """Two programs of blocks of 4; the second takes 6 tokens behind 3, the first one behind 4."""
    s = R.State(R.Geom(4, 6), np.array([0, 1, 2]), np.array([5, 2, -1, -1, -1]), np.array([1, 1, 0, 0, 1, 0], np.uint8),
                np.array([4, 3]), np.zeros(2, np.uint8), np.array([1, 0]), np.array([6, 1]), 8)
    w = R.grow(s)
    assert w["tbl_off"].tolist() == [0, 2, 5] and w["tbl"].tolist() == [5, 4, 2, 0, 1]
    assert w["free"].tolist() == [0] * 6 and w["held"].tolist() == [5, 9] and w["kv_len"].tolist() == [9, 5]
    assert w["slots"].tolist() == [11, 0, 1, 2, 3, 4, 16, -1] and w["positions"].tolist() == [3, 4, 5, 6, 7, 8, 4, -1]


def test_reserve_and_sizes():
    tp = object.__new__(TierPool)
    tp.device, tp.tbl_len = torch.device("cpu"), 3
    tp.tbl = torch.tensor([4, 5, 6], dtype=torch.int32)
    tp.reserve(2)
    assert tp.tbl_len == 3 and tp.tbl.tolist() == [4, 5, 6]
    tp.reserve(5)
    assert tp.tbl_len == 5 and tp.tbl.tolist() == [4, 5, 6, -1, -1]
    tp.tbl_off = torch.tensor([0, 2, 2, 5], dtype=torch.int32)
    tp.read_sizes()
    assert tp.nblk.tolist() == [2, 0, 3] and tp.nblk.dtype == np.int64
