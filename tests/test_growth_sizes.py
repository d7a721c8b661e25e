"""CPU-only checks of what a TierPool knows of programs that grow on the device: host
extents go by the sizes that the plan placed, whoever waits for it, and batches from host
numbers by those that the tables have."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import FirstFit, MoriError, PoolGeometry, TierPool

GEOM = PoolGeometry(2, 2, 16, 256, 64)


class Arena:
    def __init__(self, nbytes):
        self.ptr, self.nbytes, self.fit = 1 << 20, nbytes, FirstFit(nbytes)


def tier_pool(nblk, room=20):
    """One without a device behind it."""
    tp = object.__new__(TierPool)
    off = np.concatenate([[0], np.cumsum(nblk)])
    tp.geom, tp.device, tp.P, tp.ctx = GEOM, torch.device("cpu"), len(nblk), None
    tp.nblk = np.array(nblk, np.int64)
    tp.tbl_off = torch.from_numpy(off.astype(np.int32))
    tp.tbl = torch.full((int(off[-1]) + room,), -1, dtype=torch.int32)
    tp.tbl_len = tp.tbl.numel()
    tp.arena = Arena(4 * GEOM.pool_bytes)
    tp.host_off, tp.host_addr = {}, np.zeros(len(nblk), np.uint64)
    return tp


def grown(tp, nblk):
    tp.tbl_off = torch.from_numpy(np.concatenate([[0], np.cumsum(nblk)]).astype(np.int32))


def plan_of(order, nblk, category, rc=M.MORI_OK):
    """What the library says of a plan over programs of these sizes."""
    P = len(order)
    p = M.mori_plan(num_programs=P)
    arrays = dict(order=(C.c_uint32, order), prefix=(C.c_uint64, np.cumsum(np.asarray(nblk)[order]) * GEOM.block_bytes),
                  tier_old=(C.c_uint8, [0] * P), tier_new=(C.c_uint8, [0] * P), category=(C.c_uint8, category),
                  out_programs=(C.c_uint32, [0] * P), in_programs=(C.c_uint32, [0] * P))
    keep = {n: (t * P)(*(int(x) for x in v)) for n, (t, v) in arrays.items()}
    for n, v in keep.items():
        setattr(p, n, C.cast(v, C.POINTER(v._type_)))
    p.keep = keep
    return lambda ctx: (rc, p)


def test_extents_of_grown_programs(monkeypatch):
    """Every extent holds the program as the plan found it, and none overlaps another."""
    old, new = [1, 2, 0, 3], [4, 2, 5, 3]
    tp = tier_pool(old)
    grown(tp, new)
    category = [M.MORI_CAT_OUT, M.MORI_CAT_OUT, M.MORI_CAT_OUT, M.MORI_CAT_KEPT]
    monkeypatch.setattr(M, "mori_plan_wait", plan_of([2, 0, 3, 1], new, category))
    rc, _ = tp.plan_wait()
    tp.place_host_buffers()
    assert rc == M.MORI_OK and tp.nblk.tolist() == new and tp.nblk.dtype == np.int64
    assert [tp.program_bytes(p) for p in range(4)] == [n * GEOM.block_bytes for n in new]
    ends = sorted((int(tp.host_addr[p]), int(tp.host_addr[p]) + new[p] * GEOM.block_bytes) for p in range(3))
    assert all(a[1] <= b[0] for a, b in zip(ends, ends[1:]))
    assert all(tp.arena.fit.used[tp.host_off[p]] >= new[p] * GEOM.block_bytes for p in range(3))


def test_a_plan_that_failed_says_nothing_of_sizes(monkeypatch):
    tp = tier_pool([1, 2])
    monkeypatch.setattr(M, "mori_plan_wait", plan_of([0, 1], [9, 9], [0, 0], rc=M.MORI_EDEVICE))
    assert tp.plan_wait()[0] == M.MORI_EDEVICE and tp.nblk.tolist() == [1, 2]


def test_no_programs(monkeypatch):
    tp = tier_pool([])
    monkeypatch.setattr(M, "mori_plan_wait", lambda ctx: (M.MORI_OK, M.mori_plan()))
    assert tp.plan_wait()[0] == M.MORI_OK


def test_batches_of_grown_programs(monkeypatch):
    """A length that the program's blocks hold now is taken; one that they do not is refused."""
    made = []
    monkeypatch.setattr(A.TokenBatch, "__init__", lambda self, *a, **k: made.append(k))
    tp = tier_pool([1, 2])
    reads = []
    read = tp.read_sizes
    tp.read_sizes = lambda: (reads.append(1), read())
    A.TokenBatch.of(tp, [0, 1], [1, 1], [16, 32])
    assert len(made) == 1 and not reads  # nothing waits where the known sizes will do
    grown(tp, [3, 2])
    A.TokenBatch.of(tp, [0, 1], [1, 1], [48, 32])
    assert len(made) == 2 and len(reads) == 1 and tp.nblk.tolist() == [3, 2]
    with pytest.raises(MoriError) as e:
        A.TokenBatch.of(tp, [0, 1], [1, 1], [49, 32])
    assert e.value.code == M.MORI_EINVAL and len(made) == 2
    full = tier_pool([1, 2], room=0)
    full.read_sizes = lambda: reads.append(2)
    with pytest.raises(MoriError):
        A.TokenBatch.of(full, [0], [1], [17])
    assert 2 not in reads  # no room to have grown


def test_a_plan_of_other_programs_says_nothing_of_sizes(monkeypatch):
    """One enqueued through the library with fewer of them: what it left behind those is not read."""
    tp = tier_pool([1, 2, 3])
    monkeypatch.setattr(M, "mori_plan_wait", plan_of([1, 0], [7, 7], [0, 0]))
    assert tp.plan_wait()[0] == M.MORI_OK and tp.nblk.tolist() == [1, 2, 3]
