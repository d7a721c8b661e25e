"""Programs that grow between plans, swapped by the calls one by one: every byte of every
program survives, whoever made the growth and whichever call sizes the host extents."""
import numpy as np
import pytest
import torch

from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import TierPool, check
from workload import Geometry

pytestmark = pytest.mark.gpu
BT, ROW, LAYERS = 16, 256, 2


def tier_pool(nblk, num_blocks, room, arena_blocks):
    """Every program on the GPU, pages from the end of the pool, a table with room to grow."""
    off = np.concatenate([[0], np.cumsum(nblk)]).astype(np.uint32)
    total = int(off[-1])
    ids = np.random.default_rng(3).permutation(num_blocks).astype(np.uint32)
    free = np.ones(num_blocks, np.uint8)
    free[ids[:total]] = 0
    g = Geometry(LAYERS, 2, BT, ROW, num_blocks)
    tp = TierPool(g, off, ids[:total].copy(), np.zeros(len(nblk), np.uint8), free,
                  arena_bytes=arena_blocks * LAYERS * 2 * BT * ROW)
    tp.reserve(total + room)
    return tp


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).cuda()


def growth(tp, held, new, prog, direct):
    bounds = dict(num_tokens=int(sum(new)), max_new=max(new), max_kv=5000)
    if direct:
        return A.TokenGrowth(tp.geom, tp.tbl_off, tp.tbl, tp.free_map, held, dev(new), dev(prog), tier=tp.tier, **bounds)
    return A.TokenGrowth.of(tp, held, dev(new), dev(prog), **bounds)


def pages(tp, p):
    off = tp.tbl_off.cpu().numpy()
    return tp.tbl[off[p]:off[p + 1]].long()


def bytes_of(tp, p):
    return tp.pool.view(LAYERS * 2, tp.geom.num_blocks, BT * ROW)[:, pages(tp, p)].clone()


def move(tp, idle, blocks, s_out, s_in):
    """A plan and its swaps, call by call."""
    block = tp.geom.block_bytes
    check(tp.rank_partition(gpu_bytes=blocks * block, cpu_bytes=1000 * block, idleness=idle, flags=M.MORI_F_IDLENESS_GIVEN,
                            stream=s_out), "rank")
    rc, p = tp.plan_wait()
    check(rc, "plan")
    tp.place_host_buffers()
    check(tp.swap_out(M.MORI_COPY_KERNEL, s_out), "out")
    check(tp.swap_in(M.MORI_COPY_KERNEL, s_in), "in")
    return p


@pytest.mark.parametrize("direct", [False, True])
def test_grown_programs_out_and_back(direct):
    """Four neighbours of one block grow to several, go out together and come back."""
    P = 6
    tp = tier_pool([1] * P, 120, 80, 100)
    s_out, s_in = torch.cuda.Stream(), torch.cuda.Stream()
    rng = np.random.default_rng(1)
    held = torch.zeros(P, dtype=torch.int32, device="cuda")
    up, down = torch.arange(P, device="cuda") / 8.0, torch.arange(P, 0, -1, device="cuda") / 8.0
    try:
        moved, want = 0, {}
        for step in range(6):
            here = np.flatnonzero(tp.state()[1] == M.MORI_TIER_GPU)
            new = rng.integers(1, 60, len(here))
            g = growth(tp, held, new.tolist(), here.tolist(), direct)
            g.run().check()
            for p in here:
                tp.pool.view(LAYERS * 2, tp.geom.num_blocks, BT * ROW)[:, pages(tp, p)] = \
                    torch.randint(0, 256, (LAYERS * 2, len(pages(tp, p)), BT * ROW), dtype=torch.uint8, device="cuda")
            for p in here:
                want[int(p)] = bytes_of(tp, p)
            sizes = np.diff(tp.tbl_off.cpu().numpy())
            torch.cuda.synchronize()
            plan = move(tp, up if step % 2 else down, int(sizes.sum()) // 2, s_out, s_in)
            tp.synchronize()
            moved += plan.n_out + plan.n_in
            assert (tp.nblk == sizes).all() and plan.n_drop_gpu == plan.n_drop_cpu == 0
            tier = tp.state()[1]
            for p in range(P):
                if tier[p] == M.MORI_TIER_GPU:
                    assert torch.equal(bytes_of(tp, p), want[p]), p
                else:
                    assert np.array_equal(tp.host_view(p), want[p].cpu().numpy().reshape(-1)), p
        assert moved > 10
    finally:
        tp.close()


def test_batches_from_host_numbers_after_a_growth():
    tp = tier_pool([1] * 4, 60, 40, 60)
    held = torch.zeros(4, dtype=torch.int32, device="cuda")
    try:
        g = growth(tp, held, [30, 50], [1, 2], False)
        g.run().check()
        b = A.TokenBatch.of(tp, [1, 2], [30, 50], [30, 50])
        k = torch.randn(80, 2, 64, device="cuda").bfloat16()
        A.kv_append(tp.pool, tp.geom, 0, b, k, k)
        b.check()
        rows = tp.pool.view(torch.bfloat16).view(LAYERS, 2, tp.geom.num_blocks * BT, 2, 64)
        assert torch.equal(rows[0, 1, g.slots], k)
    finally:
        tp.close()
