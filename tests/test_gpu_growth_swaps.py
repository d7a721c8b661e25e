"""Programs that grow between plans, swapped by the calls one by one: every byte of every
program survives, whoever made the growth and whichever call sizes the host extents."""
import numpy as np
import pytest
import torch

from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError, TierPool, check
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


def streams_apart():
    """Two that do not share a hardware queue: one runs while the other is busy."""
    busy = torch.cuda.Stream()
    for _ in range(16):
        other = torch.cuda.Stream()
        with torch.cuda.stream(busy):
            torch.cuda._sleep(20_000_000)
            slept = busy.record_event()
        other.record_event().synchronize()
        if not slept.query():
            return other, busy
    pytest.skip("every stream waits for the others here")


def test_growth_behind_the_swap_out_while_the_swap_in_waits():
    """Swaps move what the plan placed: a program that is on its way in may grow behind the
    swap-out, its host buffer being no larger than it was."""
    tp = tier_pool([3, 2], 40, 20, 3)  # the arena ends with program 0's buffer
    s_out, s_in = streams_apart()
    held = torch.tensor([40, 20], dtype=torch.int32, device="cuda")
    far, near = torch.tensor([0.9, 0.1], device="cuda"), torch.tensor([0.1, 0.2], device="cuda")
    try:
        tp.pool.random_(0, 256)
        want = [bytes_of(tp, p) for p in (0, 1)]
        torch.cuda.synchronize()
        assert move(tp, far, 2, s_out, s_in).n_out == 1
        tp.synchronize()
        g = growth(tp, held, [70], [0], False)
        torch.cuda.synchronize()
        with torch.cuda.stream(s_in):
            torch.cuda._sleep(200_000_000)
            slept = s_in.record_event()
        assert move(tp, near, 20, s_out, s_in).n_in == 1
        g.run(stream=s_out)
        s_out.synchronize()
        assert not slept.query()  # the growth came first
        tp.synchronize()
        g.batch.check()
        assert np.diff(tp.tbl_off.cpu().numpy()).tolist() == [7, 2]
        assert torch.equal(bytes_of(tp, 0)[:, :3], want[0]) and torch.equal(bytes_of(tp, 1), want[1])
    finally:
        tp.close()


def test_a_growth_of_the_pools_tensors_ends_with_the_table_it_was_made_on():
    tp = tier_pool([1] * 3, 30, 5, 30)
    held = torch.zeros(3, dtype=torch.int32, device="cuda")
    try:
        for direct in (True, False):
            g = growth(tp, held, [3], [0], direct)
            g.run().check()
            before = [x.clone() for x in (tp.tbl_off, tp.tbl, tp.free_map, held)]
            tp.reserve(tp.tbl_len + 4)
            with pytest.raises(MoriError) as e:
                g.run()
            assert e.value.code == M.MORI_EINVAL
            after = (tp.tbl_off, tp.tbl[:before[1].numel()], tp.free_map, held)
            assert all(torch.equal(x, y) for x, y in zip(before, after))
    finally:
        tp.close()


def test_a_moved_table_is_there_for_every_stream():
    """A plan on another stream right behind a move that the current stream was busy before."""
    tp = tier_pool([1] * 8, 60, 0, 30)
    s_out, s_in = torch.cuda.Stream(), torch.cuda.Stream()
    idle = torch.arange(8, device="cuda") / 8.0
    try:
        tp.pool.random_(0, 256)
        want = [bytes_of(tp, p) for p in range(8)]
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)
        tp.reserve(50)
        assert move(tp, idle, 5, s_out, s_in).n_out == 3
        tp.synchronize()
        for p in range(8):
            if p < 5:
                assert torch.equal(bytes_of(tp, p), want[p])
            else:
                assert np.array_equal(tp.host_view(p), want[p].cpu().numpy().reshape(-1))
    finally:
        tp.close()


def test_a_pool_without_blocks_grows_into_its_only_entry():
    """A table of no entries is given one: a growth may take it, and plans know of it."""
    tp = tier_pool([0, 0], 8, 0, 8)
    held = torch.zeros(2, dtype=torch.int32, device="cuda")
    s_out, s_in = torch.cuda.Stream(), torch.cuda.Stream()
    idle = torch.tensor([0.1, 0.9], device="cuda")
    try:
        growth(tp, held, [5], [1], False).run().check()
        tp.pool.random_(0, 256)
        want = bytes_of(tp, 1)
        torch.cuda.synchronize()
        assert tp.state()[0].size == 1 and want.shape[1] == 1
        assert move(tp, idle, 0, s_out, s_in).n_out == 1
        tp.synchronize()
        assert np.array_equal(tp.host_view(1), want.cpu().numpy().reshape(-1))
        move(tp, idle, 4, s_out, s_in)
        tp.synchronize()
        assert torch.equal(bytes_of(tp, 1), want)
    finally:
        tp.close()
