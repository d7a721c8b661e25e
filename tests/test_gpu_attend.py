"""kv_attend against the 64-bit definition: head layouts, block sizes, ragged
batches from one token to prompts, padding, empty sequences, what lies in masked
and unused places, strides, streams, graphs, and the device's refusals."""
import numpy as np
import pytest
import torch

import attend_ref as R
from paper_2606_00866_amd import mori as M

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def run(inst, H, seed=0, q=None, value_dim=None, scale=None, b=None, **kw):
    from paper_2606_00866_amd import attention as A
    g = torch.Generator().manual_seed(seed)
    T = int(inst.n.sum())
    value_dim = value_dim or (512 if inst.geom.planes == 1 else inst.dim)
    scale = scale if scale is not None else (192 if inst.geom.planes == 1 else inst.dim) ** -0.5
    if q is None:
        q = (torch.randn(T, H, inst.dim, generator=g) * 2.5).to(inst.dtype)
    b = b or R.batch(inst)
    pool = inst.pool.cuda()
    lse = torch.full((T, H), 7.0, device="cuda")
    out = A.kv_attend(pool, inst.geom, inst.layer, b, q.cuda(), scale=scale, lse=lse, **kw)
    torch.cuda.synchronize()
    return q, scale, value_dim, out, lse, b


def check(inst, H, rows=None, heads=slice(None), **kw):
    """heads: those that are compared (only where inst has one key head)."""
    q, scale, vd, out, lse, b = run(inst, H, **kw)
    b.check()
    want, want_lse, mean, delta, count, top = R.attend(inst, q[:, heads], scale, vd)
    got, got_lse = out[:, heads].double().cpu().numpy(), lse[:, heads].double().cpu().numpy()
    bound = R.attend_bound(inst.dtype, want, mean, delta, count, top)
    rows = slice(None) if rows is None else rows
    assert np.isfinite(got[rows]).all()
    off = np.abs(got - want)[rows]
    assert (off <= bound[rows]).all(), f"off by {(off / bound[rows]).max():.3f} of the bound"
    empty = np.isneginf(want_lse[rows])
    assert (np.isneginf(got_lse[rows]) == empty).all()
    lse_off = np.abs(np.where(empty, 0, got_lse[rows]) - np.where(empty, 0, want_lse[rows]))
    # the sum's logarithm: the scores' error, the sum's (2^-16) and the value's own 32 bits
    assert (lse_off <= delta[rows][..., 0] * 2 + 2.0 ** -16 + 2.0 ** -22 * np.abs(np.where(empty, 0, want_lse[rows]))).all()
    return out


LAYOUTS = [(8, 4, 64), (32, 8, 128), (16, 1, 128), (7, 7, 64), (10, 2, 128), (12, 4, 64), (40, 1, 64), (5, 1, 128)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("H,kv,dim", LAYOUTS)
def test_step(H, kv, dim, dtype):
    """One token each, contexts of every size class."""
    length = [1, 2, 15, 16, 17, 33, 64, 200, 513]
    check(R.instance(1, [1] * len(length), length, kv=kv, dim=dim, dtype=dtype), H)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("H,kv,dim", LAYOUTS)
def test_chunks(H, kv, dim, dtype):
    """Chunks behind contexts, whole prompts and single tokens in one batch."""
    n = [1, 5, 17, 64, 3, 1, 70]
    length = [40, 5, 100, 64, 300, 1, 131]
    check(R.instance(2, n, length, kv=kv, dim=dim, dtype=dtype), H)


@pytest.mark.parametrize("bt", [1, 7, 16, 24, 32, 64, 128])
@pytest.mark.parametrize("n", [1, 40])
def test_block_sizes(bt, n):
    check(R.instance(3, [n, n, n], [n, 150, 333], kv=2, dim=128, bt=bt), 8)


@pytest.mark.parametrize("n", [1, 2, 4, 8, 16, 31, 32, 33, 63, 65, 127, 129, 255, 257])
def test_new_token_counts(n):
    """Rows of a key head (4 n) on both sides of every tile size."""
    check(R.instance(4, [n, 1], [n + 77, 90], kv=1, dim=128), 4)


@pytest.mark.parametrize("length", [1, 31, 32, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1025])
def test_lengths(length):
    check(R.instance(5, [1, min(20, length)], [length, length], kv=2, dim=64), 8)


def test_long_context_split():
    """One program, far more keys than one workgroup takes: split and joined."""
    check(R.instance(6, [1], [20011], kv=1, dim=128), 8)


def test_long_contexts_among_short_ones():
    check(R.instance(7, [1] * 12 + [9], [1, 3, 9000, 40, 1, 700, 64, 2, 4096, 5, 16, 1, 3001], kv=2, dim=64), 8)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("H", [16, 128, 1, 5, 24])
def test_latent_step(H, dtype):
    length = [1, 15, 64, 65, 200, 700]
    check(R.instance(8, [1] * len(length), length, kv=1, dim=576, planes=1, bt=64, dtype=dtype), H)


@pytest.mark.parametrize("H", [16, 3, 64])
def test_latent_chunks(H):
    check(R.instance(9, [1, 5, 17, 30], [40, 5, 100, 131], kv=1, dim=576, planes=1, bt=16), H)


def test_latent_long_split():
    check(R.instance(10, [1, 2], [6007, 31], kv=1, dim=576, planes=1, bt=64), 16)


def test_latent_many_heads_split():
    """More runs of keys than the chip takes at a time unless they are made longer."""
    length = [15000, 9001, 17777, 12345, 16000, 14999, 11111, 13000, 18000, 8192]
    check(R.instance(24, [1] * len(length), length, kv=1, dim=576, planes=1, bt=64), 65, heads=slice(0, 65, 16))


def test_latent_many_sequences():
    """More sequences than a wavefront has lanes, a few of them split."""
    length = [1 + 5 * i for i in range(69)] + [2500, 1]
    check(R.instance(25, [1] * 70 + [0], length, kv=1, dim=576, planes=1, bt=16), 100, heads=slice(3, 100, 24))


def test_padding_and_empty_sequences():
    """Padding tokens (before position 0), sequences without tokens and programs
    without any: zeros and -inf for the first, nothing for the others."""
    inst = R.instance(11, [3, 0, 4, 1, 0, 40], [1, 0, 4, 0, 9, 10], kv=2, dim=64)
    out = check(inst, 8)
    o = out.cpu()
    assert (o[0:2] == 0).all() and (o[7] == 0).all() and (o[8:8 + 30] == 0).all()


def test_latent_padding():
    inst = R.instance(12, [3, 1, 5], [1, 0, 2], kv=1, dim=576, planes=1)
    check(inst, 16)


def test_tokens_outside_the_sequences_are_left_alone():
    inst = R.instance(13, [2, 3], [20, 30], kv=1, dim=64)
    inst.seq_off = inst.seq_off + 1  # one token before, two behind
    q = torch.randn(8, 4, 64).to(BF16)
    from paper_2606_00866_amd import attention as A
    out = torch.full((8, 4, 64), 5.0, dtype=BF16, device="cuda")
    b = R.batch(inst, tokens=8)
    A.kv_attend(inst.pool.cuda(), inst.geom, 1, b, q.cuda(), out=out)
    b.check()
    o = out.cpu()
    assert (o[0] == 5).all() and (o[6:] == 5).all() and not (o[1:6] == 5).all(-1).any()


@pytest.mark.parametrize("planes", [1, 2])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("n", [2, 24, 100])
def test_later_tokens_do_not_reach_earlier_rows(n, bad, planes):
    """A key or value that is not finite changes only the rows that attend to it."""
    dim, H = (576, 4) if planes == 1 else (128, 4)
    inst = R.instance(14, [n], [n + 30], kv=1, dim=dim, planes=planes)
    first = n // 2  # the chunk's token that is spoilt
    for plane in range(planes):
        page, row = inst.slot(0, 30 + first)
        inst.pool[1, plane, page, row, 0, 3 + plane] = bad
    check(inst, H, rows=slice(0, first))


def test_large_scores():
    """Scores of hundreds: weights of one key, no overflow."""
    inst = R.instance(15, [1, 33], [300, 90], kv=1, dim=128)
    q = (torch.randn(34, 4, 128) * 40).to(BF16)
    check(inst, 4, q=q, scale=1.0)


def test_rising_scores_rescale():
    """Every tile of keys holds a larger score than all before it."""
    inst = R.instance(16, [1, 20], [400, 400], kv=1, dim=64)
    for b in range(2):
        for j in range(400):
            page, row = inst.slot(b, j)
            inst.pool[1, 0, page, row, 0, :] = 0.02 * j
    q = (torch.rand(21, 4, 64) + 0.5).to(BF16)
    check(inst, 4, q=q)


@pytest.mark.parametrize("scale", [0.0, -0.3])
def test_scale(scale):
    check(R.instance(17, [1, 20], [100, 70], kv=2, dim=64), 4, scale=scale)


def test_fp16_small_weights():
    """Thousands of keys far below one large score, in the type with few exponents."""
    inst = R.instance(18, [1], [4000], kv=1, dim=64, dtype=F16)
    page, row = inst.slot(0, 17)
    inst.pool[1, 0, page, row, 0, :] = 1.0
    q = torch.full((1, 2, 64), 1.25, dtype=F16)
    check(inst, 2, q=q, scale=0.125)


def test_strided_views():
    """Queries inside a fused projection's output, outputs into a wider buffer."""
    from paper_2606_00866_amd import attention as A
    for planes, dim, H, vd in ((2, 128, 8, 128), (1, 576, 8, 512)):
        inst = R.instance(19, [1, 40], [50, 90], kv=1, dim=dim, planes=planes)
        x = torch.randn(41, H + 3, dim + 16).to(BF16)
        q = x[:, 2:2 + H, 8:8 + dim]
        wide = torch.full((41, H + 1, vd + 24), 3.0, dtype=BF16, device="cuda")
        out = wide[:, :H, 16:16 + vd]
        b = R.batch(inst)
        A.kv_attend(inst.pool.cuda(), inst.geom, 1, b, x.cuda()[:, 2:2 + H, 8:8 + dim], out=out, scale=0.1)
        plain = A.kv_attend(inst.pool.cuda(), inst.geom, 1, b, q.contiguous().cuda(), scale=0.1)
        assert torch.equal(out, plain)
        w = wide.cpu()
        assert (w[:, H] == 3).all() and (w[..., :16] == 3).all() and (w[..., 16 + vd:] == 3).all()


def test_same_result_every_time():
    from paper_2606_00866_amd import attention as A
    inst = R.instance(20, [1, 1, 30], [9000, 20, 3000], kv=2, dim=128)
    q = torch.randn(32, 8, 128).to(BF16).cuda()
    b, pool = R.batch(inst), inst.pool.cuda()
    ws = A.kv_attend_workspace(inst.geom, b, q)
    first = A.kv_attend(pool, inst.geom, 1, b, q, workspace=ws)
    for fill in (0xFF, 0x7F, 0x00):  # what the workspace holds before does not matter
        ws.fill_(fill)
        assert torch.equal(A.kv_attend(pool, inst.geom, 1, b, q, workspace=ws), first)


def test_another_stream():
    from paper_2606_00866_amd import attention as A
    inst = R.instance(21, [1, 9], [5000, 600], kv=2, dim=128)
    q, b, pool = torch.randn(10, 8, 128).to(BF16).cuda(), R.batch(inst), inst.pool.cuda()
    want = A.kv_attend(pool, inst.geom, 1, b, q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    outs = [A.kv_attend(pool, inst.geom, 1, b, q, stream=s) for _ in range(3)]
    junk = [torch.full((1 << 20,), 0xAB, dtype=torch.uint8, device="cuda") for _ in range(8)]  # the current stream's
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs) and len(junk) == 8


def test_graph_replays_with_growing_programs():
    """A captured decode step: lengths and queries change between the replays, a
    padded sequence among them."""
    from paper_2606_00866_amd import attention as A
    inst = R.instance(22, [1, 1, 1], [700, 40, 0], kv=2, dim=64, spare=2)
    b = R.batch(inst, max_kv=1024)
    tbl_off, tbl, seq_off, kv_len, prog = b._keep
    pool, q = inst.pool.cuda(), torch.zeros(3, 4, 64, dtype=BF16, device="cuda")
    ws, out = A.kv_attend_workspace(inst.geom, b, q), torch.empty(3, 4, 64, dtype=BF16, device="cuda")
    A.kv_attend(pool, inst.geom, 1, b, q, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.kv_attend(pool, inst.geom, 1, b, q, out=out, workspace=ws)
    for step in range(4):
        length = np.array([700 - 13 * step, 40 - 9 * step, 0])
        kv_len.copy_(R.dev32(length))
        q.copy_(torch.randn(3, 4, 64, generator=torch.Generator().manual_seed(step)))
        out.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, A.kv_attend(pool, inst.geom, 1, b, q))
        assert (got[2] == 0).all()
        inst.length = length
        want, _, mean, delta, count, top = R.attend(inst, q.cpu(), 64 ** -0.5, 64)
        assert (np.abs(got.double().cpu().numpy() - want) <= R.attend_bound(BF16, want, mean, delta, count, top)).all()
    b.check()


def test_pages_past_4_gib():
    """A plane of more than 2^32 bytes: the last pages are the program's."""
    from paper_2606_00866_amd import attention as A
    small = R.instance(23, [2], [100], kv=8, dim=128)
    nb = (1 << 32) // (16 * 2048) + 64
    geom = R.Geom(1, 2, 16, 2048, nb)
    pool = torch.empty(2 * nb * 16 * 2048, dtype=torch.uint8, device="cuda")
    view = pool.view(BF16).view(2, nb, 16, 8, 128)
    shift = nb - small.geom.num_blocks
    view[:, shift:] = small.pool[1].cuda()
    q = torch.randn(2, 16, 128).to(BF16).cuda()
    want = A.kv_attend(small.pool.cuda(), small.geom, 1, R.batch(small), q)
    small.geom, small.tbl = geom, small.tbl + shift
    assert torch.equal(A.kv_attend(pool, geom, 0, R.batch(small), q), want)


@pytest.mark.parametrize("planes", [1, 2])
@pytest.mark.parametrize("n", [1, 50])
def test_device_refusals(n, planes):
    """Numbers that do not fit set their bit; the sequence is padding, the others
    are right, and nothing else is written."""
    dim, H = (576, 16) if planes == 1 else (64, 4)
    from paper_2606_00866_amd import attention as A

    def bits(inst, **kw):
        q, scale, vd, out, lse, b = run(inst, H, **kw)
        e = int(b.error.item())
        with pytest.raises(A.MoriError):
            b.check()
        b.check()  # cleared
        return e, out.cpu(), lse.cpu()

    fresh = lambda: R.instance(24, [n, n], [n + 60, n + 40], kv=1, dim=dim, planes=planes)
    good = run(fresh(), H)[3].cpu()
    def broken(**change):
        i = fresh()
        for k, v in change.items():
            getattr(i, k)[0] = v
        return i
    limit = int((fresh().tbl_off[fresh().prog[0] + 1] - fresh().tbl_off[fresh().prog[0]]) * 16)
    for inst, kw in ((broken(length=limit + 1), dict(max_kv=10 ** 6)), (broken(prog=2), {}),
                     (fresh(), dict(max_kv=n + 50)), (broken(prog=1 << 31), {})):
        b = R.batch(inst, **kw)
        e, out, lse = bits(inst, b=b)
        assert e == M.MORI_DEV_BAD_TOKENS
        assert (out[:n] == 0).all() and torch.isneginf(lse[:n]).all()
        assert torch.equal(out[n:], good[n:])
    if n > 1:
        inst = fresh()
        e, out, _ = bits(inst, b=R.batch(inst, max_new=n - 1))
        assert e == M.MORI_DEV_BAD_TOKENS and (out == 0).all()
    for page, bit in ((R.NONE, M.MORI_DEV_NOT_RESIDENT), (fresh().geom.num_blocks, M.MORI_DEV_PAGE_RANGE),
                      (1 << 31, M.MORI_DEV_PAGE_RANGE)):
        inst = fresh()
        inst.tbl[inst.tbl_off[inst.prog[0]] + 1] = page
        e, out, _ = bits(inst)
        assert e == bit and torch.equal(out[n:], good[n:])
    inst = fresh()
    inst.seq_off = np.array([0, 3 * n, 2 * n])  # decreasing
    e, out, _ = bits(inst)
    assert e == M.MORI_DEV_BAD_TOKENS


@pytest.mark.parametrize("planes", [1, 2])
def test_overlapping_sequences_stay_inside_the_workspace(planes):
    """Offsets that name tokens twice give more items than the workspace is for:
    the fault is reported, what is written stays in bounds."""
    from paper_2606_00866_amd import attention as A
    dim, H = (576, 16) if planes == 1 else (128, 8)
    inst = R.instance(25, [40] * 9, [3000] * 9, kv=1, dim=dim, planes=planes)
    inst.seq_off = np.array([0, 40, 0, 40, 0, 40, 0, 40, 0, 40])
    b = R.batch(inst, tokens=40)
    q = torch.randn(40, H, dim).to(BF16).cuda()
    ws = A.kv_attend_workspace(inst.geom, b, q)
    guarded = torch.full((ws.numel() + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    A.kv_attend(inst.pool.cuda(), inst.geom, 1, b, q, workspace=guarded[:ws.numel()])
    torch.cuda.synchronize()
    assert int(b.error.item()) == M.MORI_DEV_BAD_TOKENS
    assert (guarded[ws.numel():] == 0x5A).all()
