"""kv_append with positions of several axes, against a plain rotation in 64 bits."""
import numpy as np
import pytest
import torch

import attend_ref as R
from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def table(length, rot):
    return A.rope_table(length, rot, theta=1e4)


def turned(x, at, rope, sections, order, style):
    """x float64 [H][D] of one token; at: its positions by axis; rope float64."""
    rot = rope.shape[1]
    axes = A.pair_axes(sections, order)
    row = np.array([rope[at[a], i] for i, a in enumerate(axes)] + [rope[at[a], rot // 2 + i] for i, a in enumerate(axes)])
    return np.concatenate([R.rotated(x[..., :rot], row, style), x[..., rot:]], -1)


def bound(want, dtype):
    """The table's entries are the same numbers; two products and a sum in 32 bits (three
    roundings of at most 2^-24 of the larger terms), then one to dtype."""
    return R.ROUND[dtype] * np.abs(want) + R.TINY[dtype]


CASES = [
    # n, length, kv, q, dim, rot, sections, order, style, dtype, bt
    ([1] * 5, [3, 700, 17, 64, 1], 4, 8, 64, 64, (8, 12, 12), "blocks", "half", F16, 16),
    ([30, 1, 77], [30, 41, 200], 2, 6, 64, 64, (12, 10, 10), "turns", "half", BF16, 16),
    ([50, 9], [90, 9], 1, 8, 128, 128, (16, 24, 24), "blocks", "pairs", BF16, 32),
    ([50, 9], [90, 9], 2, 2, 128, 128, (24, 20, 20), "turns", "pairs", F16, 16),
    ([13], [13], 2, 4, 128, 64, (7, 11, 14), "blocks", "half", BF16, 16),       # part of the head, borders within four pairs
    ([13, 2], [40, 30], 2, 4, 128, 64, (7, 11, 14), "blocks", "pairs", F16, 24),
    ([13, 2], [40, 30], 1, 5, 64, 32, (1, 2, 3, 10), "blocks", "half", BF16, 16),
    ([33], [50], 1, 5, 64, 64, (8, 8, 8, 8), "turns", "half", BF16, 16),
    ([33], [50], 3, 3, 64, 64, (16, 16), "turns", "pairs", F16, 16),
    ([20], [20], 3, 3, 80, 64, (32,), "blocks", "half", BF16, 16),                 # one axis: positions of one's own
    ([20], [25], 3, 3, 80, 64, (32,), "turns", "pairs", BF16, 17),
    ([20], [25], 1, 1, 64, 64, (0, 32), "blocks", "half", BF16, 16),             # an axis without pairs
    ([600], [600], 1, 1, 16, 16, (3, 2, 3), "blocks", "half", F16, 16),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_against_definition(case):
    n, length, kv, heads, dim, rot, sections, order, style, dtype, bt = case
    inst = R.instance(len(str(case)), n, length, kv=kv, dim=dim, dtype=dtype, bt=bt)
    rng = np.random.default_rng(3)
    T, axes, positions = int(sum(n)), len(sections), 500
    at = rng.integers(0, positions, (axes, T))
    rope = table(positions, rot)
    x = torch.from_numpy(rng.standard_normal((T, heads + 2 * kv, dim))).to(dtype)
    d = x.cuda()
    q, k, v = d[:, :heads], d[:, heads:heads + kv], d[:, heads + kv:]
    pool = inst.pool.cuda()
    b = R.batch(inst)
    d_at = torch.full((axes, T + 5), -7, dtype=torch.int32, device="cuda")[:, 2:T + 2]  # rows of a wider tensor
    d_at.copy_(torch.from_numpy(at).int())
    out = A.kv_append(pool, inst.geom, inst.layer, b, k, v, q=q, rope=rope, style=style, positions=d_at,
                      sections=sections, order=order)
    b.check()
    table64, x64, out, got = rope.double().cpu().numpy(), x.double().numpy(), out.double().cpu().numpy(), pool.cpu()
    want = inst.pool.clone()
    seq = np.repeat(np.arange(len(n)), n)
    for t in range(T):
        pos = int(length[seq[t]] - n[seq[t]] + t - inst.seq_off[seq[t]])
        page, row = inst.slot(seq[t], pos)
        w = turned(x64[t, :heads], at[:, t], table64, sections, order, style)
        assert (np.abs(out[t] - w) <= 1.01 * bound(w, dtype) + 2.0 ** -22 * np.abs(x64[t]).max()).all()
        w = turned(x64[t, heads:heads + kv], at[:, t], table64, sections, order, style)
        g = got[inst.layer, 0, page, row].double().numpy()
        assert (np.abs(g - w) <= 1.01 * bound(w, dtype) + 2.0 ** -22 * np.abs(x64[t]).max()).all()
        assert torch.equal(got[inst.layer, 1, page, row], x[t, heads + kv:])
        want[inst.layer, 0, page, row] = got[inst.layer, 0, page, row]
        want[inst.layer, 1, page, row] = x[t, heads + kv:]
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))  # nothing else was written


@pytest.mark.parametrize("style", ["half", "pairs"])
@pytest.mark.parametrize("order", ["blocks", "turns"])
def test_equal_axes_are_a_token_position(style, order):
    """Where every axis has the token's own position, the result is that of the plain call,
    bit for bit; padding included (a sequence shorter than what it brings)."""
    inst = R.instance(5, [40, 3, 1], [100, 3, 30], kv=2, dim=64)
    inst.n[1] = 7  # four of them are padding
    inst.seq_off = np.concatenate([[0], np.cumsum(inst.n)])
    T = int(inst.n.sum())
    pos = np.concatenate([np.arange(l - m, l) for m, l in zip(inst.n, inst.length)])
    rope = table(120, 64)
    x = torch.randn(T, 10, 64, device="cuda").bfloat16()
    at = torch.from_numpy(np.stack([pos] * 3)).int().cuda()  # negative where it is padding: not looked at
    pools, outs = [], []
    for kw in ({}, dict(positions=at, sections=(12, 10, 10), order=order)):
        pool, b = inst.pool.cuda(), R.batch(inst)
        outs.append(A.kv_append(pool, inst.geom, 1, b, x[:, 6:8], x[:, 8:], q=x[:, :6], rope=rope, style=style, **kw))
        pools.append(pool)
        if not kw:
            b.check()
    assert torch.equal(outs[0], outs[1])
    assert torch.equal(pools[0].view(torch.int16), pools[1].view(torch.int16))
    assert (outs[1][40:44] == 0).all()
    b.check()


def test_latent_pool():
    inst = R.instance(8, [9, 4], [30, 4], kv=1, dim=576, planes=1, bt=64)
    T, rope = 13, table(60, 64)
    k, v, q = (torch.randn(T, h, d, device="cuda").bfloat16() for h, d in ((1, 512), (1, 64), (4, 64)))
    at = torch.randint(0, 60, (3, T), device="cuda", dtype=torch.int32)
    pool, b = inst.pool.cuda(), R.batch(inst)
    out = A.kv_append(pool, inst.geom, 1, b, k, v, q=q, rope=rope, style="pairs", positions=at, sections=(8, 12, 12))
    b.check()
    t64, at = rope.double().cpu().numpy(), at.cpu().numpy()
    seq = np.repeat([0, 1], [9, 4])
    for t in range(T):
        w = turned(q[t].double().cpu().numpy(), at[:, t], t64, (8, 12, 12), "blocks", "pairs")
        assert (np.abs(out[t].double().cpu().numpy() - w) <= 1.01 * bound(w, BF16) + 2.0 ** -20).all()
        page, row = inst.slot(seq[t], int(inst.length[seq[t]] - inst.n[seq[t]] + t - inst.seq_off[seq[t]]))
        g = pool[1, 0, page, row, 0].cpu()
        assert torch.equal(g[:512], k[t, 0].cpu())
        w = turned(v[t].double().cpu().numpy(), at[:, t], t64, (8, 12, 12), "blocks", "pairs")[0]
        assert (np.abs(g[512:].double().numpy() - w) <= 1.01 * bound(w, BF16) + 2.0 ** -20).all()


@pytest.mark.parametrize("value", [-1, 50, 2 ** 31 - 1, -2 ** 31])
def test_positions_without_a_row(value):
    """That token is not stored and its query is 0; the others are."""
    inst = R.instance(9, [6], [20], kv=2, dim=64)
    rope = table(50, 64)
    x = torch.randn(6, 6, 64, device="cuda").bfloat16()
    at = torch.randint(0, 50, (3, 6), device="cuda", dtype=torch.int32)
    pools, outs = [], []
    for bad in (False, True):
        a = at.clone()
        if bad:
            a[2, 4] = value
        pool, b = inst.pool.cuda(), R.batch(inst)
        outs.append(A.kv_append(pool, inst.geom, 1, b, x[:, 2:4], x[:, 4:], q=x[:, :2], rope=rope, positions=a,
                                sections=(8, 12, 12)))
        pools.append(pool.cpu())
        if bad:
            with pytest.raises(MoriError) as e:
                b.check()
            assert e.value.detail == M.MORI_DEV_BAD_TOKENS
        else:
            b.check()
    page, row = inst.slot(0, 18)
    assert (outs[1][4] == 0).all() and torch.equal(pools[1][1, :, page, row], inst.pool[1, :, page, row])
    outs[0][4] = 0
    pools[0][1, :, page, row] = inst.pool[1, :, page, row]
    assert torch.equal(outs[0], outs[1]) and torch.equal(pools[0].view(torch.int16), pools[1].view(torch.int16))


def test_large_batch():
    """More tokens than a workgroup's, odd heads; all outputs against the same rotation in
    32 bits on the device, in another order of work."""
    n, kv, heads, dim = [700, 1, 1300], 3, 7, 128
    inst = R.instance(10, n, [900, 40, 1300], kv=kv, dim=dim, layers=1, layer=0)
    T, s = sum(n), (16, 24, 24)
    rope = table(2000, dim)
    x = torch.randn(T, heads + 2 * kv, dim, device="cuda").bfloat16()
    at = torch.randint(0, 2000, (3, T), device="cuda", dtype=torch.int32)
    pool, b = inst.pool.cuda(), R.batch(inst)
    out = A.kv_append(pool, inst.geom, 0, b, x[:, heads:heads + kv], x[:, heads + kv:], q=x[:, :heads], rope=rope,
                      positions=at, sections=s)
    b.check()
    axis = torch.tensor(A.pair_axes(s), device="cuda")
    row = at.long()[axis].t()
    c, sn = (rope.double()[row, torch.arange(64, device="cuda") + o][:, None] for o in (0, 64))
    y = x.double()
    w = torch.cat([y[..., :64] * c - y[..., 64:] * sn, y[..., 64:] * c + y[..., :64] * sn], -1)
    tol = 1.01 * 2.0 ** -8 * w.abs() + 2.0 ** -20
    assert ((out.double() - w[:, :heads]).abs() <= tol[:, :heads]).all()
    seq = np.repeat(np.arange(3), n)
    pos = inst.length[seq] - inst.n[seq] + np.arange(T) - inst.seq_off[seq]
    page = torch.from_numpy(inst.tbl[inst.tbl_off[inst.prog[seq]] + pos // 16]).cuda()
    r = torch.from_numpy(pos % 16).cuda()
    assert ((pool[0, 0, page, r].double() - w[:, heads:heads + kv]).abs() <= tol[:, heads:heads + kv]).all()
    assert torch.equal(pool[0, 1, page, r], x[:, heads + kv:])


def test_graph_replays():
    """Positions are read at replay."""
    inst = R.instance(11, [20, 1], [50, 9], kv=2, dim=64)
    rope, x = table(80, 64), torch.randn(21, 6, 64, device="cuda").bfloat16()
    at = torch.randint(0, 80, (3, 21), device="cuda", dtype=torch.int32)
    pool, b, out = inst.pool.cuda(), R.batch(inst), torch.empty(21, 2, 64, device="cuda", dtype=BF16)
    call = lambda p, o: A.kv_append(p, inst.geom, 1, b, x[:, 2:4], x[:, 4:], q=x[:, :2], q_out=o, rope=rope, positions=at,
                                    sections=(12, 10, 10), order="turns")
    call(pool, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(pool, out)
    for _ in range(4):
        at.copy_(torch.randint(0, 80, (3, 21), device="cuda", dtype=torch.int32))
        graph.replay()
        p, o = inst.pool.cuda(), torch.empty_like(out)
        call(p, o)
        assert torch.equal(o, out) and torch.equal(p.view(torch.int16), pool.view(torch.int16))
    b.check()
