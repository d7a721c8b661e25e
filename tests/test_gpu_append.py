"""kv_append against the 64-bit definition: both pool forms, rotation styles and
widths, strides, padding, and that no other byte of the pool changes."""
import numpy as np
import pytest
import torch

import attend_ref as R
from paper_2606_00866_amd import mori as M

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def rope(positions, rot, seed=0):
    """Cosines and sines of arbitrary angles, as 32-bit numbers."""
    a = np.random.default_rng(seed).uniform(-3.2, 3.2, (positions, rot // 2))
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1)).float()


def expect(inst, k, v, q, table, style):
    """The pool and the rotated queries by the formula (float64), and the bound of
    a rotated element: two products and a sum in 32 bits, one rounding."""
    t = table.double().numpy() if table is not None else np.zeros((1 << 20, 0))
    pool = inst.pool.double().numpy().copy()
    latent = inst.geom.planes == 1
    qo = None if q is None else np.zeros(q.shape)
    for b in range(inst.n.size):
        for i in range(int(inst.n[b])):
            tok, pos = int(inst.seq_off[b]) + i, int(inst.length[b] - inst.n[b]) + i
            if pos < 0:
                continue
            page, row = inst.slot(b, pos)
            if latent:
                pool[inst.layer, 0, page, row, 0] = np.concatenate(
                    [k[tok, 0].double().numpy(), R.rotated(v[tok, 0].double().numpy(), t[pos], style)])
            else:
                pool[inst.layer, 0, page, row] = R.rotated(k[tok].double().numpy(), t[pos], style)
                pool[inst.layer, 1, page, row] = v[tok].double().numpy()
            if q is not None:
                qo[tok] = R.rotated(q[tok].double().numpy(), t[pos], style)
    return pool, qo


def close(got, want, dtype, size):
    got = got.double().cpu().numpy()
    same = np.isnan(got) & np.isnan(want)
    off = np.where(same, 0, np.abs(got - np.where(same, 0, want)))
    # three roundings in 32 bits of numbers up to 2 * size, one to dtype
    return (off <= R.ROUND[dtype] * np.abs(np.where(same, 0, want)) * 1.001 + 6 * 2.0 ** -24 * size + R.TINY[dtype]).all()


def check(inst, H, rot, style, seed=0, with_q=True):
    from paper_2606_00866_amd import attention as A
    g = torch.Generator().manual_seed(seed)
    T, latent = int(inst.n.sum()), inst.geom.planes == 1
    rnd = lambda *s: torch.randn(*s, generator=g).to(inst.dtype)
    table = rope(max(1, int(inst.length.max())), rot) if rot else None
    k = rnd(T, inst.kv, inst.dim - rot if latent else inst.dim)
    v = rnd(T, inst.kv, rot if latent else inst.dim)
    q = rnd(T, H, rot if latent else inst.dim) if with_q else None
    pool, b = inst.pool.cuda(), R.batch(inst)
    c = lambda x: None if x is None else x.cuda()
    got = A.kv_append(pool, inst.geom, inst.layer, b, c(k), c(v), q=c(q), rope=c(table), style=style)
    b.check()
    want, want_q = expect(inst, k, v, q, table, style)
    assert close(pool, want, inst.dtype, 10.0)
    if with_q:
        assert close(got, want_q, inst.dtype, 10.0)
    return pool


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("style", ["half", "pairs"])
@pytest.mark.parametrize("H,kv,dim,rot", [(8, 4, 64, 64), (32, 8, 128, 128), (3, 1, 128, 32), (1, 1, 16, 16), (6, 2, 80, 80),
                                          (5, 5, 96, 48), (2, 1, 576, 64), (4, 4, 64, 0)])
def test_kv_pools(H, kv, dim, rot, style, dtype):
    check(R.instance(1, [1, 17, 5, 0, 40, 1], [1, 60, 5, 3, 40, 100], kv=kv, dim=dim, dtype=dtype), H, rot, style)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("style", ["half", "pairs"])
@pytest.mark.parametrize("H,dim,rot", [(128, 576, 64), (1, 576, 64), (16, 192, 32), (3, 32, 16)])
def test_latent_pools(H, dim, rot, style, dtype):
    check(R.instance(2, [1, 17, 5, 1], [64, 65, 5, 200], kv=1, dim=dim, planes=1, bt=64, dtype=dtype), H, rot, style)


@pytest.mark.parametrize("bt", [1, 7, 16, 24, 64])
def test_block_sizes_without_queries(bt):
    check(R.instance(3, [3, 50], [10, 120], kv=2, dim=64, bt=bt), 1, 64, "half", with_q=False)


@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 128, 129, 300, 1000, 4096])
def test_many_sequences(B):
    """The search for a token's sequence, empty ones among them."""
    rng = np.random.default_rng(B)
    n = rng.choice([0, 1, 1, 1, 2, 3], size=B)
    check(R.instance(4, n, n + rng.integers(0, 20, size=B), kv=1, dim=16, layers=1, layer=0, spare=0), 1, 16, "half")


def test_large_batch():
    check(R.instance(5, [900, 1, 0, 411], [1000, 5, 0, 411], kv=2, dim=64), 4, 64, "half")


def test_padding():
    """Tokens before position 0: not stored, their queries come back as zeros."""
    from paper_2606_00866_amd import attention as A
    inst = R.instance(6, [3, 1, 5], [1, 0, 5], kv=2, dim=64)
    before = inst.pool.clone()
    k, v, q = (torch.randn(9, h, 64).to(BF16).cuda() for h in (2, 2, 4))
    pool, b = inst.pool.cuda(), R.batch(inst)
    out = A.kv_append(pool, inst.geom, 1, b, k, v, q=q, rope=rope(16, 64).cuda())
    b.check()
    assert (out[:2] == 0).all() and (out[3] == 0).all() and not (out[4:] == 0).all(-1).any()
    page, row = inst.slot(0, 0)
    now = pool.cpu()
    assert not torch.equal(now[1, 0, page, row], before[1, 0, page, row])
    changed = (now.view(torch.int16) != before.view(torch.int16)).flatten(4).any(-1).sum().item()
    assert changed == 2 * 6  # six stored tokens, two planes


def test_fused_projection_in_place():
    """Queries, keys and values side by side; the queries rotated where they are."""
    from paper_2606_00866_amd import attention as A
    H, kv, D, T = 6, 2, 128, 23
    inst = R.instance(7, [20, 3], [20, 70], kv=kv, dim=D)
    x = torch.randn(T, H + 2 * kv, D).to(BF16)
    y, b, t = x.cuda(), R.batch(inst), rope(80, D)
    pool = inst.pool.cuda()
    q = y[:, :H]
    A.kv_append(pool, inst.geom, 1, b, y[:, H:H + kv], y[:, H + kv:], q=q, q_out=q, rope=t.cuda())
    b.check()
    want, want_q = expect(inst, x[:, H:H + kv], x[:, H + kv:], x[:, :H], t, "half")
    assert close(pool, want, BF16, 10.0) and close(q, want_q, BF16, 10.0)
    assert torch.equal(y[:, H:].cpu(), x[:, H:])


def test_broadcast_and_single_strides():
    """One key head for all tokens (stride 0) and views of one token or one head."""
    from paper_2606_00866_amd import attention as A
    inst = R.instance(8, [7], [7], kv=1, dim=64)
    k = torch.randn(1, 1, 64).to(BF16).cuda()
    pool, b = inst.pool.cuda(), R.batch(inst)
    A.kv_append(pool, inst.geom, 1, b, k.expand(7, 1, 64), k.expand(7, 1, 64))
    for j in range(7):
        page, row = inst.slot(0, j)
        assert torch.equal(pool[1, 0, page, row], k[0]) and torch.equal(pool[1, 1, page, row], k[0])


def test_nonfinite_values_travel():
    from paper_2606_00866_amd import attention as A
    inst = R.instance(9, [4], [4], kv=1, dim=64)
    v = torch.full((4, 1, 64), float("inf"), dtype=F16)
    v[1] = float("nan")
    inst2 = R.instance(9, [4], [4], kv=1, dim=64, dtype=F16)
    pool, b = inst2.pool.cuda(), R.batch(inst2)
    A.kv_append(pool, inst2.geom, 1, b, torch.zeros(4, 1, 64, dtype=F16).cuda(), v.cuda(), rope=rope(4, 64).cuda())
    for j in range(4):
        page, row = inst2.slot(0, j)
        got = pool[1, 1, page, row].cpu()
        assert torch.isnan(got).all() if j == 1 else torch.isinf(got).all()
    assert inst.n[0] == 4


def test_device_refusals():
    """A token without a page, past the rotation table or of a sequence that does
    not fit: its bit, nothing stored for it, the others stored."""
    from paper_2606_00866_amd import attention as A
    H, D = 2, 64

    def go(change=None, table=64, **kw):
        inst = R.instance(10, [2, 3], [20, 30], kv=1, dim=D)
        if change:
            change(inst)
        before = inst.pool.clone()
        k, v, q = (torch.ones(5, h, D).to(BF16).cuda() for h in (1, 1, H))
        pool, b = inst.pool.cuda(), R.batch(inst, **kw)
        out = A.kv_append(pool, inst.geom, 1, b, k, v, q=q, rope=rope(table, D).cuda())
        e = int(b.error.item())
        now = pool.cpu()
        return e, (now.view(torch.int16) != before.view(torch.int16)).flatten(4).any(-1).sum().item(), out.cpu()

    assert go()[:2] == (0, 10)

    def page(value):
        def f(i):
            i.tbl[i.tbl_off[i.prog[0]] + 1] = value  # positions 16.. of sequence 0: both its tokens
        return f
    for value, bit in ((R.NONE, M.MORI_DEV_NOT_RESIDENT), (10 ** 6, M.MORI_DEV_PAGE_RANGE), (1 << 31, M.MORI_DEV_PAGE_RANGE)):
        e, stored, out = go(page(value))
        assert (e, stored) == (bit, 6) and not (out == 0).all(-1).any()
    e, stored, out = go(table=20)  # sequence 1 is at 27..29
    assert (e, stored) == (M.MORI_DEV_BAD_TOKENS, 4) and (out[2:] == 0).all()
    for change in (lambda i: i.length.__setitem__(0, 200), lambda i: i.prog.__setitem__(0, 2)):
        e, stored, out = go(change, max_kv=1000)
        assert (e, stored) == (M.MORI_DEV_BAD_TOKENS, 6) and (out[:2] == 0).all()
    e, stored, _ = go(max_new=2)
    assert (e, stored) == (M.MORI_DEV_BAD_TOKENS, 4)
    e, stored, _ = go(max_kv=25)
    assert (e, stored) == (M.MORI_DEV_BAD_TOKENS, 4)


def test_graph_capture():
    from paper_2606_00866_amd import attention as A
    inst = R.instance(11, [1, 1], [5, 40], kv=2, dim=64, spare=2)
    b, t = R.batch(inst, max_kv=60), rope(64, 64).cuda()
    kv_len = b._keep[3]
    pool = inst.pool.cuda()
    k, v, q = (torch.zeros(2, h, 64, dtype=BF16, device="cuda") for h in (2, 2, 4))
    out = torch.empty_like(q)
    A.kv_append(pool, inst.geom, 1, b, k, v, q=q, q_out=out, rope=t)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.kv_append(pool, inst.geom, 1, b, k, v, q=q, q_out=out, rope=t)
    for step in range(1, 5):
        kv_len.add_(1)
        for x in (k, v, q):
            x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(step)))
        other = pool.clone()
        graph.replay()
        torch.cuda.synchronize()
        want_q = A.kv_append(other, inst.geom, 1, b, k, v, q=q, rope=t)
        assert torch.equal(other.view(torch.int16), pool.view(torch.int16)) and torch.equal(want_q, out)
    b.check()


def test_pages_past_4_gib():
    from paper_2606_00866_amd import attention as A
    nb = (1 << 32) // (16 * 2048) + 8
    geom = R.Geom(1, 2, 16, 2048, nb)
    pool = torch.zeros(2 * nb * 16 * 2048, dtype=torch.uint8, device="cuda")
    tbl = np.array([nb - 1, nb - 3])
    b = A.TokenBatch(geom, R.dev32([0, 2]), R.dev32(tbl), R.dev32([0, 2]), R.dev32([20]), num_tokens=2, max_new=2, max_kv=20)
    k, v = torch.randn(2, 8, 128).to(BF16).cuda(), torch.randn(2, 8, 128).to(BF16).cuda()
    A.kv_append(pool, geom, 0, b, k, v)
    b.check()
    view = pool.view(BF16).view(2, nb, 16, 8, 128)
    assert torch.equal(view[0, nb - 3, 2:4], k) and torch.equal(view[1, nb - 3, 2:4], v)
    assert int((view != 0).sum()) == int((k != 0).sum() + (v != 0).sum())
