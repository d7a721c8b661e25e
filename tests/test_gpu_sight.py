"""Attention with caps, biases by distance, windows and ranges, against the definition in
64 bits.  Free pages, other layers and rows past a program's length hold NaN."""
import numpy as np
import pytest
import torch

import attend_ref as R
import sight_ref as S
from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def queries(inst, H, scale=2.5, seed=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(int(inst.n.sum()), H, inst.dim, generator=g) * scale).to(inst.dtype)


def positions(inst):
    return np.concatenate([np.arange(l - n, l) for n, l in zip(inst.n, inst.length)]).astype(np.int64)


def documents(inst, mean, seed=1):
    """Where each token's document begins."""
    rng, out = np.random.default_rng(seed), []
    for n, l in zip(inst.n.tolist(), inst.length.tolist()):
        starts = np.concatenate([[0], np.cumsum(rng.integers(1, 2 * mean + 1, 2 + 4 * l // mean))])
        pos = np.arange(l - n, l)
        out.append(np.where(pos < 0, 0, starts[np.maximum(np.searchsorted(starts, pos, side="right") - 1, 0)]))
    return np.concatenate(out).astype(np.int32)


def slopes_of(H):
    return np.exp2(-8.0 * np.arange(1, H + 1) / H).astype(np.float32)


def dev(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def run(inst, q, scale, lse=True, **kw):
    b = R.batch(inst)
    out = torch.full((*q.shape,), float("nan"), dtype=q.dtype, device="cuda")
    l = torch.full(q.shape[:2], float("nan"), device="cuda") if lse else None
    k = {n: dev(x) if isinstance(x, np.ndarray) else x for n, x in kw.items()}
    A.kv_attend(inst.pool.cuda(), inst.geom, inst.layer, b, q.cuda(), scale=scale, out=out, lse=l, **k)
    b.check()
    return out.double().cpu().numpy(), l.double().cpu().numpy() if lse else None


def compare(inst, q, scale, **kw):
    out, lse = run(inst, q, scale, **kw)
    want, want_lse, bound, delta = S.attend(inst, q, scale, **kw)
    bad = ~(np.abs(out - want) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:3], np.abs(out - want)[bad][:3], bound[bad][:3])
    none = np.isneginf(want_lse)
    assert (np.isneginf(lse) == none).all() and (out[none] == 0).all()
    # the sum's error: every weight by its score's, the sum and the logarithm by 2^-16
    assert (np.abs(lse - want_lse)[~none] <= (2 * delta + 2.0 ** -16 * (1 + np.abs(want_lse)))[~none]).all()


SIGHTS = {
    "cap": lambda inst, H: dict(cap=20.0),
    "cap_below_scores": lambda inst, H: dict(cap=2.0),
    "large_cap": lambda inst, H: dict(cap=30000.0),
    "slopes": lambda inst, H: dict(slopes=slopes_of(H)),
    "window": lambda inst, H: dict(window=37),
    "window_of_one": lambda inst, H: dict(window=1),
    "window_of_2000": lambda inst, H: dict(window=2000),
    "wide_window": lambda inst, H: dict(window=100000),
    "documents": lambda inst, H: dict(first=documents(inst, 30)),
    "long_documents": lambda inst, H: dict(first=documents(inst, 300)),
    "prefix": lambda inst, H: dict(end=np.maximum(positions(inst) + 1, 50).astype(np.int32)),
    "all_see_all": lambda inst, H: dict(end=np.full(int(inst.n.sum()), 1 << 30, np.int32)),
    "everything": lambda inst, H: dict(cap=15.0, slopes=slopes_of(H), window=90, first=documents(inst, 200),
                                       end=(positions(inst) + 1 + np.arange(int(inst.n.sum())) % 40).astype(np.int32)),
}
# n, length, kv, q heads, dim, bt: steps of 16 and 32 rows, tiles of 128, split and whole
FORMS = {
    "step": ([1] * 5, [1, 33, 300, 700, 64], 2, 8, 64, 16),
    "step_long": ([1, 1], [5000, 1700], 1, 8, 128, 16),
    "few": ([4, 1, 3], [4, 90, 400], 2, 8, 128, 16),
    "few_32": ([4, 2], [60, 900], 1, 8, 64, 24),
    "tile": ([70, 1, 33], [70, 400, 600], 2, 4, 128, 16),
    "tile_64": ([50, 20], [700, 20], 1, 5, 64, 32),
    "tile_odd_pages": ([40, 9], [300, 150], 1, 8, 128, 7),
    "tile_odd_pages_64": ([60], [500], 2, 2, 64, 12),
    "tile_many_heads": ([5, 2], [200, 90], 1, 160, 64, 16),
    "prompt": ([260], [260], 1, 3, 128, 16),
    "tile_long": ([40, 3], [4700, 2300], 1, 4, 128, 16),
    "step_many": ([1] * 130, list(range(1, 131)), 1, 4, 64, 16),
    "few_many": ([1 + i % 3 for i in range(70)], [3 + 5 * i for i in range(70)], 1, 4, 64, 16),
    "tile_many": ([1] * 40 + [45] + [1] * 40, [2 + 3 * i for i in range(40)] + [1700] + [90] * 40, 2, 4, 64, 16),
}


@pytest.mark.parametrize("sight", SIGHTS)
@pytest.mark.parametrize("form", FORMS)
def test_against_definition(form, sight):
    n, length, kv, H, dim, bt = FORMS[form]
    dtype = F16 if len(form + sight) % 3 == 0 else BF16
    inst = R.instance(len(form) * 31 + len(sight), n, length, kv=kv, dim=dim, dtype=dtype, bt=bt)
    q = queries(inst, H, 8.0 if "cap" in sight else 2.5)
    compare(inst, q, dim ** -0.5, **SIGHTS[sight](inst, H))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("form", ["step", "few", "tile", "tile_odd_pages"])
def test_a_sight_that_says_nothing(form, dtype):
    """A window past every length: the plain call's result within the same bound, and a
    call with ranges that are the causal ones gives the same bits."""
    n, length, kv, H, dim, bt = FORMS[form]
    inst = R.instance(77, n, length, kv=kv, dim=dim, dtype=dtype, bt=bt)
    q = queries(inst, H)
    compare(inst, q, dim ** -0.5, window=1 << 31)
    a, la = run(inst, q, dim ** -0.5, window=1 << 31)
    b, lb = run(inst, q, dim ** -0.5, first=np.full(q.shape[0], -5, np.int32), end=(positions(inst) + 1).astype(np.int32))
    assert np.array_equal(a, b) and np.array_equal(la, lb)


@pytest.mark.parametrize("form", ["step", "few", "tile"])
def test_rows_that_see_nothing(form):
    """Some tokens' ranges are empty, upside down or outside: zeros, and no others change."""
    n, length, kv, H, dim, bt = FORMS[form]
    inst = R.instance(78, n, length, kv=kv, dim=dim, bt=bt)
    q = queries(inst, H)
    T = q.shape[0]
    first, end = np.zeros(T, np.int32), (positions(inst) + 1).astype(np.int32)
    whole, _ = run(inst, q, 0.1, first=first, end=end)
    f, e = first.copy(), end.copy()
    f[0], e[0] = 5, 5
    if T > 2:
        f[1], e[1] = 2 ** 31 - 1, 2 ** 31 - 1
        f[2], e[2] = 0, -2 ** 31
    if T > 4:
        f[4] = 100000
    compare(inst, q, 0.1, first=f, end=e)
    out, _ = run(inst, q, 0.1, first=f, end=e)
    empty = [0] + ([1, 2] if T > 2 else []) + ([4] if T > 4 else [])
    assert (out[empty] == 0).all()
    if form == "step":
        rest = np.setdiff1d(np.arange(T), empty)
        assert np.array_equal(out[rest], whole[rest])
    none = np.full(T, 1 << 30, np.int32)
    out, lse = run(inst, q, 0.1, first=none)
    assert (out == 0).all() and np.isneginf(lse).all()


def test_padding():
    """Tokens before position 0: zeros, whatever their ranges say."""
    inst = R.instance(79, [8, 40], [3, 20], kv=2, dim=64)
    q = queries(inst, 4)
    for kw in (dict(window=2), dict(first=np.zeros(48, np.int32), end=np.full(48, 9, np.int32)), dict(cap=5.0)):
        compare(inst, q, 0.125, **kw)


def test_unseen_pages_need_not_be_there():
    """Pages that no token's range reaches hold no page id: nothing is reported."""
    for n, length, kv, H, dim, bt in (([1, 1], [900, 500], 2, 8, 64, 16), ([40], [2000], 1, 8, 128, 16),
                                      ([40], [2000], 1, 8, 128, 12), ([40], [2000], 1, 8, 64, 12)):
        inst = R.instance(80, n, length, kv=kv, dim=dim, bt=bt)
        q = queries(inst, H)
        want = run(inst, q, 0.1, window=50)[0]
        for b in range(len(n)):
            p = inst.prog[b]
            first = max(0, length[b] - n[b] + 1 - 50)
            inst.tbl[inst.tbl_off[p]:inst.tbl_off[p] + first // bt] = R.NONE
            inst.tbl[inst.tbl_off[p] - (-length[b] // bt):inst.tbl_off[p + 1]] = R.NONE
        assert np.array_equal(run(inst, q, 0.1, window=50)[0], want)
        with pytest.raises(MoriError) as e:
            run(inst, q, 0.1, window=2000)
        assert e.value.detail == M.MORI_DEV_NOT_RESIDENT


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("form", ["step", "few", "tile", "tile_odd_pages", "prompt"])
def test_what_a_row_does_not_see_does_not_reach_it(form, bad):
    """Values and keys that are not finite, seen by some rows, by none, or by all."""
    n, length, kv, H, dim, bt = FORMS[form]
    for where, kw in (("before", dict(window=20)), ("after", dict(end=None)), ("between", dict(first=None))):
        inst = R.instance(81, n, length, kv=kv, dim=dim, bt=bt)
        q = queries(inst, H)
        pos = positions(inst)
        if where == "after":  # every token stops short of its own position by a few
            kw = dict(end=(pos - 2).astype(np.int32))
        if where == "between":
            kw = dict(first=documents(inst, 17))
        b = int(np.argmax(inst.length))
        L = int(inst.length[b])
        at = {"before": max(0, L - 21 - n[b] // 2), "after": L - 1, "between": L - n[b] // 2 - 1}[where]
        page, row = inst.slot(b, at)
        for plane in (0, 1):
            inst.pool[inst.layer, plane, page, row, :, 3 + plane] = bad
        out, _ = run(inst, q, 0.1, **kw)
        t0, m = int(inst.seq_off[b]), n[b]
        seen = np.zeros(q.shape[0], bool)
        for i in range(m):
            p = L - m + i
            lo = max(0, p + 1 - 20) if where == "before" else int(kw["first"][t0 + i]) if where == "between" else 0
            hi = int(kw["end"][t0 + i]) if where == "after" else p + 1
            seen[t0 + i] = lo <= at < hi
        assert not seen.all()
        page, row = inst.slot(b, at)
        for plane in (0, 1):
            inst.pool[inst.layer, plane, page, row, :, 3 + plane] = 0
        want, _, bound, _ = S.attend(inst, q, 0.1, **kw)
        assert (np.abs(out - want) <= bound)[~seen].all(), (where, np.argwhere(~(np.abs(out - want) <= bound)[~seen])[:4])


@pytest.mark.parametrize("window", range(5, 13))
@pytest.mark.parametrize("dim", [64, 128])
def test_first_key_inside_a_load(window, dim):
    """The tiles' kernel loads a page's rows a few at a time: those before the first key that
    is seen hold NaN, and so does what is behind the program's last row."""
    inst = R.instance(90, [1], [301], kv=1, dim=dim)
    for at in range(301 - window):
        page, row = inst.slot(0, at)
        inst.pool[1, :, page, row] = float("nan")
    compare(inst, queries(inst, 40), 0.1, window=window)
    compare(inst, queries(inst, 40), 0.1, first=np.array([301 - window], np.int32), slopes=slopes_of(40))


def test_more_tiles_than_are_split():
    """Enough tiles to fill the chip: each is one item, as the tiles' lines have them."""
    inst = R.instance(91, [900, 20, 700], [900, 400, 1500], kv=16, dim=64, bt=16)
    q = queries(inst, 48)
    assert (inst.n.sum() * 3 // 128 + 3) * 16 < 2048  # split: the other side of the rule, by the bits
    a = run(inst, q, 0.1, window=300)
    big = R.instance(91, [900, 20, 700] * 4, [900, 400, 1500] * 4, kv=16, dim=64, bt=16)
    big.pool = big.pool * 0
    assert (big.n.sum() * 3 // 128 + 12) * 16 >= 2048
    for b in range(12):  # the same programs four times
        for p in (0, 1):
            j = np.arange(int(big.length[b]))
            pages = big.tbl[big.tbl_off[big.prog[b]] + j // 16]
            big.pool[1, p, torch.from_numpy(pages), torch.from_numpy(j % 16)] = torch.from_numpy(inst.rows(p, b % 3, j.size)).bfloat16()
    out, lse = run(big, q.repeat(4, 1, 1), 0.1, window=300)
    T = q.shape[0]
    for i in range(4):
        # the two sum runs in other places: a rounding of the weights and of the result
        assert (np.abs(out[i * T:(i + 1) * T] - a[0]) <= 2.0 ** -7 * np.abs(a[0]) + 2.0 ** -8).all()
        assert np.allclose(lse[i * T:(i + 1) * T], a[1], atol=1e-4)
    t = np.array([0, 1, 31, 32, 899, 905, 950, 1619])
    for b, rows in ((0, t[t < 900]), (1, [900 + 5]), (2, [920 + 30, 1619])):
        L, n, k = int(inst.length[b]), int(inst.n[b]), [inst.rows(p, b, int(inst.length[b])) for p in (0, 1)]
        for r in rows:
            pos = L - n + int(r) - int(inst.seq_off[b])
            lo = max(0, pos - 299)
            for h in (0, 47):
                s = k[0][lo:pos + 1, h // 3] @ q[r, h].double().numpy() * 0.1
                w = np.exp(s - s.max())
                want = w @ k[1][lo:pos + 1, h // 3] / w.sum()
                assert (np.abs(out[int(r), h] - want) <= 2.0 ** -6).all()


def test_capped_infinities():
    """Infinite scores are the cap: what a key of 1000 gives (its score is 100, and tanh 20
    is 1 in 32 bits), with the same weights everywhere."""
    out = []
    for value in (float("inf"), 1000.0):
        inst = R.instance(82, [1, 30], [40, 60], kv=1, dim=64)
        q = queries(inst, 8)
        q[..., 5] = torch.where(q[..., 5] < 0, -1.0, 1.0).to(BF16)
        for b, at in ((0, 7), (1, 10)):
            page, row = inst.slot(b, at)
            inst.pool[1, 0, page, row, 0, :] = 0
            inst.pool[1, 0, page, row, 0, 5] = value
        out.append(run(inst, q, 0.1, cap=5.0)[0])
    assert np.array_equal(*out)
    want, _, bound, _ = S.attend(inst, q, 0.1, cap=5.0)
    assert (np.abs(out[0] - want) <= bound).all()


@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0])
def test_scales(scale):
    inst = R.instance(83, [1, 40], [300, 90], kv=2, dim=64)
    q = queries(inst, 4, 1.0)
    for kw in (dict(cap=3.0), dict(slopes=np.array([0.5, -0.01, 0.0, 1e-8], np.float32)), dict(window=30)):
        compare(inst, q, scale, **kw)


@pytest.mark.parametrize("form", ["step_long", "tile", "few"])
def test_repeats_and_workspaces(form):
    """The same bits every time, with a workspace given for any sight, dirty from others."""
    n, length, kv, H, dim, bt = FORMS[form]
    inst = R.instance(84, n, length, kv=kv, dim=dim, bt=bt)
    q, pool, b = queries(inst, H).cuda(), inst.pool.cuda(), R.batch(inst)
    ws = A.kv_attend_workspace(inst.geom, b, q, sight=True)
    ws.fill_(255)
    first = dev(documents(inst, 100))
    calls = [dict(cap=9.0), dict(window=64), dict(first=first), dict(slopes=dev(slopes_of(H)))]
    one = [A.kv_attend(pool, inst.geom, 1, b, q, scale=0.1, **kw) for kw in calls]
    for _ in range(3):
        for kw, want in zip(calls, one):
            assert torch.equal(A.kv_attend(pool, inst.geom, 1, b, q, scale=0.1, workspace=ws, **kw), want)
    b.check()


def test_graph_replays():
    """Ranges, lengths and slopes are read at replay."""
    inst = R.instance(85, [1, 20, 5], [200, 300, 50], kv=2, dim=64)
    q, pool, b = queries(inst, 8).cuda(), inst.pool.cuda(), R.batch(inst)
    ws = A.kv_attend_workspace(inst.geom, b, q, sight=True)
    first, slopes = torch.zeros(26, dtype=torch.int32, device="cuda"), torch.zeros(8, device="cuda")
    out = torch.empty_like(q)
    call = lambda o, w: A.kv_attend(pool, inst.geom, 1, b, q, scale=0.1, out=o, workspace=w, first=first, slopes=slopes, cap=8.0)
    call(out, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, ws)
    other = torch.empty_like(ws)
    for i in range(5):
        first.copy_(dev(documents(inst, 20 + 10 * i, seed=i)))
        slopes.copy_(dev(slopes_of(8) * i))
        graph.replay()
        want = torch.empty_like(q)
        call(want, other)
        torch.randn(10000, device="cuda").sum().item()
        assert torch.equal(out, want)
    b.check()


def test_strided_queries_and_outputs():
    inst = R.instance(86, [30, 1], [80, 200], kv=2, dim=64)
    big = torch.randn(31, 12, 64).to(BF16)
    o = torch.zeros(31, 8, 192, dtype=BF16, device="cuda")
    b = R.batch(inst)
    x = big.cuda()
    A.kv_attend(inst.pool.cuda(), inst.geom, 1, b, x[:, 2:10], scale=0.2, out=o[:, :, 64:128], window=25)
    want, _, bound, _ = S.attend(inst, big[:, 2:10], 0.2, window=25)
    assert (np.abs(o[:, :, 64:128].double().cpu().numpy() - want) <= bound).all()
    assert (o[:, :, :64] == 0).all() and (o[:, :, 128:] == 0).all()
    b.check()


def test_rows_behind_the_last_sequence():
    """More tokens than the sequences have: those rows are left as they were."""
    inst = R.instance(87, [40, 1], [80, 200], kv=2, dim=64)
    for n in ([40, 1], [1, 1]):
        inst.n = np.array(n)
        inst.seq_off = np.concatenate([[0], np.cumsum(n)])
        T = sum(n) + 6
        b = R.batch(inst, tokens=T)
        q = torch.randn(T, 4, 64, device="cuda").bfloat16()
        o = torch.full((T, 4, 64), 7.0, device="cuda", dtype=BF16)
        A.kv_attend(inst.pool.cuda(), inst.geom, 1, b, q, scale=0.2, out=o, cap=4.0, window=30)
        b.check()
        assert (o[-6:] == 7).all() and torch.isfinite(o).all()


def test_bad_batches():
    """Lengths past the bounds: the bit, zeros, and nothing read out of range."""
    inst = R.instance(88, [6, 3], [80, 200], kv=2, dim=64)
    inst.length[0] = 10 ** 6
    q = queries(inst, 4)
    for kw in (dict(window=10), dict(first=np.zeros(9, np.int32)), dict(end=np.full(9, 1 << 30, np.int32))):
        b = R.batch(inst, max_kv=300)
        k = {n: dev(x) if isinstance(x, np.ndarray) else x for n, x in kw.items()}
        out = A.kv_attend(inst.pool.cuda(), inst.geom, 1, b, q.cuda(), scale=0.2, **k)
        with pytest.raises(MoriError) as e:
            b.check()
        assert e.value.detail == M.MORI_DEV_BAD_TOKENS
        assert (out[:6] == 0).all() and torch.isfinite(out).all() and (out[6:] != 0).any()


@pytest.mark.parametrize("form", ["step_long", "few_many", "tile_long", "tile_many"])
def test_workspace_is_what_is_used(form):
    """Exactly the size asked for, with bytes behind it that stay as they are."""
    n, length, kv, H, dim, bt = FORMS[form]
    inst = R.instance(95, n, length, kv=kv, dim=dim, bt=bt)
    q, pool, b = queries(inst, H).cuda(), inst.pool.cuda(), R.batch(inst)
    size = A.kv_attend_workspace(inst.geom, b, q, sight=True).numel()
    guarded = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    for kw in (dict(cap=5.0), dict(window=900), dict(first=dev(documents(inst, 500)))):
        A.kv_attend(pool, inst.geom, 1, b, q, scale=0.1, workspace=guarded[:size], **kw)
        assert (guarded[size:] == 0x5A).all()
    b.check()


@pytest.mark.parametrize("n,H", [(40, 8), (1, 8)])
def test_overlapping_sequences_stay_inside_the_workspace(n, H):
    """Offsets that name tokens twice give more tiles and items than there is room for: the
    fault is reported, what is written stays in bounds."""
    inst = R.instance(96, [n] * 9, [3000] * 9, kv=1, dim=128)
    inst.seq_off = np.array([0, n, 0, n, 0, n, 0, n, 0, n])
    b = R.batch(inst, tokens=n)
    q = torch.randn(n, H, 128).to(BF16).cuda()
    size = A.kv_attend_workspace(inst.geom, b, q, sight=True).numel()
    guarded = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    for kw in (dict(cap=5.0), dict(window=2500), dict(end=torch.full((n,), 3000, dtype=torch.int32, device="cuda"))):
        A.kv_attend(inst.pool.cuda(), inst.geom, 1, b, q, scale=0.1, workspace=guarded[:size], **kw)
        torch.cuda.synchronize()
        assert int(b.error.item()) == M.MORI_DEV_BAD_TOKENS
        assert (guarded[size:] == 0x5A).all()


def test_overlap_of_calls():
    """Two calls of one batch on two streams, a workspace each, at once and again."""
    inst = R.instance(97, [60, 1, 1], [2000, 900, 1500], kv=2, dim=64)
    q, pool, b = queries(inst, 8).cuda(), inst.pool.cuda(), R.batch(inst)
    first = dev(documents(inst, 300))
    kws = [dict(window=700, cap=9.0), dict(first=first, slopes=dev(slopes_of(8)))]
    want = [A.kv_attend(pool, inst.geom, 1, b, q, scale=0.1, **kw) for kw in kws]
    ws = [A.kv_attend_workspace(inst.geom, b, q, sight=True) for _ in kws]
    out = [torch.empty_like(w) for w in want]
    streams = [torch.cuda.Stream() for _ in kws]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, kw, w, o in zip(streams, kws, ws, out):
            A.kv_attend(pool, inst.geom, 1, b, q, scale=0.1, workspace=w, out=o, stream=s, **kw)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(out, want))
    b.check()


def test_pages_behind_four_gigabytes():
    """A pool whose planes pass 2^32 bytes, the programs' pages at its end: the same bits as
    over a small one, appended with axes and attended to with a sight."""
    layers, bt, dim, blocks = 1, 16, 128, (1 << 20) + 3000
    for n, length, H in (([1, 3], [300, 900], 4), ([50, 20], [600, 300], 4)):
        inst = R.instance(98, n, length, kv=1, dim=dim, bt=bt, layers=1, layer=0)
        T = sum(n)
        x = torch.randn(T, H + 2, dim, device="cuda").bfloat16()
        at = torch.randint(0, 500, (3, T), device="cuda", dtype=torch.int32)
        rope, kw = A.rope_table(500, dim), dict(scale=0.1, cap=7.0, window=250, slopes=dev(slopes_of(H)))
        out = []
        for large in (False, True):
            if large:
                small = inst.pool
                inst.geom = R.Geom(layers, 2, bt, dim * 2, blocks)
                pool = torch.empty(1, 2, blocks, bt, 1, dim, dtype=BF16, device="cuda")
                shift = blocks - small.shape[2]
                pool[:, :, shift:] = small.cuda()
                inst.tbl = inst.tbl + shift
            else:
                pool = inst.pool.cuda()
            b = R.batch(inst)
            q = A.kv_append(pool, inst.geom, 0, b, x[:, H:H + 1], x[:, H + 1:], q=x[:, :H], rope=rope, positions=at,
                            sections=(16, 24, 24))
            out.append(A.kv_attend(pool, inst.geom, 0, b, q, **kw))
            b.check()
        assert torch.equal(*out) and torch.isfinite(out[0]).all()
        del pool
        torch.cuda.empty_cache()


# n, length, kv, q heads, dim, bt: tiles of which some or all have several runs
SPLIT = {
    "odd_pages": ([45, 3], [1900, 1111], 2, 6, 128, 7),
    "odd_pages_64": ([33], [2050], 3, 9, 64, 24),
    "many_runs": ([40], [20000], 1, 2, 64, 64),  # more than a wavefront has lanes
    "many_runs_128": ([17, 1], [17500, 300], 1, 8, 128, 16),
    "many_tiles": ([30] * 33, [900 + 37 * i for i in range(33)], 1, 9, 128, 16),
    "a_long_one": ([20] * 35 + [300], [20 + i for i in range(35)] + [2900], 1, 8, 128, 32),
    "last_rows": ([27, 43], [1500, 1501], 1, 5, 64, 16),  # tiles of 7 and 87 rows
}


@pytest.mark.parametrize("sight", ["cap", "slopes", "window_of_2000", "long_documents", "prefix", "everything"])
@pytest.mark.parametrize("form", SPLIT)
def test_split_tiles(form, sight):
    n, length, kv, H, dim, bt = SPLIT[form]
    inst = R.instance(len(form) * 7 + len(sight), n, length, kv=kv, dim=dim, dtype=F16 if len(form + sight) % 2 else BF16, bt=bt)
    compare(inst, queries(inst, H, 8.0 if "cap" in sight else 2.5), dim ** -0.5, **SIGHTS[sight](inst, H))


@pytest.mark.parametrize("window", [640, 730, 770, 900, 1030, 1300])
def test_windows_around_the_choice_to_split(window):
    for n, kv in ((40, 2), (600, 4)):  # few workgroups, and over 128
        inst = R.instance(window + n, [n] * 3, [window + n, 2500, n], kv=kv, dim=64, dtype=BF16, bt=16)
        compare(inst, queries(inst, 2 * kv), 0.125, window=window, slopes=slopes_of(2 * kv))


@pytest.mark.parametrize("sight", ["cap", "slopes", "window", "documents", "long_documents", "prefix", "everything"])
@pytest.mark.parametrize("seqs,kv,dim", [(70, 32, 64), (9, 128, 64), (40, 32, 128), (50, 64, 64)])
def test_whole_tiles_in_the_order_of_their_length(seqs, kv, dim, sight):
    """More workgroups than are split, of a few tiles; the longest run first."""
    g = np.random.default_rng(seqs)
    n = g.integers(0, 18, seqs).tolist()
    n[seqs // 2] = 17  # 34 rows or more
    length = [a + int(b) for a, b in zip(n, g.integers(0, 230, seqs))]
    length[0] = n[0]
    inst = R.instance(seqs + len(sight), n, length, kv=kv, dim=dim, dtype=F16 if len(sight) % 2 else BF16, bt=16)
    H = kv * (4 if kv < 64 else 2)
    assert (sum(n) * (H // kv) // 128 + seqs) * kv >= 1024
    compare(inst, queries(inst, H, 8.0 if "cap" in sight else 2.5), dim ** -0.5, **SIGHTS[sight](inst, H))


def test_whole_tiles_of_one_prompt():
    """Documents in a prompt whose tiles fill the chip many times."""
    inst = R.instance(5, [700], [760], kv=32, dim=64, dtype=BF16, bt=16)
    q = queries(inst, 64 * 6)
    compare(inst, q, 0.125, first=documents(inst, 90), slopes=slopes_of(64 * 6))
