"""Attention with a sight on both sides of the rules by which the host runs a batch: tiles
that are split or whole, listed or not.  What the rule takes is seen by the workspace."""
import numpy as np
import pytest
import torch

import attend_ref as R
import sight_ref as S
from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError
from test_gpu_sight import compare, dev, documents, positions, queries, run, slopes_of

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def how(inst, q, batch=None, **kw):
    """Tiles, workgroups, whether tiles have room for partial sums, whether for a list."""
    b = batch or R.batch(inst)
    k = {n: dev(x) if isinstance(x, np.ndarray) else x for n, x in kw.items()}
    sight = A._sight(inst.geom, b, q.shape[1], *(k.get(n) for n in ("cap", "slopes", "window", "first", "end")))
    rc, n = M.mori_kv_attend_sight_workspace(A._empty_pool(inst.geom), b.desc, A._attend_desc(inst.geom, q.cuda(), None), sight)
    assert rc == M.MORI_OK
    tiles = b.num_tokens * (q.shape[1] // inst.kv) // 128 + b.num_seqs
    split = n >= tiles * inst.kv * 128 * inst.dim * 4
    return tiles, tiles * inst.kv, split, split or n > tiles * 48


# ---- bounds of a batch that does not fit ---------------------------------------------

BAD = {
    "few_whole": ([40] * 3, 300, 1, 8, False),
    "many_whole": ([9] * 70, 400, 2, 8, False),
    "many_split": ([40] * 70, 900, 1, 8, True),
    "ordered": ([5] * 70, 300, 32, 256, False),
}


@pytest.mark.parametrize("bad", ["falls", "past"])
@pytest.mark.parametrize("form", BAD)
def test_bad_ranges_of_any_sequence_are_reported(form, bad):
    """Not the first sequence's: the bit, its rows left alone, the others as they are without it."""
    n, length, kv, H, split = BAD[form]
    inst = R.instance(3, n, [length + i for i in range(len(n))], kv=kv, dim=64)
    q = queries(inst, H)
    for at in sorted({len(n) - 1, len(n) // 2}):
        off = inst.seq_off.copy()
        if bad == "past":
            off[at + 1:] = 10 ** 6 + np.arange(len(n) - at)  # this one's end and all behind it
        else:
            off[at + 1:] = off[at] - 1 - np.arange(len(n) - at)
        for kw in (dict(cap=20.0), dict(first=documents(inst, 60)), dict(window=200)):
            keep, inst.seq_off = inst.seq_off, off
            b = R.batch(inst)
            inst.seq_off = keep
            if "window" not in kw:
                assert how(inst, q, b, **kw)[2] == split
            k = {m: dev(x) if isinstance(x, np.ndarray) else x for m, x in kw.items()}
            out = torch.full_like(q, 7.0).cuda()
            A.kv_attend(inst.pool.cuda(), inst.geom, inst.layer, b, q.cuda(), scale=0.1, out=out, **k)
            with pytest.raises(MoriError) as e:
                b.check()
            assert e.value.detail == M.MORI_DEV_BAD_TOKENS
            assert (out[int(keep[at]):] == 7).all()
            for s in {0, at - 1}:
                t = slice(int(keep[s]), int(keep[s + 1]))
                want, _, bound, _ = S.attend(alone(inst, s), q[t], 0.1, **{m: x[t] if m == "first" else x for m, x in kw.items()})
                assert (np.abs(out[t].double().cpu().numpy() - want) <= bound).all()


def alone(inst, b):
    """A batch of one of its sequences."""
    return R.Inst(inst.geom, inst.dtype, inst.kv, inst.dim, inst.n[b:b + 1], inst.length[b:b + 1], inst.prog[b:b + 1],
                  inst.tbl_off, inst.tbl, np.array([0, inst.n[b]]), inst.pool, inst.layer)


# ---- an empty batch -------------------------------------------------------------------

def test_an_empty_batch_lists_no_items():
    """Offsets and lengths of 0, as a growth that did not fit leaves them, where whole tiles are
    listed: every item names no tile, outputs stay."""
    inst = R.instance(4, [5] * 70, [300] * 70, kv=32, dim=64)
    q = queries(inst, 256).cuda()
    b = R.batch(inst)
    tiles, _, split, listed = how(inst, q, b, cap=5.0)
    assert listed and not split
    ws = torch.zeros(A.kv_attend_workspace(inst.geom, b, q, sight=True).numel(), dtype=torch.uint8, device="cuda")
    b.seq_off.zero_()
    b.kv_len.zero_()
    out = torch.full_like(q, 7.0)
    A.kv_attend(inst.pool.cuda(), inst.geom, 1, b, q, scale=0.1, out=out, workspace=ws, cap=5.0)
    b.check()
    assert (out == 7).all()
    assert (ws[48 * tiles:52 * tiles].view(torch.int32) == -1).all()


# ---- pages that no token sees ----------------------------------------------------------

GAPS = {
    "step": ([2, 1, 2], [900, 40, 700], 2, 8, 64, 16),
    "step_long": ([2], [6000], 1, 8, 128, 16),
    "few_32": ([4], [900], 1, 8, 64, 24),
    "tile": ([40], [700], 1, 4, 128, 16),
    "tile_split": ([40], [6000], 1, 4, 128, 16),
    "tile_odd_pages": ([40], [3000], 1, 8, 128, 7),
    "tile_64": ([40, 3], [5000, 900], 1, 4, 64, 32),
    "tile_large_pages": ([40], [4000], 1, 4, 128, 256),
}


@pytest.mark.parametrize("kw", [dict(), dict(cap=9.0), dict(slopes=True)], ids=["plain", "cap", "slopes"])
@pytest.mark.parametrize("form", GAPS)
def test_pages_between_ranges_need_not_be_there(form, kw):
    """Tokens of one sequence that see its first keys, and others that see its last: pages
    between have no id, or one past the pool.  Nothing is reported, and one that some token
    sees is."""
    n, length, kv, H, dim, bt = GAPS[form]
    inst = R.instance(5, n, length, kv=kv, dim=dim, bt=bt)
    q = queries(inst, H)
    kw = {m: slopes_of(H) if m == "slopes" else x for m, x in kw.items()}
    T, first, end = q.shape[0], [], []
    for m, L in zip(n, length):
        i = np.arange(m)
        first.append(np.where(i % 2, L - 20, 3))
        end.append(np.where(i % 2, L, 19))
    first, end = (np.concatenate(x).astype(np.int32) for x in (first, end))
    want, _, bound, _ = S.attend(inst, q, 0.1, first=first, end=end, **kw)
    b = int(np.argmax(length))
    p, L = int(inst.prog[b]), length[b]
    e0 = int(inst.tbl_off[p])
    lo, hi = -(-19 // bt), (L - 20) // bt  # blocks that nobody sees
    assert hi - lo >= 1
    good = inst.tbl.copy()
    for page in (R.NONE, inst.geom.num_blocks + 5):
        inst.tbl[e0 + lo:e0 + hi] = page
        assert (np.abs(run(inst, q, 0.1, first=first, end=end, **kw)[0] - want) <= bound).all()
        for block, seen in ((lo - 1, True), (hi, True), (lo, False)):
            inst.tbl = good.copy()
            inst.tbl[e0 + lo:e0 + hi] = R.NONE
            inst.tbl[e0 + block] = page
            if seen:
                with pytest.raises(MoriError) as e:
                    run(inst, q, 0.1, first=first, end=end, **kw)
                assert e.value.detail == (M.MORI_DEV_NOT_RESIDENT if page == R.NONE else M.MORI_DEV_PAGE_RANGE)
            else:
                run(inst, q, 0.1, first=first, end=end, **kw)
        inst.tbl = good.copy()


def test_pages_between_ranges_whose_stand_in_is_not_finite():
    """What an absent page's rows are taken from reaches nobody, NaN or not."""
    for form in ("step", "tile", "tile_odd_pages"):
        n, length, kv, H, dim, bt = GAPS[form]
        inst = R.instance(6, n, length, kv=kv, dim=dim, bt=bt)
        q = queries(inst, H)
        i = np.concatenate([np.arange(m) for m in n])
        L = np.repeat(length, n)
        first, end = np.where(i % 2, L - 20, 3).astype(np.int32), np.where(i % 2, L, 19).astype(np.int32)
        b = int(np.argmax(length))
        e0 = int(inst.tbl_off[inst.prog[b]])
        want, _, bound, _ = S.attend(inst, q, 0.1, first=first, end=end)
        inst.tbl[e0 - (-19 // bt):e0 + (length[b] - 20) // bt] = R.NONE
        if 0 not in inst.tbl:
            inst.pool[:, :, 0] = float("nan")
        out, _ = run(inst, q, 0.1, first=first, end=end)
        assert (np.abs(out - want) <= bound).all()


# ---- split and whole --------------------------------------------------------------------

def test_split_and_whole_tiles_of_the_same_programs():
    """Few workgroups, whose tiles are split, and four times as many, whose are not."""
    kw = dict(cap=20.0)
    inst = R.instance(91, [900, 20, 700], [900, 400, 1500], kv=16, dim=64, bt=16)
    q = queries(inst, 48)
    assert how(inst, q, **kw)[1:3] == (40 * 16, True)
    a = run(inst, q, 0.1, **kw)
    big = R.instance(91, [900, 20, 700] * 4, [900, 400, 1500] * 4, kv=16, dim=64, bt=16)
    for b in range(12):  # the same programs four times
        for p in (0, 1):
            j = np.arange(int(big.length[b]))
            pages = big.tbl[big.tbl_off[big.prog[b]] + j // 16]
            big.pool[1, p, torch.from_numpy(pages), torch.from_numpy(j % 16)] = torch.from_numpy(inst.rows(p, b % 3, j.size)).bfloat16()
    tiles, groups, split, listed = how(big, q.repeat(4, 1, 1), **kw)
    assert groups >= 2048 and not split and listed
    out, lse = run(big, q.repeat(4, 1, 1), 0.1, **kw)
    T = q.shape[0]
    rows = np.array([0, 1, 400, 899, 900, 919, 920, 1300, 1619])
    heads = [0, 23, 47]
    for t in rows:
        b = int(np.searchsorted(inst.seq_off, t, side="right")) - 1
        pos = int(inst.length[b] - inst.n[b] + t - inst.seq_off[b])
        for h in heads:
            k, v = (inst.rows(p, b, pos + 1)[:, h // 3] for p in (0, 1))
            s = 20.0 * np.tanh(k @ q[t, h].double().numpy() * 0.1 / 20.0)
            w = np.exp(s - s.max())
            top = s.max() + np.log(w.sum())
            w /= w.sum()
            # weights and results rounded to 16 bits, scores of about 8 to 2^-14
            bound = 2.0 ** -8 * 1.1 * (w @ np.abs(v) + np.abs(w @ v)) + 2.0 ** -10
            for o, l, at in ((a[0], a[1], t), *((out, lse, i * T + t) for i in range(4))):
                assert (np.abs(o[at, h] - w @ v) <= bound).all()
                assert abs(l[at, h] - top) <= 2.0 ** -10
    for i in range(1, 4):  # the same runs in other places: the same bits
        assert np.array_equal(out[i * T:(i + 1) * T], out[:T]) and np.array_equal(lse[i * T:(i + 1) * T], lse[:T])


@pytest.mark.parametrize("sight", ["cap", "slopes", "window", "documents"])
@pytest.mark.parametrize("seqs,kv,dim", [(18, 128, 64), (66, 32, 128), (40, 64, 128)])
def test_whole_tiles_in_the_order_of_their_length(seqs, kv, dim, sight):
    g = np.random.default_rng(seqs)
    n = g.integers(0, 18, seqs).tolist()
    n[seqs // 2] = 17  # 34 rows or more
    length = [a + int(b) for a, b in zip(n, g.integers(0, 230, seqs))]
    length[0] = n[0]
    inst = R.instance(seqs + len(sight), n, length, kv=kv, dim=dim, dtype=F16 if len(sight) % 2 else BF16, bt=16)
    H = kv * (4 if kv < 64 else 2)
    kw = {"cap": dict(cap=20.0), "slopes": dict(slopes=slopes_of(H)), "window": dict(window=37),
          "documents": dict(first=documents(inst, 30))}[sight]
    q = queries(inst, H, 8.0 if sight == "cap" else 2.5)
    _, groups, split, listed = how(inst, q, **kw)
    assert groups >= 2048 and not split and listed
    compare(inst, q, dim ** -0.5, **kw)


# workgroups of a batch, and the keys up to which windows' tiles stay whole there
BANDS = {"128": (8, 1024), "256": (16, 2560), "about_full": (24, 5120), "above": (40, 5120)}


@pytest.mark.parametrize("more", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("band", BANDS)
def test_windows_on_both_sides_of_the_choice_to_split(band, dim, more):
    kv, keys = BANDS[band]
    window = keys - 17 - (8 if dim == 64 else 4) + more  # with a tile's 17 tokens and a load's rows
    n = [17] * 16
    length = [17 + 5 * i for i in range(15)] + [window + 300]
    inst = R.instance(kv + window, n, length, kv=kv, dim=dim, dtype=BF16, bt=16, layers=1, layer=0)
    H = 2 * kv
    q = queries(inst, H)
    tiles, groups, split, _ = how(inst, q, window=window, slopes=slopes_of(H))
    assert {"128": 128 <= groups < 256, "256": 256 <= groups < 400, "about_full": 400 <= groups <= 640,
            "above": 640 < groups < 2048}[band]
    assert split == more
    compare(inst, q, dim ** -0.5, window=window, slopes=slopes_of(H))
