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
