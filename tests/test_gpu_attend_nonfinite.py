"""Infinities and NaN that a row attends to come out as the definition has them, and
those that it does not attend to stay out, in every form of the attention kernels."""
import numpy as np
import pytest
import torch

import attend_ref as R

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
# query heads of one key head: decode steps of 16 and 32 rows, and the chunks' kernel
HEADS = {"step16": 4, "step32": 20, "chunk": 40}


def attend(inst, H, seed=0):
    from paper_2606_00866_amd import attention as A
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn(int(inst.n.sum()), H, inst.dim, generator=g) * 2.5).to(inst.dtype)
    scale = (192 if inst.geom.planes == 1 else inst.dim) ** -0.5
    b = R.batch(inst)
    out = A.kv_attend(inst.pool.cuda(), inst.geom, inst.layer, b, q.cuda(), scale=scale)
    b.check()
    return q, scale, out.double().cpu().numpy()


@pytest.mark.parametrize("bt", [16, 7, 1])
@pytest.mark.parametrize("length", [1, 2, 30, 31, 32, 33, 63, 64, 65, 95, 300])
@pytest.mark.parametrize("form", HEADS)
def test_last_value_infinite(form, length, bt):
    """A decode step whose newest value holds an infinity: that element of every head is the
    infinity (its weight is not 0), at any length, and the others are what they were."""
    H, D = HEADS[form], 128
    inst = R.instance(41, [1], [length], kv=1, dim=D, bt=bt)
    q, scale, plain = attend(inst, H)
    want, _, mean, delta, count, top = R.attend(inst, q, scale, D)
    page, row = inst.slot(0, length - 1)
    inst.pool[1, 1, page, row, 0, 5] = float("inf")
    inst.pool[1, 1, page, row, 0, 77] = -float("inf")
    _, _, out = attend(inst, H)
    assert (out[..., 5] == np.inf).all() and (out[..., 77] == -np.inf).all()
    rest = np.setdiff1d(np.arange(D), [5, 77])
    bound = R.attend_bound(inst.dtype, want, mean, delta, count, top)
    assert (np.abs(out - want) <= bound)[..., rest].all()
    assert np.array_equal(out[..., rest], plain[..., rest])


@pytest.mark.parametrize("planes,H,n", [(2, 5, 4), (2, 8, 4), (1, 8, 4), (1, 16, 4), (1, 32, 4), (2, 40, 3)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_later_tokens_do_not_reach_earlier_rows(planes, H, n, bad):
    """A few new tokens: rows of 20 and 32 (decode kernel), 32, 64 and 128 (latents), 120 (chunks)."""
    dim = 576 if planes == 1 else 128
    inst = R.instance(42, [n], [n + 45], kv=1, dim=dim, planes=planes)
    first = n // 2
    for plane in range(planes):
        page, row = inst.slot(0, 45 + first)
        inst.pool[1, plane, page, row, 0, 3 + plane] = bad
    q, scale, out = attend(inst, H)
    inst.length = inst.length - (n - first)  # the rows before it, over what they may see
    inst.n = np.array([first])
    inst.seq_off = np.array([0, first])
    want, _, mean, delta, count, top = R.attend(inst, q[:first], scale, 512 if planes == 1 else dim)
    assert (np.abs(out[:first] - want) <= R.attend_bound(inst.dtype, want, mean, delta, count, top)).all()
