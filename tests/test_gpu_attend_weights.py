"""kv_attend's weights over a wide range: keys far below one that draws most of the
weight, scores that keep rising, in every form of the attention kernels."""
import numpy as np
import pytest
import torch

import attend_ref as R

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16

# query heads, key heads, new tokens, latent: decode steps of 16 and 32 rows, chunks, latent
# rows of 16, 32, 64 and 128
FORMS = {"step16": (4, 1, 1, False), "step32": (20, 1, 1, False), "chunk": (4, 1, 20, False), "latent16": (16, 1, 1, True),
         "latent32": (20, 1, 1, True), "latent64": (40, 1, 1, True), "latent128": (100, 1, 1, True)}
SINK = 17.5  # the first key's score over the others', in nats: 2^25.2


def attend(inst, q, scale):
    from paper_2606_00866_amd import attention as A
    b = R.batch(inst)
    lse = torch.empty(q.shape[:2], device="cuda")
    out = A.kv_attend(inst.pool.cuda(), inst.geom, inst.layer, b, q.cuda(), scale=scale, lse=lse)
    b.check()
    return out, lse


def compare(inst, q, scale, heads):
    """No allowance for weights below the type's normal numbers: those here are above."""
    out, lse = attend(inst, q, scale)
    value = 512 if inst.geom.planes == 1 else inst.dim
    want, want_lse, mean, delta, _, _ = R.attend(inst, q[:, heads], scale, value)
    off = np.abs(out[:, heads].double().cpu().numpy() - want)
    bound = R.attend_bound(inst.dtype, want, mean, delta, 0, 0)
    assert (off <= bound).all(), f"off by {(off / bound).max():.3f} of the bound"
    lse_off = np.abs(lse[:, heads].double().cpu().numpy() - want_lse)
    assert (lse_off <= 2 * delta[..., 0] + 2.0 ** -16 + 2.0 ** -22 * np.abs(want_lse)).all()


def sunk(form, length, others=(), dtype=F16):
    """Sequences of which the first's first key outscores the others by SINK and has the value
    0, while theirs are hundreds: what the many small weights bring is all of the result."""
    H, kv, n, latent = FORMS[form]
    dim, rot = (576, 64) if latent else (64, 64)
    lengths = [length, *others]
    inst = R.instance(31, [n] + [1] * len(others), lengths, kv=kv, dim=dim, planes=1 if latent else 2, dtype=dtype)
    rng = np.random.default_rng(5)
    for b, L in enumerate(lengths):
        j = np.arange(L)
        entry = inst.tbl_off[inst.prog[b]] + j // 16
        at = torch.from_numpy(inst.tbl[entry]), torch.from_numpy(j % 16)
        score = torch.from_numpy(rng.uniform(-0.25, 0.25, (L, kv, rot)) / rot)
        value = torch.from_numpy(rng.uniform(300, 900, (L, kv, dim - rot if latent else dim)))
        if b == 0:
            score[0], value[0] = SINK / rot, 0
        row = torch.cat([value, score], -1) if latent else score
        inst.pool[1, 0, at[0], at[1]] = row.to(dtype)
        if not latent:
            inst.pool[1, 1, at[0], at[1]] = value.to(dtype)
    T = int(inst.n.sum())
    q = torch.zeros(T, H, dim, dtype=dtype)
    q[..., dim - rot:] = 1.0
    return inst, q, H


@pytest.mark.parametrize("form", ["step16", "chunk", "latent16", "latent128"])
def test_sum_of_small_weights_beside_a_large_one(form):
    """A batch so large that no context is split: 40000 weights of 2^-25 are added to one of 1,
    each below half a step of the sum that holds it."""
    inst, q, H = sunk(form, 40000, [1] * 2200, BF16)
    compare(inst, q, 1.0, slice(0, H, max(1, H // 2)))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("length", [250, 2000])
def test_small_weights_beside_a_large_one(form, length):
    inst, q, H = sunk(form, length)
    compare(inst, q, 1.0, slice(0, H, max(1, H // 3)))


@pytest.mark.parametrize("form", ["step16", "chunk", "latent16", "latent128"])
def test_small_weights_in_one_run(form):
    """A batch so large that no context is split: 40000 small weights meet the large one in
    the same sum."""
    inst, q, H = sunk(form, 40000, [1] * 2200)
    compare(inst, q, 1.0, slice(0, H, max(1, H // 2)))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("form", FORMS)
def test_rising_scores(form, dtype):
    """Every few keys a larger score than all before: the sums follow it each time."""
    H, kv, n, latent = FORMS[form]
    dim, rot = (576, 64) if latent else (64, 64)
    inst = R.instance(32, [n], [400], kv=kv, dim=dim, planes=1 if latent else 2, dtype=dtype)
    for j in range(400):
        page, row = inst.slot(0, j)
        inst.pool[1, 0, page, row, 0, dim - rot:] = 0.02 * j
    g = torch.Generator().manual_seed(3)
    q = torch.zeros(n, H, dim)
    q[..., dim - rot:] = torch.rand(n, H, rot, generator=g) + 0.5  # some rows rise faster than others
    compare(inst, q.to(dtype), 0.125, slice(0, H, max(1, H // 4)))
