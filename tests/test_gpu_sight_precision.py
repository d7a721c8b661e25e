"""Steps with a sight: weights keep 16 bits (fp16 22), and values that are not finite give
what the definition gives."""
import numpy as np
import pytest
import torch

import attend_ref as R
import sight_ref as S
from test_gpu_sight import queries, run, slopes_of

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16
STEPS = {
    "one": ([1] * 24, list(range(2, 50, 2)), 2, 8, 64, 16),
    "one_128": ([1] * 6, [3, 9, 20, 40, 70, 130], 2, 8, 128, 16),
    "few_32": ([4, 2, 3], [8, 30, 60], 2, 16, 128, 16),
    "few_32_64": ([4, 2, 3], [8, 30, 60], 2, 16, 64, 7),
    "split": ([1, 1], [3000, 1700], 1, 8, 128, 16),
}
# a weight is two 16-bit numbers: the second is off by half a step of what is at most half a step of the first
PAIR = {t: r * r for t, r in R.ROUND.items()}


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("sight", ["cap", "slopes", "window"])
@pytest.mark.parametrize("form", STEPS)
def test_weights(form, sight, dtype):
    n, length, kv, H, dim, bt = STEPS[form]
    inst = R.instance(len(form), n, length, kv=kv, dim=dim, dtype=dtype, bt=bt)
    q = queries(inst, H, 0.3)
    kw = {"cap": dict(cap=20.0), "slopes": dict(slopes=slopes_of(H) / 8), "window": dict(window=1 << 20)}[sight]
    out, _ = run(inst, q, dim ** -0.5, **kw)
    want, _, _, delta = S.attend(inst, q, dim ** -0.5, **kw)
    sizes = inst.pool.clone()
    sizes[:, 1] = sizes[:, 1].abs()
    mean, *_ = S.attend(R.Inst(**{**inst.__dict__, "pool": sizes}), q, dim ** -0.5, **kw)  # of the values' sizes
    top, count = np.nanmax(sizes[inst.layer, 1].double().numpy()), max(length)
    # as attend_ref.attend_bound but for the weights' rounding
    weights = PAIR[dtype] * 1.01 + 2 * np.expm1(2 * delta[..., None]) + 2.0 ** -16
    bound = weights * mean + R.ROUND[dtype] * (np.abs(want) + weights * mean) + R.TINY[dtype] * (count * top + 1)
    bad = ~(np.abs(out - want) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:3], np.abs(out - want)[bad][:3], bound[bad][:3])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("form", STEPS)
def test_values_that_are_not_finite(form, value, dtype):
    """Seen by every token of a sequence, or by some: infinite in that element where it is the
    only such value, NaN where both infinities or a NaN meet, and no other element touched."""
    n, length, kv, H, dim, bt = STEPS[form]
    inst = R.instance(len(form), n, length, kv=kv, dim=dim, dtype=dtype, bt=bt)
    q = queries(inst, H, 0.3)
    for b in range(len(n)):
        for at in {0, length[b] // 2, length[b] - 1}:
            page, row = inst.slot(b, at)
            inst.pool[inst.layer, 1, page, row, :, 5 + at % 2] = value
    page, row = inst.slot(0, 1)
    inst.pool[inst.layer, 1, page, row, :, 9] = float("inf")
    page, row = inst.slot(0, 0)
    inst.pool[inst.layer, 1, page, row, :, 9] = -float("inf")
    for kw in (dict(cap=20.0), dict(window=1 << 20), dict(slopes=slopes_of(H) / 64)):
        out, _ = run(inst, q, dim ** -0.5, **kw)
        with np.errstate(invalid="ignore"):
            want, _, bound, _ = S.attend(inst, q, dim ** -0.5, **kw)
        finite = np.isfinite(want)
        assert finite.any() and not finite.all()
        same = lambda f: np.array_equal(f(out), f(want))
        assert same(np.isnan) and same(np.isposinf) and same(np.isneginf)
        clean = R.Inst(**{**inst.__dict__, "pool": torch.where(torch.isfinite(inst.pool), inst.pool, 0)})
        want, _, bound, _ = S.attend(clean, q, dim ** -0.5, **kw)
        assert (np.abs(out - want) <= bound)[finite].all()


def test_the_same_bits_with_ranges_that_say_nothing():
    """What is seen is the same however it is said."""
    n, length, kv, H, dim, bt = STEPS["few_32"]
    inst = R.instance(3, n, length, kv=kv, dim=dim, bt=bt)
    q = queries(inst, H)
    T = q.shape[0]
    a = run(inst, q, 0.1, window=1 << 31)
    b = run(inst, q, 0.1, first=np.full(T, -7, np.int32))
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
