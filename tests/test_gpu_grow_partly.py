"""Growth that rewrites some of the arrays in place and writes the others elsewhere: every
array, whole, for each such choice, in one workgroup's pool and in a larger one."""
import numpy as np
import pytest
import torch

import grow_ref as R
from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError
from test_gpu_grow import arrays, dev, same

pytestmark = pytest.mark.gpu
NAMES = ("tbl_off", "tbl", "free", "held")


def growth(s, in_place, **bounds):
    x = dict(tbl_off=dev(s.tbl_off), tbl=dev(s.tbl), free=dev(s.free, np.uint8), held=dev(s.held))
    into = []
    for i, n in enumerate(NAMES):  # entries past the tables are left alone: as the plain form has them
        into.append(x[n] if in_place >> i & 1 else x[n].clone() if n == "tbl" else torch.full_like(x[n], 77))
    g = A.TokenGrowth(s.geom, x["tbl_off"], x["tbl"], x["free"], x["held"], dev(s.new), dev(s.prog), tier=dev(s.tier, np.uint8),
                      into=tuple(into), **{**dict(num_tokens=s.T, max_new=s.max_new, max_kv=s.max_kv), **bounds})
    g.state, g.before = tuple(into), x
    return g


def check(g, s, want, in_place):
    same(arrays(g), want)
    for i, n in enumerate(NAMES):
        if not in_place >> i & 1:
            assert np.array_equal(g.before[n].cpu().numpy(), getattr(s, n)), n


@pytest.mark.parametrize("form", ["small", "large", "most"])
@pytest.mark.parametrize("in_place", range(1, 15))
def test_against_definition(in_place, form):
    kw = {"small": dict(held=60), "large": dict(held=900, spare_pages=17000, bt=4), "most": dict(bt=8, held=60)}[form]
    programs, seqs, new = {"small": (20, 12, (0, 40)), "large": (60, 40, (0, 300)), "most": (2000, 1500, (0, 9))}[form]
    s = R.instance(in_place, programs, seqs, new, **kw)
    g = growth(s, in_place)
    g.run()
    check(g, s, R.grow(s), in_place)
    g.batch.check()


@pytest.mark.parametrize("pages", [40, 17000])
@pytest.mark.parametrize("in_place", range(1, 15))
def test_what_does_not_fit_changes_nothing(in_place, pages):
    s = R.instance(40 + in_place, 25, 12, (60, 90), held=100, spare_blocks=0, spare_pages=pages)
    g = growth(s, in_place, max_new=59)
    g.run()
    check(g, s, R.refused(s), in_place)
    with pytest.raises(MoriError) as e:
        g.batch.check()
    assert e.value.detail == M.MORI_DEV_BAD_TOKENS
