"""CPU-only checks of positions with several axes: pairs and axes, tables, refusals."""
import math

import pytest
import torch

from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError
from test_attention_checks import DIM, H, KV, T, append, batch, geometry, pool  # noqa: F401


def test_pair_axes():
    assert A.pair_axes((2, 1, 3)) == [0, 0, 1, 2, 2, 2]
    assert A.pair_axes((2, 2, 2), "turns") == [0, 1, 2, 0, 1, 2]
    assert A.pair_axes((4, 1, 2), "turns") == [0, 1, 2, 0, 0, 2, 0]
    assert A.pair_axes((3,), "turns") == [0, 0, 0]
    assert A.pair_axes((24, 20, 20), "turns").count(1) == 20


@pytest.mark.parametrize("sections,order", [((1, 5, 1), "turns"), ((0, 2), "turns"), ((1, 2, 3, 4, 5), "blocks"), ((), "blocks"),
                                            ((-1, 3), "blocks"), ((1.5, 2.5), "blocks"), ((4, 4), "rows")])
def test_sections_that_do_not_fit(sections, order):
    with pytest.raises(MoriError):
        A.pair_axes(sections, order)


def test_tables():
    t = A.rope_table(50, 32, 100.0, device="cpu", restart=(4, 12))
    for p in (0, 3, 49):
        for i in range(16):
            a = p * (100.0 ** (-2 * i / 8) if i < 4 else 100.0 ** (-2 * (i - 4) / 24))
            assert abs(t[p, i].item() - math.cos(a)) < 2 ** -23 and abs(t[p, 16 + i].item() - math.sin(a)) < 2 ** -23
    assert torch.equal(A.rope_table(50, 32, device="cpu"), A.rope_table(50, 32, device="cpu", restart=(16,)))
    with pytest.raises(MoriError):
        A.rope_table(5, 32, device="cpu", restart=(4, 11))


@pytest.fixture
def axes_calls(monkeypatch):
    seen = []
    monkeypatch.setattr(M, "mori_kv_append", lambda *a, **k: seen.append(("append", a)) or M.MORI_OK)
    monkeypatch.setattr(M, "mori_kv_append_axes", lambda *a, **k: seen.append(("axes", a)) or M.MORI_OK)
    monkeypatch.setattr(A, "_stream_of", lambda *a, **k: 0)
    monkeypatch.setattr(A, "_current_device", lambda: 0, raising=False)
    return seen


def given(**kw):
    return {**dict(rope=torch.zeros(30, 64), positions=torch.zeros(3, T, dtype=torch.int32), sections=(8, 12, 12)), **kw}


def test_what_fits_is_called(axes_calls):
    append(**given())
    append(**given(sections=[12, 10, 10], order="turns"))
    append(**given(positions=torch.zeros(1, T, dtype=torch.int32), sections=(32,)))
    append(**given(positions=torch.zeros(3, 2 * T, dtype=torch.int32)[:, :T]))
    append(rope=torch.zeros(30, 64))
    assert [n for n, _ in axes_calls] == ["axes"] * 4 + ["append"]
    x = axes_calls[1][1][4]
    assert (x.num_axes, x.order, list(x.sections), x.axis_stride) == (3, M.MORI_AXES_TURNS, [12, 10, 10, 0], T)
    assert axes_calls[3][1][4].axis_stride == 2 * T


@pytest.mark.parametrize("bad", [
    dict(positions=None), dict(sections=None), dict(positions=torch.zeros(3, T)), dict(positions=torch.zeros(T, dtype=torch.int32)),
    dict(positions=torch.zeros(3, T + 1, dtype=torch.int32)), dict(positions=torch.zeros(5, T, dtype=torch.int32)),
    dict(positions=torch.zeros(T, 3, dtype=torch.int32).t()), dict(positions=torch.zeros(1, T, dtype=torch.int32).expand(3, T)),
    dict(positions=torch.zeros(3, T, dtype=torch.int32, device="meta")), dict(sections=(8, 12)), dict(sections=(8, 12, 11)),
    dict(order="rows"), dict(rope=None), dict(sections=(1, 1, 30), order="turns")], ids=str)
def test_refused(axes_calls, bad):
    with pytest.raises(MoriError) as e:
        append(**given(**bad))
    assert e.value.code == M.MORI_EINVAL and not axes_calls


POOL = dict(layers=2, planes=2, block_tokens=16, row_bytes=KV * DIM * 2, num_blocks=8, base=4096)
TOKENS = dict(num_seqs=1, num_tokens=4, max_new=4, max_kv=40, seq_off=4096, kv_len=4096, num_programs=1, tbl_len=8,
              tbl_off=4096, tbl=4096)
AXES = dict(num_axes=3, order=0, at=4096, axis_stride=4)


@pytest.mark.parametrize("bad", [
    dict(num_axes=0), dict(num_axes=5), dict(order=2), dict(at=None), dict(at=4098), dict(axis_stride=3), dict(s=(8, 12, 11, 0)),
    dict(s=(8, 12, 11, 1)), dict(s=(2, 15, 15, 0), order=1), dict(s=(2 ** 31, 2 ** 31, 32, 0)), dict(rot=0), dict(rot=32)], ids=str)
def test_refused_by_the_library(bad):
    rows = lambda: M.mori_rows(4096, 64, 64)
    a = M.mori_append(M.MORI_DT_BF16, KV, DIM, 0, bad.get("rot", 64), 0, 30, 4096, rows(), rows())
    x = M.mori_axes(**{**AXES, **{k: v for k, v in bad.items() if k not in ("s", "rot")}})
    x.sections[:] = bad.get("s", (8, 12, 12, 0))
    assert M.mori_kv_append_axes(M.mori_pool(**POOL), 0, M.mori_tokens(**TOKENS), a, x) == M.MORI_EINVAL


def test_no_axes_are_refused():
    import ctypes as C
    a = M.mori_append(M.MORI_DT_BF16, KV, DIM, 0, 64, 0, 30, 4096)
    assert M.lib().mori_kv_append_axes(C.byref(M.mori_pool(**POOL)), 0, C.byref(M.mori_tokens(**TOKENS)), C.byref(a), None,
                                       None, None) == M.MORI_EINVAL
