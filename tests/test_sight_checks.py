"""CPU-only checks of attention with caps, biases, windows and ranges: what the library
and the Python entry point refuse, workspaces, and the plain definition on worked rows."""
import ctypes as C

import numpy as np
import pytest
import torch

import attend_ref as R
import sight_ref as S
from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError
from test_attention_checks import H, T, attend, batch, geometry, pool  # noqa: F401

POOL = dict(layers=2, planes=2, block_tokens=16, row_bytes=256, num_blocks=64, base=4096)
TOKENS = dict(num_seqs=2, num_tokens=90, max_new=80, max_kv=900, seq_off=4096, kv_len=4096, num_programs=2, tbl_len=64,
              tbl_off=4096, tbl=4096)


def desc(**kw):
    rows = lambda: M.mori_rows(4096, 256, 64)
    return M.mori_attend(**{**dict(dtype=M.MORI_DT_BF16, q_heads=4, kv_heads=2, head_dim=64, value_dim=64, scale=0.1,
                                   q=rows(), out=rows()), **kw})


def size(sight, tokens=None, pool_=None, attend_=None):
    return M.mori_kv_attend_sight_workspace(M.mori_pool(**{**POOL, **(pool_ or {})}), M.mori_tokens(**{**TOKENS, **(tokens or {})}),
                                            attend_ or desc(), M.mori_sight(**sight))


@pytest.mark.parametrize("bad", [dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=-1.0), dict(cap=1e-45),
                                 dict(cap=3.0e38), dict(slopes=4098), dict(first=4097), dict(end=4099)], ids=str)
def test_refused_by_the_library(bad):
    assert size(bad)[0] == M.MORI_EINVAL
    assert M.mori_kv_attend_sight(M.mori_pool(**POOL), 0, M.mori_tokens(**TOKENS), desc(), M.mori_sight(**bad), 4096,
                                  1 << 40) == M.MORI_EINVAL


def test_latent_pools_and_no_sight_are_refused():
    latent = dict(planes=1, row_bytes=1152)
    a = desc(kv_heads=1, head_dim=576, value_dim=512)
    assert M.mori_kv_attend_workspace(M.mori_pool(**{**POOL, **latent}), M.mori_tokens(**TOKENS), a)[0] == M.MORI_OK
    assert size(dict(window=5), pool_=latent, attend_=a)[0] == M.MORI_EINVAL
    p, t, n = M.mori_pool(**POOL), M.mori_tokens(**TOKENS), C.c_uint64()
    assert M.lib().mori_kv_attend_sight_workspace(C.byref(p), C.byref(t), C.byref(desc()), None, C.byref(n)) == M.MORI_EINVAL
    assert M.lib().mori_kv_attend_sight(C.byref(p), 0, C.byref(t), C.byref(desc()), None, 4096, 1 << 40, None, None) == M.MORI_EINVAL


@pytest.mark.parametrize("tokens", [dict(), dict(max_new=1, num_tokens=2), dict(max_kv=10 ** 6), dict(num_tokens=30000, max_new=29000),
                                    dict(num_tokens=4000, num_seqs=4000, max_new=1)], ids=str)
def test_workspaces(tokens):
    """One made without a window holds every other's; a short one is refused."""
    rc, most = size(dict(), tokens)
    assert rc == M.MORI_OK
    for s in (dict(window=1), dict(window=100), dict(window=2 ** 32 - 1), dict(cap=5.0), dict(first=4096), dict(end=4096, window=7)):
        rc, n = size(s, tokens)
        assert rc == M.MORI_OK and n <= most
        if n:
            p, t = M.mori_pool(**POOL), M.mori_tokens(**{**TOKENS, **tokens})
            for ws, short in ((4096, n - 1), (0, n), (4096 + 16, n)):
                assert M.mori_kv_attend_sight(p, 0, t, desc(), M.mori_sight(**s), ws, short) == M.MORI_EINVAL


@pytest.fixture
def calls(monkeypatch):
    seen = []
    monkeypatch.setattr(M, "mori_kv_attend", lambda *a, **k: seen.append(("plain", a)) or M.MORI_OK)
    monkeypatch.setattr(M, "mori_kv_attend_sight", lambda *a, **k: seen.append(("sight", a)) or M.MORI_OK)
    monkeypatch.setattr(M, "mori_kv_attend_workspace", lambda *a, **k: (M.MORI_OK, 512))
    monkeypatch.setattr(M, "mori_kv_attend_sight_workspace", lambda *a, **k: (M.MORI_OK, 768))
    monkeypatch.setattr(A, "_stream_of", lambda *a, **k: 0)
    monkeypatch.setattr(A, "_current_device", lambda: 0, raising=False)
    return seen


def ints(n=T, **kw):
    return torch.zeros(n, dtype=torch.int32, **kw)


def test_what_fits_is_called(calls):
    attend()
    for kw in (dict(cap=5.0), dict(slopes=torch.zeros(H)), dict(window=4), dict(first=ints()), dict(end=ints()),
               dict(cap=1.0, window=2 ** 32 - 1, first=ints(), end=ints(), slopes=torch.ones(H))):
        attend(**kw)
    assert [n for n, _ in calls] == ["plain"] + ["sight"] * 6
    s = calls[-1][1][4]
    assert (s.cap, s.window) == (1.0, 2 ** 32 - 1) and s.first and s.end and s.slopes and calls[-1][1][6] == 768
    q = torch.zeros(T, H, 64, dtype=torch.bfloat16)
    assert A.kv_attend_workspace(geometry(), batch(), q).nbytes == 512
    assert A.kv_attend_workspace(geometry(), batch(), q, sight=True).nbytes == 768


@pytest.mark.parametrize("bad", [
    dict(cap=0.0), dict(cap=-1.0), dict(cap=float("inf")), dict(cap=float("nan")), dict(window=0), dict(window=-3),
    dict(window=2 ** 32), dict(slopes=torch.zeros(H + 1)), dict(slopes=torch.zeros(H).double()), dict(slopes=torch.zeros(1, H)),
    dict(slopes=torch.zeros(2 * H)[::2]), dict(first=ints(T + 1)), dict(first=ints().long()), dict(end=ints(2 * T)[::2]),
    dict(end=ints(device="meta")), dict(slopes=torch.zeros(H, requires_grad=True))], ids=str)
def test_refused(calls, bad):
    with pytest.raises(MoriError) as e:
        attend(**bad)
    assert e.value.code == M.MORI_EINVAL and not calls


def test_latent_pools(calls):
    with pytest.raises(MoriError):
        g = geometry(planes=1, row_bytes=1152)
        p = torch.zeros(2, 1, 8, 16, 576, dtype=torch.bfloat16)
        A.kv_attend(p, g, 0, batch(planes=1, row_bytes=1152), torch.zeros(T, H, 576, dtype=torch.bfloat16), scale=0.1, window=4)
    assert not calls


def test_definition():
    """Against masks over all keys in torch, in 64 bits."""
    inst = R.instance(1, [4, 1], [9, 6], kv=2, dim=8)
    q = torch.randn(5, 4, 8).to(inst.dtype)
    first, end = np.array([0, 3, 8, 2, 1], np.int32), np.array([6, 9, 8, 30, 5], np.int32)
    slopes = np.array([0.5, -0.1, 0.0, 2.0])
    for kw in (dict(), dict(cap=1.5), dict(slopes=slopes), dict(window=3), dict(first=first), dict(end=end),
               dict(cap=0.7, slopes=slopes, window=5, first=first, end=end)):
        out, lse, bound, _ = S.attend(inst, q, 0.4, **kw)
        for b, (n, L) in enumerate(((4, 9), (1, 6))):
            k, v = (torch.from_numpy(inst.rows(p, b, L)) for p in (0, 1))
            t = torch.arange(n) + int(inst.seq_off[b])
            pos, at = torch.arange(L - n, L), torch.arange(L)
            s = torch.einsum("thd,lhd->htl", q[t].double(), k.repeat_interleave(2, 1)) * 0.4
            if "cap" in kw:
                s = kw["cap"] * torch.tanh(s / kw["cap"])
            if "slopes" in kw:
                s = s - torch.from_numpy(slopes)[:, None, None] * (pos[:, None] - at).abs()
            lo = torch.maximum(pos + 1 - kw.get("window", 100), torch.from_numpy(kw["first"])[t] if "first" in kw else pos * 0)
            hi = torch.from_numpy(kw["end"])[t] if "end" in kw else pos + 1
            seen = (at >= lo[:, None]) & (at < hi[:, None])
            s = s.masked_fill(~seen, -float("inf"))
            want = torch.einsum("htl,lhd->thd", torch.softmax(s, -1).nan_to_num(0), v.repeat_interleave(2, 1))
            assert np.allclose(out[t], want, atol=1e-12) and np.allclose(lse[t], s.logsumexp(-1).t(), atol=1e-12)
        assert (bound > 0).all() and (bound < 0.3).all()


@pytest.mark.parametrize("bad", [dict(cap=1e-50), dict(cap=2.0 ** -150), dict(window=0.5), dict(window=4.5),
                                 dict(window=float("nan"))], ids=str)
def test_numbers_that_would_be_rounded_away_are_refused(calls, bad):
    """As 32 bits, or cut to an integer, they would say nothing, or something else."""
    with pytest.raises(MoriError) as e:
        attend(**bad)
    assert e.value.code == M.MORI_EINVAL and not calls


def test_a_workspace_for_no_sight_holds_all():
    """Whether tiles are split depends on the window and the ranges too."""
    g = np.random.default_rng(1)
    for _ in range(3000):
        B, kv = int(g.integers(1, 80)), int(2 ** g.integers(0, 4))
        T = int(B * 2 ** g.uniform(0, 11))
        tokens = dict(num_seqs=B, num_tokens=T, max_new=int(g.integers(-(-T // B), T + 1)), num_programs=B,
                      max_kv=int(2 ** g.uniform(0, 16)))
        tokens["max_new"] = min(tokens["max_new"], tokens["max_kv"])
        a = desc(q_heads=kv * int(g.integers(1, 9)), kv_heads=kv)
        pool_ = dict(row_bytes=128 * kv)
        rc, most = size(dict(), tokens, pool_, a)
        if rc != M.MORI_OK:
            continue
        for more in (dict(), dict(first=4096), dict(end=4096), dict(cap=3.0), dict(slopes=4096)):
            for window in (0, 1, int(2 ** g.uniform(0, 13)), 700, 2000, 5000):
                rc, n = size(dict(window=window, **more), tokens, pool_, a)
                assert rc == M.MORI_OK and n <= most, (tokens, kv, more, window, n, most)
