"""CPU-only checks of the Python entry points of the token operators: what does not
fit raises before the library is called.  The batch is made without its device
checks, on host tensors; the library's calls are replaced, so no address is used."""
import dataclasses

import pytest
import torch

from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError, PoolGeometry

BF16, F16 = torch.bfloat16, torch.float16
KV, DIM, H, T = 2, 64, 4, 3
GEOM = dict(layers=2, planes=2, block_tokens=16, row_bytes=KV * DIM * 2, num_blocks=8)


def geometry(**kw):
    return PoolGeometry(**{**GEOM, **kw})


@pytest.fixture
def calls(monkeypatch):
    """What reaches the library: a list of (name, arguments)."""
    seen = []
    monkeypatch.setattr(M, "mori_kv_append", lambda *a, **k: seen.append(("append", a)) or M.MORI_OK)
    monkeypatch.setattr(M, "mori_kv_attend", lambda *a, **k: seen.append(("attend", a)) or M.MORI_OK)
    monkeypatch.setattr(M, "mori_kv_attend_workspace", lambda *a, **k: (M.MORI_OK, 512))
    monkeypatch.setattr(A, "_stream_of", lambda *a, **k: 0)
    monkeypatch.setattr(A, "_current_device", lambda: 0, raising=False)
    return seen


def batch(**kw):
    b = object.__new__(A.TokenBatch)
    b.geom, b.num_seqs, b.num_tokens = geometry(**kw), 1, T
    b.shape, b.pool_bytes = dataclasses.astuple(b.geom), b.geom.pool_bytes
    b.device, b.index, b.error = torch.device("cpu"), 0, torch.zeros(1, dtype=torch.int32)
    b.desc = M.mori_tokens(num_seqs=1, num_tokens=T, max_new=T, max_kv=40)
    return b


def pool(dtype=BF16, device="cpu"):
    return torch.zeros(2, 2, 8, 16, KV, DIM, dtype=BF16, device=device).view(dtype)


def append(p=None, geom=None, b=None, dtype=BF16, **kw):
    k = torch.zeros(T, KV, DIM, dtype=dtype)
    return A.kv_append(pool() if p is None else p, geom or geometry(), 0, b or batch(), k, k.clone(), **kw)


def attend(p=None, geom=None, b=None, dtype=BF16, **kw):
    q = torch.zeros(T, H, DIM, dtype=dtype)
    return A.kv_attend(pool() if p is None else p, geom or geometry(), 0, b or batch(), q, **kw)


def refused(call, calls, **kw):
    with pytest.raises(MoriError) as e:
        call(**kw)
    assert e.value.code == M.MORI_EINVAL and not calls


def test_what_fits_is_called(calls):
    for p in (pool(), pool(torch.uint8), pool(torch.int16)):
        append(p=p)
        attend(p=p)
        attend(p=p, workspace=torch.empty(512, dtype=torch.uint8))
    assert [n for n, _ in calls] == ["append", "attend", "attend"] * 3
    attend(workspace=torch.empty(128, dtype=torch.float32))
    assert calls[-1][1][5] == 512  # bytes, whatever the type


def test_workspace(calls):
    """Somewhere else than the batch, or not one piece."""
    for w in (torch.empty(512, dtype=torch.uint8, device="meta"), torch.empty(1024, dtype=torch.uint8)[::2],
              torch.empty(16, 64, dtype=torch.uint8).t()):
        refused(attend, calls, workspace=w)


@pytest.mark.parametrize("call", [append, attend])
def test_pool(calls, call):
    """On another device than the batch, of the other 16-bit type, of another size."""
    refused(call, calls, p=pool(device="meta"))
    for dtype, other in ((F16, BF16), (BF16, F16)):
        refused(call, calls, p=pool(other), dtype=dtype)
    refused(call, calls, p=pool(torch.float32))
    refused(call, calls, p=pool()[:1])


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("change", [dict(block_tokens=32, num_blocks=4), dict(block_tokens=8, num_blocks=16),
                                    dict(layers=1, num_blocks=16), dict(layers=4, planes=1)])
def test_geometry_of_the_batch(calls, call, change):
    """Another division of the same bytes: the batch's tables do not speak of it."""
    assert geometry(**change).pool_bytes == geometry().pool_bytes
    refused(call, calls, geom=geometry(**change))
    refused(call, calls, b=batch(**change))


def test_geometry_of_the_workspace(calls):
    q = torch.zeros(T, H, DIM, dtype=BF16)
    assert A.kv_attend_workspace(geometry(), batch(), q).numel() == 512
    with pytest.raises(MoriError):
        A.kv_attend_workspace(geometry(block_tokens=32, num_blocks=4), batch(), q)


def test_inputs_elsewhere(calls):
    k = torch.zeros(T, KV, DIM, dtype=BF16)
    for kk, vv, kw in ((k.to("meta"), k, {}), (k, k.to("meta"), {}), (k, k, dict(q=k.to("meta"))),
                       (k, k, dict(q=k, q_out=k.to("meta"))), (k, k, dict(rope=torch.zeros(40, 64, device="meta")))):
        with pytest.raises(MoriError):
            A.kv_append(pool(), geometry(), 0, batch(), kk, vv, **kw)
    refused(attend, calls, out=torch.zeros(T, H, DIM, dtype=BF16, device="meta"))
    refused(attend, calls, lse=torch.zeros(T, H, device="meta"))
    assert not calls


def test_gradients_are_refused(calls):
    """Where they are recorded; under no_grad the same tensors are taken."""
    x = lambda h: torch.zeros(T, h, DIM, dtype=BF16)
    needs = lambda h: x(h).requires_grad_()
    for k, v, kw in ((needs(KV), x(KV), {}), (x(KV), needs(KV), {}), (x(KV), x(KV), dict(q=needs(H))),
                     (x(KV), x(KV), dict(q=x(H), q_out=needs(H))),
                     (x(KV), x(KV), dict(rope=torch.zeros(40, DIM, requires_grad=True)))):
        go = lambda: A.kv_append(pool(), geometry(), 0, batch(), k, v, **kw)
        with pytest.raises(MoriError) as e:
            go()
        assert e.value.code == M.MORI_EINVAL and not calls
        with torch.no_grad():
            go()
        assert calls.pop()
    for q, kw in ((needs(H), {}), (x(H), dict(out=needs(H))), (x(H), dict(lse=torch.zeros(T, H, requires_grad=True)))):
        go = lambda: A.kv_attend(pool(), geometry(), 0, batch(), q, **kw)
        with pytest.raises(MoriError) as e:
            go()
        assert e.value.code == M.MORI_EINVAL and not calls
        with torch.no_grad():
            go()
        assert calls.pop()


def test_what_is_written_counts_as_changed(calls):
    """A tensor saved for a backward pass and then rewritten here is noticed there."""
    p, q, out, lse = pool(), torch.zeros(T, H, DIM, dtype=BF16), torch.zeros(T, H, DIM, dtype=BF16), torch.zeros(T, H)
    k = torch.zeros(T, KV, DIM, dtype=BF16)
    w = torch.ones(DIM, dtype=BF16, requires_grad=True)
    y = (q * w).sum()
    before = p._version, out._version, lse._version
    A.kv_append(p, geometry(), 0, batch(), k, k, q=q, q_out=q)
    A.kv_attend(p, geometry(), 0, batch(), q, out=out, lse=lse)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    assert (p._version, out._version, lse._version) == tuple(b + 1 for b in before)
    with torch.inference_mode():
        q = torch.zeros(T, H, DIM, dtype=BF16)
        A.kv_append(p, geometry(), 0, batch(), k, k, q=q, q_out=q)
        A.kv_attend(p, geometry(), 0, batch(), q)


def test_query_widths_that_no_row_holds(calls):
    for shape, kw in (((T, H, 0), {}), ((T, H, 48), {}), ((T, H), {}), ((T, H, 64), dict(planes=1, layers=4)),
                      ((T, H, 32), dict(planes=1, layers=4))):
        q = torch.zeros(*shape, dtype=BF16)
        with pytest.raises(MoriError):
            A.kv_attend(pool(), geometry(**kw), 0, batch(**kw), q)
    assert not calls


@pytest.mark.parametrize("call", [append, attend])
def test_another_device_is_current(calls, monkeypatch, call):
    """The library launches on the current device: the batch's is made that for the call."""
    now = [1]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.before, now[0] = now[0], self.index

        def __exit__(self, *_):
            now[0] = self.before

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(A, "_current_device", lambda: now[0], raising=False)
    for name in ("mori_kv_append", "mori_kv_attend"):
        monkeypatch.setattr(M, name, lambda *a, **k: calls.append(now[0]) or M.MORI_OK)
    call()
    assert calls == [0] and now == [1]


def test_a_stream_of_another_device(monkeypatch):
    class Stream:
        cuda_stream, device = 64, torch.device("cuda", 1)

    b = batch()
    b._last = 0
    with pytest.raises(MoriError):
        A._stream_of(b, Stream())


def test_latent_pools_ask_for_the_model_s_scale(calls):
    """The row's width is not the width of the model's heads: taking it is not silent."""
    import warnings

    b, g = batch(planes=1, row_bytes=1152), geometry(planes=1, row_bytes=1152)
    p, q = torch.zeros(g.pool_bytes, dtype=torch.uint8), torch.zeros(T, H, 576, dtype=BF16)
    with pytest.warns(UserWarning, match="scale"):
        A.kv_attend(p, g, 0, b, q)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        A.kv_attend(p, g, 0, b, q, scale=192 ** -0.5)
        attend()
    assert [c[1][3].scale for c in calls] == pytest.approx([576 ** -0.5, 192 ** -0.5, DIM ** -0.5])
