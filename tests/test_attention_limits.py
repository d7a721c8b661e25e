"""CPU-only: batches whose launch would have 2^32 threads or more are refused on the
host.  Up to there a call goes on to the launch, which no device takes here."""

import pytest
import torch

from test_attention_host import M, append, attend, pool, rows, tokens  # noqa: F401 (M is a fixture)


@pytest.fixture(autouse=True)
def no_device():
    if torch.cuda.is_available():
        pytest.skip("the calls that fit would run")


@pytest.mark.parametrize("q_heads", [0, 8])
def test_append(M, q_heads):
    units = (q_heads + 2 * 4) * 64 // 16  # 16 elements a thread
    a = append(M, q_heads=q_heads) if q_heads else append(M, q=rows(M, None), q_out=rows(M, None))
    most = (2 ** 32 - 256) // units
    call = lambda t: M.mori_kv_append(pool(M), 0, tokens(M, num_tokens=t), a)
    assert call(most) == M.MORI_EHIP
    for t in (most + 1, 2 * most, 2 ** 31 - 1):
        assert call(t) == M.MORI_EINVAL, t


@pytest.mark.parametrize("heads,max_new,rows_", [(8, 1, 16), (8, 12, 32), (8, 100, 128)])
def test_attend(M, heads, max_new, rows_):
    """The workspace call says the same."""
    p, a = pool(M), attend(M, q_heads=heads)
    size = lambda t: M.mori_kv_attend_workspace(p, tokens(M, num_tokens=t, max_new=max_new), a)[0]
    group = heads // 4
    most = ((2 ** 32 // 256 - 1) // 4 - 2) * rows_ // group  # 4 key heads, 2 sequences
    fits = most * heads < 2 ** 31
    assert size(min(most, 2 ** 31 // heads - 1)) == M.MORI_OK
    assert size(2 ** 27 // heads) == M.MORI_OK
    if fits:
        for t in (most + rows_, 2 ** 31 // heads - 1):
            assert size(t) == M.MORI_EINVAL, t
            assert M.mori_kv_attend(p, 0, tokens(M, num_tokens=t, max_new=max_new), a, 0x1000, 1 << 40) == M.MORI_EINVAL
