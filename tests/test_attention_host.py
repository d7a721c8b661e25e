"""CPU-only checks of the token operators: every argument that does not fit is
refused on the host, before the HIP runtime is touched."""
import ctypes as C
import os

import pytest


@pytest.fixture(scope="module")
def M():
    from paper_2606_00866_amd import build, mori
    if not os.path.exists(mori.LIB_PATH):
        build.build()
    mori.lib()
    return mori


A16 = 0x1000  # an aligned address; nothing here is dereferenced


def pool(M, **kw):
    return M.mori_pool(**{**dict(layers=2, planes=2, block_tokens=16, row_bytes=4 * 64 * 2, num_blocks=8, base=A16), **kw})


def tokens(M, **kw):
    return M.mori_tokens(**{**dict(num_seqs=2, num_tokens=5, max_new=3, max_kv=40, seq_off=A16, kv_len=A16, program=None,
                                   num_programs=2, tbl_len=8, tbl_off=A16, tbl=A16), **kw})


def rows(M, data=A16, token=256, head=64):
    return M.mori_rows(data, token, head)


def append(M, **kw):
    return M.mori_append(**{**dict(dtype=1, kv_heads=4, head_dim=64, q_heads=8, rot_dim=64, rope_style=0, rope_len=40,
                                   rope=A16, k=rows(M), v=rows(M), q=rows(M), q_out=rows(M)), **kw})


def attend(M, **kw):
    return M.mori_attend(**{**dict(dtype=1, q_heads=8, kv_heads=4, head_dim=64, value_dim=64, scale=0.125, q=rows(M),
                                   out=rows(M), lse=None), **kw})


BAD_POOLS = [dict(base=0), dict(base=A16 + 16), dict(planes=3), dict(row_bytes=24), dict(num_blocks=0),
             dict(num_blocks=0xFFFFFFFF), dict(block_tokens=0), dict(layers=0), dict(row_bytes=1024)]
BAD_TOKENS = [dict(num_seqs=0), dict(num_seqs=4097), dict(seq_off=None), dict(kv_len=None), dict(tbl_off=None),
              dict(tbl=None), dict(num_programs=0), dict(max_kv=0), dict(max_kv=1 << 31), dict(num_tokens=1 << 31)]
EMPTY = dict(num_tokens=0)


def test_append_refusals(M):
    call = lambda p=None, layer=0, t=None, a=None: M.mori_kv_append(p or pool(M), layer, t or tokens(M), a or append(M))
    for bad in BAD_POOLS:
        assert call(p=pool(M, **bad)) == M.MORI_EINVAL, bad
    for bad in BAD_TOKENS:
        assert call(t=tokens(M, **bad)) == M.MORI_EINVAL, bad
    assert call(layer=2) == M.MORI_EINVAL
    r = lambda **kw: rows(M, **kw)
    for bad in (dict(dtype=2), dict(rope_style=2), dict(kv_heads=0), dict(kv_heads=2), dict(head_dim=0), dict(head_dim=72),
                dict(head_dim=128), dict(rot_dim=8), dict(rot_dim=80), dict(rope=None), dict(rope=A16 + 4), dict(rope_len=0),
                dict(q_heads=0), dict(q_heads=1025), dict(k=r(data=None)), dict(k=r(data=A16 + 8)), dict(v=r(token=12)),
                dict(v=r(head=4)), dict(q=r(data=A16 + 2)), dict(q_out=r(data=None)), dict(q_out=r(token=4))):
        assert call(a=append(M, **bad)) == M.MORI_EINVAL, bad
    latent = pool(M, planes=1, row_bytes=576 * 2)
    for bad in (dict(head_dim=576, kv_heads=1, rot_dim=0), dict(head_dim=576, kv_heads=1, rot_dim=576),
                dict(head_dim=288, kv_heads=2, rot_dim=64)):
        assert call(p=latent, a=append(M, **bad)) == M.MORI_EINVAL, bad
    assert call(t=tokens(M, **EMPTY)) == M.MORI_OK
    L = M.lib()
    p, t, a = pool(M), tokens(M), append(M)
    for args in ((None, 0, C.byref(t), C.byref(a)), (C.byref(p), 0, None, C.byref(a)), (C.byref(p), 0, C.byref(t), None)):
        assert L.mori_kv_append(*args, None, None) == M.MORI_EINVAL


def test_attend_refusals(M):
    def call(p=None, layer=0, t=None, a=None, ws=A16, n=1 << 40):
        return M.mori_kv_attend(p or pool(M), layer, t or tokens(M), a or attend(M), ws, n)

    size = lambda p=None, t=None, a=None: M.mori_kv_attend_workspace(p or pool(M), t or tokens(M), a or attend(M))[0]
    for bad in BAD_POOLS:
        assert call(p=pool(M, **bad)) == M.MORI_EINVAL and size(p=pool(M, **bad)) == M.MORI_EINVAL, bad
    for bad in BAD_TOKENS:
        assert call(t=tokens(M, **bad)) == M.MORI_EINVAL and size(t=tokens(M, **bad)) == M.MORI_EINVAL, bad
    assert call(layer=2) == M.MORI_EINVAL
    for bad in (dict(dtype=2), dict(q_heads=0), dict(q_heads=6), dict(q_heads=1028), dict(kv_heads=0), dict(kv_heads=2),
                dict(head_dim=32), dict(head_dim=128), dict(value_dim=32), dict(scale=float("nan")),
                dict(scale=float("inf"))):
        assert call(a=attend(M, **bad)) == M.MORI_EINVAL and size(a=attend(M, **bad)) == M.MORI_EINVAL, bad
    r = lambda **kw: rows(M, **kw)
    for bad in (dict(q=r(data=None)), dict(q=r(data=A16 + 8)), dict(q=r(token=4)), dict(out=r(data=None)),
                dict(out=r(head=2))):
        assert call(a=attend(M, **bad)) == M.MORI_EINVAL, bad
    # row sizes of other head dimensions, and latents of other widths
    assert call(p=pool(M, row_bytes=4 * 96 * 2), a=attend(M, head_dim=96, value_dim=96)) == M.MORI_EINVAL
    for dim, value in ((576, 576), (512, 512), (640, 512)):
        assert call(p=pool(M, planes=1, row_bytes=dim * 2), a=attend(M, kv_heads=1, head_dim=dim, value_dim=value)) == \
            M.MORI_EINVAL
    latent = attend(M, kv_heads=1, head_dim=576, value_dim=512)
    assert size(p=pool(M, planes=1, row_bytes=1152), a=latent) == M.MORI_OK
    assert call(t=tokens(M, **EMPTY)) == M.MORI_OK
    # a workspace that is short, missing or misaligned
    t = tokens(M, num_seqs=1, num_tokens=1, max_new=1, max_kv=100000)
    rc, n = M.mori_kv_attend_workspace(pool(M), t, attend(M))
    assert rc == M.MORI_OK
    if n:
        assert call(t=t, n=n - 1) == M.MORI_EINVAL and call(t=t, ws=0) == M.MORI_EINVAL
        assert call(t=t, ws=A16 + 128) == M.MORI_EINVAL
    assert M.lib().mori_kv_attend_workspace(C.byref(pool(M)), C.byref(t), C.byref(attend(M)), None) == M.MORI_EINVAL


def test_workspace_does_not_grow_without_bound(M):
    """It follows tokens, sequences and heads, not the context length."""
    at = lambda **kw: M.mori_kv_attend_workspace(pool(M, row_bytes=8 * 128 * 2), tokens(M, **kw),
                                                 attend(M, q_heads=32, kv_heads=8, head_dim=128, value_dim=128))[1]
    step = dict(num_seqs=64, num_tokens=64, max_new=1)
    assert at(**step, max_kv=1 << 20) == at(**step, max_kv=1 << 30) < 1 << 30


def test_structures_match_the_header(M, tmp_path):
    """Sizes and offsets of the binding's structures, as a C compiler lays them out."""
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ("mori_tokens", "mori_rows", "mori_append", "mori_attend")
    lines = [f'printf("{n} %zu\\n", sizeof({n}));' for n in names]
    for n in names:
        lines += [f'printf("{n}.{f[0]} %zu\\n", offsetof({n}, {f[0]}));' for f in getattr(M, n)._fields_]
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "mori.h"\nint main(void) {\n' + "\n".join(lines) +
                   "\nreturn 0; }\n")
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), "-o", str(exe), str(src)], check=True)
    for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines():
        name, value = line.split()
        s, _, f = name.partition(".")
        got = getattr(getattr(M, s), f).offset if f else C.sizeof(getattr(M, s))
        assert got == int(value), line
