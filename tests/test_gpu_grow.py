"""Tables that grow on the device, against the plain definition: every array, whole."""
import numpy as np
import pytest
import torch

import grow_ref as R
from paper_2606_00866_amd import attention as A
from paper_2606_00866_amd import mori as M
from paper_2606_00866_amd.tiering import MoriError

pytestmark = pytest.mark.gpu


def dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a).astype(dtype)).cuda()


def growth(s, in_place, tier=True, program=True, **bounds):
    x = dict(tbl_off=dev(s.tbl_off), tbl=dev(s.tbl), free=dev(s.free, np.uint8), held=dev(s.held))
    into = None
    if not in_place:  # entries past the tables stay as they are: give them what the plain form has there
        into = (torch.full_like(x["tbl_off"], 77), x["tbl"].clone(), torch.full_like(x["free"], 77),
                torch.full_like(x["held"], 77))
    b = bounds if len(bounds) == 3 else {**dict(num_tokens=s.T, max_new=s.max_new, max_kv=s.max_kv), **bounds}
    g = A.TokenGrowth(s.geom, x["tbl_off"], x["tbl"], x["free"], x["held"], dev(s.new), dev(s.prog) if program else None,
                      tier=dev(s.tier, np.uint8) if tier else None, into=into, **b)
    g.state = into or (x["tbl_off"], x["tbl"], x["free"], x["held"])
    g.before = x
    return g


def arrays(g):
    off, tbl, free, held = (x.cpu().numpy() for x in g.state)
    return dict(tbl_off=off, tbl=tbl, free=free, held=held, seq_off=g.batch.seq_off.cpu().numpy(),
                kv_len=g.batch.kv_len.cpu().numpy(), slots=g.slots.cpu().numpy(), positions=g.positions.cpu().numpy())


def same(got, want):
    for name, x in want.items():
        assert np.array_equal(got[name], x), name


CASES = {
    "one": (1, 1, 1, dict(held=15)),
    "one_long": (1, 1, 5000, dict(held=40000, bt=64)),
    "step": (8, 8, 1, dict(held=800)),
    "step_of_some": (64, 23, 1, dict(held=500)),
    "nothing_new": (9, 5, 0, dict()),
    "some_nothing": (40, 40, (0, 3), dict(bt=4)),
    "chunks": (12, 7, (1, 300), dict(held=900)),
    "odd_block": (33, 20, (0, 90), dict(bt=24, held=300)),
    "block_of_one": (10, 10, (0, 40), dict(bt=1, held=30, spare_blocks=0)),
    "block_of_17": (100, 64, (1, 50), dict(bt=17)),
    "empty_tables": (50, 30, (0, 33), dict(held=0, spare_blocks=0)),
    "large_blocks": (6, 4, (1, 700), dict(bt=512, held=3000)),
    "wave_edge": (64, 64, (1, 4), dict(bt=2, held=20)),
    "past_a_wave": (65, 65, (1, 4), dict(bt=2, held=20)),
    "most_programs": (4096, 4096, (0, 9), dict(bt=8, held=60)),
    "few_of_most": (4095, 3, (1, 70), dict(held=100)),
    "tiles": (300, 200, (1, 400), dict(held=900, spare_pages=13000)),
    "pages_from_the_end": (200, 100, (1, 300), dict(held=2000, spare_pages=0, free_first=True)),
    "taken_over_tiles": (30, 30, (2000, 4000), dict(bt=4, held=50, spare_pages=3)),
    # on both sides of what a workgroup of 64, 256 and 1024 threads takes: pages, entries, tokens, programs
    "pages_1024": (10, 8, (0, 40), dict(held=50, spare_pages=980)),
    "pages_1030": (10, 8, (0, 40), dict(held=50, spare_pages=1020)),
    "entries_512": (20, 8, (0, 20), dict(held=50, room=520)),
    "tokens_256": (8, 8, 30, dict(held=50, pad=16)),
    "tokens_257": (8, 8, 30, dict(held=50, pad=17)),
    "programs_65": (65, 30, (0, 5), dict(held=20)),
    "pages_17": (2, 1, 40, dict(held=20, spare_pages=9)),
    "small_programs": (1024, 1024, (0, 4), dict(bt=4, held=12, spare_pages=900)),
    "programs_above": (1025, 40, (0, 4), dict(bt=4, held=12)),
    "programs_257": (257, 257, 1, dict(bt=4, held=12)),
    "some_256": (256, 256, (0, 3), dict(bt=4, held=8, spare_blocks=1)),
    "pages_4096": (30, 20, (0, 40), dict(held=50, spare_pages=4000)),
    "pages_above": (30, 20, (0, 40), dict(held=50, spare_pages=16390)),
    "entries_above": (40, 20, (0, 40), dict(held=50, room=8192)),
    "tokens_above": (8, 8, 500, dict(held=50, pad=97)),
    "tokens_4096": (8, 8, 500, dict(held=50, pad=96)),
    "large_step": (200, 100, 1, dict(held=500, spare_pages=17000)),
}


@pytest.mark.parametrize("in_place", [False, True])
def test_large_pools(in_place):
    """More pages than 2^19: larger tiles.  Pages are taken on both sides of tile borders, and
    the last tile is a part of one."""
    s = R.instance(21, 50, 40, (500, 4000), bt=4, held=300, spare_pages=0)
    used = s.free.size
    pages = (1 << 19) + 4096 + 777
    free = np.zeros(pages, np.uint8)
    at = np.sort(np.random.default_rng(2).permutation(np.arange(used, pages))[:s.extra["grown"] + 9])
    free[at] = 1
    free[-3:] = 1
    s.free, s.geom.num_blocks = free, pages
    g = growth(s, in_place)
    g.run()
    same(arrays(g), R.grow(s))
    g.batch.check()


def test_no_tokens():
    s = R.instance(22, 9, 4, 0, pad=0)
    g = growth(s, True)
    assert g.slots.numel() == g.positions.numel() == 0
    g.run()
    same(arrays(g), R.grow(s))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("name", CASES)
def test_against_definition(name, in_place):
    programs, seqs, new, kw = CASES[name]
    s = R.instance(len(name), programs, seqs, new, **kw)
    g = growth(s, in_place)
    for _ in range(1 if in_place else 3):
        g.run()
        same(arrays(g), R.grow(s))
    g.batch.check()
    if not in_place:  # what was before is left alone
        same({k: v.cpu().numpy() for k, v in g.before.items()}, dict(tbl_off=s.tbl_off, tbl=s.tbl, free=s.free, held=s.held))


def test_without_tier_and_program():
    s = R.instance(3, 20, 20, (0, 30), off_gpu=0.0)
    s.prog = np.arange(20)
    s.tbl = np.concatenate([s.tbl, np.full(200, -1)])
    s.free = np.concatenate([s.free, np.ones(200, np.uint8)])
    s.geom.num_blocks += 200
    g = growth(s, True, tier=False, program=False)
    g.run()
    same(arrays(g), R.grow(s))


def test_steps_in_place():
    """Forty steps of one growth: every state follows from the last."""
    s = R.instance(11, 30, 20, 1, bt=4, held=50, spare_pages=300, room=300)
    g = growth(s, True, max_kv=400)
    for _ in range(40):
        g.run()
        want = R.grow(s)
        same(arrays(g), want)
        s.tbl_off, s.tbl, s.free, s.held = (want[k] for k in ("tbl_off", "tbl", "free", "held"))
    g.batch.check()


def refusals():
    def pages(s):
        s.free[np.flatnonzero(s.free)[s.extra["grown"] - 1:]] = 0

    def entries(s):
        s.tbl = s.tbl[:s.tbl_off[-1] + s.extra["grown"] - 1]

    def twice(s):
        s.prog[3] = s.prog[0]

    def outside(s):
        s.prog[2] = s.held.size

    def off_gpu(s):
        s.tier[s.prog[1]] = 1

    def more_held(s):
        p = s.prog[0]
        s.held[p] = (s.tbl_off[p + 1] - s.tbl_off[p]) * s.geom.block_tokens + 1

    def negative(s):
        s.new[0] = -1

    return {"pages": (pages, M.MORI_DEV_NOSPC, {}), "entries": (entries, M.MORI_DEV_NOSPC, {}),
            "twice": (twice, M.MORI_DEV_BAD_TOKENS, {}), "outside": (outside, M.MORI_DEV_BAD_TOKENS, {}),
            "off_gpu": (off_gpu, M.MORI_DEV_NOT_RESIDENT, {}), "more_held": (more_held, M.MORI_DEV_BAD_TOKENS, {}),
            "negative": (negative, M.MORI_DEV_BAD_TOKENS, {}), "max_new": (None, M.MORI_DEV_BAD_TOKENS, dict(max_new=89)),
            "max_kv": (None, M.MORI_DEV_BAD_TOKENS, dict(max_kv=100)),
            "tokens": (None, M.MORI_DEV_BAD_TOKENS, dict(num_tokens=500))}


@pytest.mark.parametrize("pages", [40, 17000])  # one workgroup's pool, and a larger one
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("name", refusals())
def test_what_does_not_fit_changes_nothing(name, in_place, pages):
    spoil, bits, bounds = refusals()[name]
    s = R.instance(5, 25, 12, (60, 90), held=100, spare_blocks=0, spare_pages=pages)
    s.new[5] = 90
    if spoil:
        if name == "pages":  # one page fewer than needed; with all of them it fits
            s.free[np.flatnonzero(s.free)[s.extra["grown"]:]] = 0
            assert R.grow(s) is not None
        kv, most = s.max_kv, s.max_new
        spoil(s)
        bounds = dict(max_kv=4 * kv, max_new=most, num_tokens=s.T)
    g = growth(s, in_place, **bounds)
    s.T = bounds.get("num_tokens", s.T)
    g.run()
    same(arrays(g), R.refused(s))
    with pytest.raises(MoriError) as e:
        g.batch.check()
    assert e.value.detail == bits


@pytest.mark.parametrize("pages", [40, 17000])
@pytest.mark.parametrize("bad", ["start", "falls", "long"])
def test_bad_offsets(bad, pages):
    """In place nothing is written; the batch is empty."""
    s = R.instance(6, 25, 12, (1, 9), spare_pages=pages)
    if bad == "start":
        s.tbl_off[0] = 1
    elif bad == "falls":
        s.tbl_off[7] = s.tbl_off[8] + 1
    else:
        s.tbl_off[-1] = s.tbl.size + 1
    g = growth(s, True)
    g.run()
    same(arrays(g), R.refused(s))
    with pytest.raises(MoriError) as e:
        g.batch.check()
    assert e.value.detail & M.MORI_DEV_BAD_TBL_OFF


@pytest.mark.parametrize("pad", [5, 5000])
def test_exactly_enough(pad):
    for spare in (0, 1):
        s = R.instance(8, 25, 12, (60, 90), held=100, spare_blocks=0, spare_pages=spare, room=spare, pad=pad)
        g = growth(s, True)
        g.run()
        same(arrays(g), R.grow(s))
        g.batch.check()


@pytest.mark.parametrize("page,bit", [(-1, M.MORI_DEV_NOT_RESIDENT), (10 ** 6, M.MORI_DEV_PAGE_RANGE)])
@pytest.mark.parametrize("pad", [5, 5000])
def test_old_block_without_page(page, bit, pad):
    """The token's slot is -1; the rest stands."""
    s = R.instance(9, 10, 10, 3, held=60, spare_blocks=2, off_gpu=0.0, pad=pad)
    p = int(s.prog[4])
    s.held[p] = 20
    s.tbl_off[p + 1:] += max(0, 3 - int(s.tbl_off[p + 1] - s.tbl_off[p]))
    s.tbl = np.arange(int(s.tbl_off[-1]) + 30)
    s.tbl[s.tbl_off[-1]:] = -1
    s.free = np.concatenate([np.zeros(s.tbl_off[-1], np.uint8), np.ones(40, np.uint8)])
    s.geom.num_blocks = s.free.size
    s.tbl[s.tbl_off[p] + 1] = page
    want = R.grow(s)
    want["slots"][4 * 3:4 * 3 + 3] = -1
    g = growth(s, True)
    g.run()
    same(arrays(g), want)
    with pytest.raises(MoriError) as e:
        g.batch.check()
    assert e.value.detail == bit


def test_graph_replays():
    """A captured step replays in place; counts may change between replays, eager work runs
    between them."""
    s = R.instance(12, 40, 30, (0, 5), bt=4, held=50, spare_pages=2000, room=2000)
    g = growth(s, True, max_new=9, max_kv=2000, num_tokens=300)
    s.T = 300
    new = g.batch._keep[9]
    assert new.numel() == 30
    g.run()  # warm
    want = R.grow(s)
    same(arrays(g), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.run()
    rng = np.random.default_rng(1)
    for i in range(6):
        s.tbl_off, s.tbl, s.free, s.held = (want[k] for k in ("tbl_off", "tbl", "free", "held"))
        s.new = rng.integers(0, 10, 30)
        new.copy_(dev(s.new))
        graph.replay()
        torch.randn(1000, device="cuda").sum().item()
        want = R.grow(s)
        same(arrays(g), want)
    g.batch.check()


def test_other_stream():
    s = R.instance(13, 40, 30, (0, 60), held=500)
    g = growth(s, False)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    g.run(stream=st)
    st.synchronize()
    same(arrays(g), R.grow(s))
    with torch.cuda.stream(st):
        g.run()
    g.batch.check()
    same(arrays(g), R.grow(s))
