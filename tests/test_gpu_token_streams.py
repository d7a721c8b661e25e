"""The batch's error word where calls and checks are on different streams: nothing
here synchronises the device between a call and its check."""
import pytest
import torch

import attend_ref as R
from paper_2606_00866_amd import mori as M

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
H, KV, DIM = 4, 1, 64


class Case:
    """A batch's inputs, all of them ready; sequence 0 is longer than its blocks if bad."""

    def __init__(self, bad=True):
        self.inst = R.instance(51, [2, 3], [20, 30], kv=KV, dim=DIM)
        if bad:
            self.inst.length[0] = 200
        i = self.inst
        self.parts = [R.dev32(a) for a in (i.tbl_off, i.tbl, i.seq_off, i.length, i.prog)]
        self.pool = i.pool.cuda()
        self.k, self.v = (torch.ones(5, KV, DIM, dtype=BF16, device="cuda") for _ in range(2))
        self.q = torch.ones(5, H, DIM, dtype=BF16, device="cuda")
        self.out = torch.empty_like(self.q)
        self.work = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
        self.load = torch.randn(4096, 4096, device="cuda").to(BF16)
        self.batch()  # what a first batch allocates is there
        self.busy()
        torch.cuda.synchronize()

    def batch(self):
        from paper_2606_00866_amd import attention as A
        return A.TokenBatch(self.inst.geom, *self.parts[:4], program=self.parts[4], num_tokens=5, max_new=3, max_kv=1000)

    def busy(self, n=60):
        """Some ten milliseconds of products on the current stream."""
        x = self.load
        for _ in range(n):
            x = x @ self.load
        return x

    def call(self, name, b, **kw):
        from paper_2606_00866_amd import attention as A
        if name == "append":
            A.kv_append(self.pool, self.inst.geom, 1, b, self.k, self.v, **kw)
        else:
            A.kv_attend(self.pool, self.inst.geom, 1, b, self.q, out=self.out, workspace=self.work, **kw)


def found(b):
    from paper_2606_00866_amd.tiering import MoriError
    with pytest.raises(MoriError) as e:
        b.check()
    assert e.value.detail == M.MORI_DEV_BAD_TOKENS


@pytest.mark.parametrize("name", ["append", "attend"])
@pytest.mark.parametrize("how", ["argument", "current"])
def test_check_waits_for_the_call_s_stream(name, how):
    c, side = Case(), torch.cuda.Stream()
    b = c.batch()
    for _ in range(2):  # found, cleared, found again
        with torch.cuda.stream(side):
            c.busy()
            if how == "current":
                c.call(name, b)
        if how == "argument":
            c.call(name, b, stream=side)
        found(b)
    b.check()


def test_check_waits_for_every_stream():
    c, streams = Case(), [torch.cuda.Stream() for _ in range(3)]
    b = c.batch()
    with torch.cuda.stream(streams[0]):
        c.busy()
    for s in streams:
        c.call("append", b, stream=s)
    c.call("append", b)
    found(b)
    b.check()


def test_a_side_stream_checks():
    """Batch and call on the current stream, which is busy; the check on another."""
    c, side = Case(), torch.cuda.Stream()
    c.busy()
    b = c.batch()
    c.call("attend", b)
    with torch.cuda.stream(side):
        found(b)
        b.check()


@pytest.mark.parametrize("name", ["append", "attend"])
def test_the_word_is_cleared_before_the_first_call(name):
    """The batch is made on a stream with much to do, and used at once on another."""
    c, side = Case(), torch.cuda.Stream()
    c.busy()
    b = c.batch()
    c.call(name, b, stream=side)
    found(b)


def test_the_word_outlives_its_batch():
    """A batch dropped while a call of another stream is under way: its error word's
    memory is nobody else's yet."""
    c, side = Case(), torch.cuda.Stream()
    b = c.batch()
    with torch.cuda.stream(side):
        c.busy()
    c.call("append", b, stream=side)
    del b
    later = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    assert all(int(x) == 0 for x in later)


def test_the_word_outlives_its_batch_after_a_capture():
    """The other stream's first call was captured: its next one is not in the graph."""
    c, side = Case(), torch.cuda.Stream()
    b = c.batch()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.call("append", b)
    with torch.cuda.stream(side):
        c.busy()
    c.call("append", b, stream=side)
    del b
    later = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    assert all(int(x) == 0 for x in later)


def test_made_on_a_side_stream():
    """And used on the default one, at once; what is checked on the side waits for it."""
    c, side = Case(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.batch()  # what a first batch allocates there is there
        c.busy()
        torch.cuda.synchronize()
        c.busy()
        b = c.batch()
    c.call("append", b)
    found(b)
    c.busy()
    c.call("attend", b)
    with torch.cuda.stream(side):
        found(b)
        b.check()


def test_the_numbers_outlive_their_batch():
    """What ``TokenBatch.of`` copies to the device belongs to the batch alone: dropped while a
    call of another stream is under way, it is read as it was."""
    from types import SimpleNamespace

    from paper_2606_00866_amd import attention as A
    c, side = Case(bad=False), torch.cuda.Stream()
    i = c.inst
    c.call("attend", c.batch())
    want = c.out.clone()
    c.out.zero_()
    tp = SimpleNamespace(geom=i.geom, P=2, nblk=i.tbl_off[1:] - i.tbl_off[:-1], device="cuda", tbl_off=c.parts[0], tbl=c.parts[1])
    b = A.TokenBatch.of(tp, i.prog, i.n, i.length)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        c.busy()
    c.call("attend", b, stream=side)
    del b
    later = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    assert torch.equal(c.out, want) and len(later) == 64


def test_captured_without_a_call_before():
    """The batch's first call is one that is captured; replays report as calls do."""
    c = Case()
    b = c.batch()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call("append", b)
        c.call("attend", b)
    b.check()  # nothing has run
    for _ in range(3):
        graph.replay()
        found(b)
        b.check()


def test_good_batches_pass():
    c, side = Case(bad=False), torch.cuda.Stream()
    b = c.batch()
    c.call("append", b, stream=side)
    b.check()
    c.call("attend", b)
    c.call("attend", b, stream=side)
    b.check()
