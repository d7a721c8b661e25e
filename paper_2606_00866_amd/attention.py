"""What a model does with the paged KV pool, for torch tensors on the device:
``kv_append`` writes new tokens' keys and values into the programs' pages (and
rotates them and their queries by position), ``kv_attend`` lets the queries
attend to everything the programs hold.  ``TokenBatch`` says which tokens of
which programs; it is made once a step and used in every layer.

Like ``mori``, this only marshals arguments: the work runs in libmori's kernels,
on the current stream unless one is given, and nothing here waits for the device
(but ``TokenBatch.check``).  Arguments that do not fit raise ``MoriError`` before
anything is enqueued.  The operators serve: where gradients are recorded, tensors
that require them are refused, and what is written counts as changed in place.
"""
from __future__ import annotations

import contextlib
import warnings

import numpy as np
import torch

from . import mori as M
from .tiering import MoriError, PoolGeometry, check

DTYPES = {torch.float16: M.MORI_DT_F16, torch.bfloat16: M.MORI_DT_BF16}
STYLES = {"half": M.MORI_ROPE_HALF, "pairs": M.MORI_ROPE_PAIRS}
_current_device = torch._C._cuda_getDevice
LATENT_ROPE = 64  # rotated elements behind the latent part of a latent row


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise MoriError(what, M.MORI_EINVAL)


def rope_table(positions: int, rot_dim: int, theta: float = 10000.0, device="cuda") -> torch.Tensor:
    """float32 [positions][rot_dim]: the cosines of every pair's angle, then the
    sines; pair i turns by position * theta^(-2i / rot_dim).  Angles are taken in
    64 bits, so long contexts keep their precision."""
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * \
        theta ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64, device=device) / rot_dim)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _stream_of(batch, stream) -> int:
    """The handle of the stream that a call runs on, by default the current one of the
    batch's device; the batch's error word is ready for it."""
    handle = torch._C._cuda_getCurrentRawStream(batch.index) if stream is None else stream.cuda_stream
    if stream is not None and stream.device != batch.device:
        raise MoriError(f"a stream of {stream.device} for a batch on {batch.device}", M.MORI_EINVAL)
    if handle != batch._last:
        batch._enter(handle)
    return handle


def _needs_gradients(what: str) -> MoriError:
    """These operators have no backward pass: where gradients are recorded, tensors
    that need them are refused instead of being left out of the record."""
    return MoriError(f"{what}: no gradients pass through a paged pool (detach, or call under torch.no_grad())",
                     M.MORI_EINVAL)


def _stream_at(handle: int, device: torch.device) -> torch.cuda.Stream:
    """The stream of a handle; that of the default stream is 0, which ExternalStream does
    not take for it."""
    return torch.cuda.ExternalStream(handle, device) if handle else torch.cuda.default_stream(device)


def _on(stream):
    """Where this module's own allocations belong: the stream that uses them, so
    that the allocator hands their memory on in that stream's order."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


class TokenBatch:
    """New tokens of some programs, packed one program after the other.

    tbl_off, tbl: the pool's block tables (int32, as ``TierPool`` keeps them).
    seq_off int32 [B+1]: sequence b is tokens seq_off[b] .. seq_off[b+1]-1, the
    last of the kv_len[b] (int32 [B]) tokens that program[b] (int32 [B]; None:
    program b) holds once they are appended; tokens before position 0 are padding.
    num_tokens, max_new, max_kv: the batch's tokens and the most that any sequence
    brings and holds, as the host knows them (the device checks them).  The
    tensors may be rewritten between steps, also under a captured graph, as long
    as these bounds hold.

    A batch is for pools of the geometry that it was made with.

    ``error`` collects the device's MORI_DEV_* bits; ``check`` waits, reads and
    clears it.  Calls may run on any streams; those stay alive until ``check`` or
    the batch's end."""

    def __init__(self, geom, tbl_off: torch.Tensor, tbl: torch.Tensor, seq_off: torch.Tensor, kv_len: torch.Tensor,
                 program: torch.Tensor | None = None, *, num_tokens: int, max_new: int, max_kv: int):
        self.shape = tuple(int(getattr(geom, name)) for name in
                           ("layers", "planes", "block_tokens", "row_bytes", "num_blocks"))
        self.geom = PoolGeometry(*self.shape)
        self.pool_bytes = self.geom.pool_bytes
        self.num_seqs, self.num_tokens = int(kv_len.numel()), int(num_tokens)
        for name, x, n in (("tbl_off", tbl_off, None), ("tbl", tbl, None), ("seq_off", seq_off, self.num_seqs + 1),
                           ("kv_len", kv_len, self.num_seqs), ("program", program, self.num_seqs)):
            if x is None:
                continue
            _need(x.dtype == torch.int32 and x.is_contiguous() and x.dim() == 1 and x.device.type == "cuda" and
                  x.device == kv_len.device, f"TokenBatch: {name} is a contiguous int32 vector on the batch's device")
            _need(n is None or x.numel() == n, f"TokenBatch: {name} has {x.numel()} entries, not {n}")
        _need(num_tokens >= 0 and max_new >= 0 and 0 < max_kv < 1 << 31, "TokenBatch: bounds out of range")
        _need(tbl_off.numel() >= 2, "TokenBatch: tbl_off is empty")
        self.device = kv_len.device
        self.index = kv_len.device.index
        self.error = torch.zeros(1, dtype=torch.int32, device=self.device)
        # Streams other than the one that clears the word wait for that, and check waits for them.
        made = torch.cuda.current_stream(self.device)
        self._made, self._last = made.cuda_stream, None
        self._used, self._ordered = set(), {self._made}
        self._ready = None if torch.cuda.is_current_stream_capturing() else made.record_event()
        self._keep = (tbl_off, tbl, seq_off, kv_len, program)
        self.desc = M.mori_tokens(self.num_seqs, self.num_tokens, int(max_new), int(max_kv), seq_off.data_ptr(),
                                  kv_len.data_ptr(), program.data_ptr() if program is not None else None,
                                  tbl_off.numel() - 1, tbl.numel(), tbl_off.data_ptr(), tbl.data_ptr())

    @classmethod
    def of(cls, tier_pool, programs, new_tokens, kv_len) -> "TokenBatch":
        """A batch of a ``TierPool``'s programs from host numbers: new_tokens[i] new
        tokens of programs[i], which then holds kv_len[i]."""
        n, length = np.asarray(new_tokens, np.int64), np.asarray(kv_len, np.int64)
        prog = np.asarray(programs, np.int64)
        _need(n.ndim == 1 and n.shape == length.shape == prog.shape, "TokenBatch: one number per sequence")
        _need(bool((n >= 0).all() and (length >= 0).all() and (prog >= 0).all() and (prog < tier_pool.P).all()),
              "TokenBatch: numbers out of range")
        _need(bool((length <= tier_pool.nblk[prog] * tier_pool.geom.block_tokens).all()),
              "TokenBatch: more tokens than the program's blocks hold")
        dev = lambda a: torch.from_numpy(a.astype(np.int32)).to(tier_pool.device)
        off = np.concatenate([[0], np.cumsum(n)])
        return cls(tier_pool.geom, tier_pool.tbl_off, tier_pool.tbl, dev(off), dev(length), dev(prog),
                   num_tokens=int(off[-1]), max_new=int(n.max(initial=0)), max_kv=max(1, int(length.max(initial=1))))

    def _enter(self, handle: int) -> None:
        """A call is about to use the stream: its first one, or the first after another's."""
        self._used.add(handle)
        self._last = handle
        if handle in self._ordered:
            return
        stream = _stream_at(handle, self.device)
        with torch.cuda.stream(stream):
            if torch.cuda.is_current_stream_capturing():  # a graph's inputs are ready before it is replayed
                self._last = None
                return
        if self._ready is not None:
            stream.wait_event(self._ready)
        for x in (self.error, *self._keep):
            if x is not None:
                x.record_stream(stream)
        self._ordered.add(handle)

    def check(self) -> None:
        """Raises MoriError if the device found fault with the batch since the last check.
        Waits for every call since then, on whichever stream it was made.  Replays of a
        captured graph are work of the stream that replays it: check on that stream, or
        behind it."""
        here = torch.cuda.current_stream(self.device)
        if self._ready is not None and here.cuda_stream != self._made:
            here.wait_event(self._ready)
        for handle in self._used:
            if handle != here.cuda_stream:
                here.wait_stream(_stream_at(handle, self.device))
        bits = int(self.error.item())
        if bits:
            self.error.zero_()
            here.synchronize()  # cleared before any stream's next call
        self._used.clear()
        self._ordered = {self._made}
        self._last = self._ready = None
        if bits:
            raise MoriError("token batch", M.MORI_EDEVICE, bits)


def _same_geometry(geom, batch: TokenBatch) -> None:
    if (geom.layers, geom.planes, geom.block_tokens, geom.row_bytes, geom.num_blocks) != batch.shape:
        raise MoriError("geom is not the batch's", M.MORI_EINVAL)


def _pool(pool: torch.Tensor, geom, batch: TokenBatch, dtype: torch.dtype) -> M.mori_pool:
    """The pool as bytes (any integer type) or as what its rows hold."""
    _same_geometry(geom, batch)
    if not pool.is_contiguous() or pool.device != batch.device or pool.nbytes != batch.pool_bytes:
        raise MoriError("pool does not have its geometry's bytes on the batch's device", M.MORI_EINVAL)
    if pool.dtype != dtype and pool.dtype.is_floating_point:
        raise MoriError(f"the pool is of {pool.dtype}, the tokens of {dtype}", M.MORI_EINVAL)
    return M.mori_pool(*batch.shape, pool.data_ptr())


def _rows(name: str, x: torch.Tensor, batch: TokenBatch, dtype: torch.dtype, heads: int | None = None,
          dim: int | None = None, written: bool = False) -> M.mori_rows:
    """A [tokens][heads][elements] view with its strides; elements are adjacent.
    Views to write have a place for every element (no broadcast)."""
    shape, strides = x.shape, x.stride()
    if len(shape) != 3 or shape[0] != batch.num_tokens or x.dtype != dtype or x.device != batch.device:
        raise MoriError(f"{name}: [{batch.num_tokens}][heads][elements] of {dtype} on {batch.device}", M.MORI_EINVAL)
    tokens, h, d = shape
    if (heads is not None and h != heads) or (dim is not None and d != dim):
        raise MoriError(f"{name}: shape {tuple(shape)}, not [tokens][{heads}][{dim}]", M.MORI_EINVAL)
    # a stride over one token or one head is never used; views may carry any value there
    token = strides[0] if tokens > 1 else 0
    head = strides[1] if h > 1 else 0
    if (d and strides[2] != 1) or (written and ((tokens > 1 and not token) or (h > 1 and not head))):
        raise MoriError(f"{name}: strides {strides}: elements are adjacent, and views to write have a place for each",
                        M.MORI_EINVAL)
    return M.mori_rows(x.data_ptr() or None, token, head)


def kv_append(pool: torch.Tensor, geom, layer: int, batch: TokenBatch, k: torch.Tensor, v: torch.Tensor, *,
              q: torch.Tensor | None = None, q_out: torch.Tensor | None = None, rope: torch.Tensor | None = None,
              style: str = "half", stream=None):
    """Stores the batch's keys and values in one layer of the pool.

    planes 2: k, v [T][kv_heads][head_dim]; the first rope.shape[1] elements of
    every key head turn with the token's position.  planes 1: k [T][1][latent]
    copied, v [T][1][rot] rotated behind it.  q, if given, is rotated the same way
    ([T][q_heads][head_dim], or [T][q_heads][rot] with planes 1) into q_out, which
    may be q; returns q_out (allocated if not given)."""
    if _current_device() != batch.index:  # launches go to the current device
        with torch.cuda.device(batch.index):
            return kv_append(pool, geom, layer, batch, k, v, q=q, q_out=q_out, rope=rope, style=style, stream=stream)
    if torch.is_grad_enabled() and (k.requires_grad or v.requires_grad or pool.requires_grad or
                                    (q is not None and q.requires_grad) or
                                    (q_out is not None and q_out.requires_grad) or
                                    (rope is not None and rope.requires_grad)):
        raise _needs_gradients("kv_append")
    dtype = k.dtype
    if dtype not in DTYPES or style not in STYLES:
        raise MoriError("kv_append: float16 or bfloat16, style 'half' or 'pairs'", M.MORI_EINVAL)
    if k.dim() != 3 or v.dim() != 3:
        raise MoriError("kv_append: k and v are [tokens][heads][elements]", M.MORI_EINVAL)
    latent, heads, dim = geom.planes == 1, k.shape[1], k.shape[2]
    if latent:
        dim += v.shape[2]
    rot = positions = 0
    if rope is not None:
        if rope.dtype != torch.float32 or rope.dim() != 2 or not rope.is_contiguous() or rope.device != batch.device:
            raise MoriError("kv_append: rope is a contiguous float32 [positions][rot_dim] on the batch's device",
                            M.MORI_EINVAL)
        positions, rot = rope.shape
    a = M.mori_append(DTYPES[dtype], heads, dim, 0, rot, STYLES[style], positions, rope.data_ptr() if rot else None)
    a.k = _rows("k", k, batch, dtype, 1 if latent else None)
    a.v = _rows("v", v, batch, dtype, heads, rot if latent else dim)
    if q is not None:
        a.q = _rows("q", q, batch, dtype, None, rot if latent else dim)
        if q_out is None:
            with _on(stream):
                q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        a.q_out = _rows("q_out", q_out, batch, dtype, q.shape[1], q.shape[2], True)
        a.q_heads = q.shape[1]
    check(M.mori_kv_append(_pool(pool, geom, batch, dtype), int(layer), batch.desc, a, batch.error.data_ptr(),
                           _stream_of(batch, stream)), "mori_kv_append")
    torch.autograd.graph.increment_version((pool,) if q is None else (pool, q_out))
    return q_out


def _attend_desc(geom, q: torch.Tensor, scale: float | None) -> M.mori_attend:
    shape, dtype = q.shape, DTYPES.get(q.dtype)
    if dtype is None or len(shape) != 3:
        raise MoriError("kv_attend: q is [tokens][heads][elements] of float16 or bfloat16", M.MORI_EINVAL)
    dim = shape[2]
    value = dim - LATENT_ROPE if geom.planes == 1 else dim
    if value <= 0 or geom.row_bytes % (2 * dim):
        raise MoriError(f"kv_attend: rows of {geom.row_bytes} B hold no heads of {dim}", M.MORI_EINVAL)
    return M.mori_attend(dtype, shape[1], geom.row_bytes // (2 * dim), dim, value,
                         dim ** -0.5 if scale is None else float(scale))


def _empty_pool(geom) -> M.mori_pool:
    """The pool as a description only (the workspace call reads no memory)."""
    return M.mori_pool(geom.layers, geom.planes, geom.block_tokens, geom.row_bytes, geom.num_blocks, 256)


def kv_attend_workspace(geom, batch: TokenBatch, q: torch.Tensor) -> torch.Tensor:
    """Device workspace for kv_attend of this batch, in every layer; calls that may
    overlap (on other streams) need one each."""
    _same_geometry(geom, batch)
    a = _attend_desc(geom, q, None)
    rc, n = M.mori_kv_attend_workspace(_empty_pool(geom), batch.desc, a)
    check(rc, "mori_kv_attend_workspace")
    return torch.empty(n, dtype=torch.uint8, device=batch.device)


def kv_attend(pool: torch.Tensor, geom, layer: int, batch: TokenBatch, q: torch.Tensor, *, scale: float | None = None,
              out: torch.Tensor | None = None, lse: torch.Tensor | None = None,
              workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Causal attention of the batch's tokens over their programs' pages in one
    layer.  q [T][q_heads][head_dim] (latent pools: [T][q_heads][576], in the latent
    space).  scale: head_dim ** -0.5 unless given; a latent row's width says nothing
    of the model's own (its heads' width before compression, 128 + 64 where rows are
    512 + 64), so on latent pools leaving it out warns.  Returns out [T][q_heads]
    [head_dim] (latent pools: 512), allocated if not given; lse, a float32
    [T][q_heads] tensor, takes the logarithms of the rows' sums.  The workspace is
    allocated here unless given."""
    if _current_device() != batch.index:  # launches go to the current device
        with torch.cuda.device(batch.index):
            return kv_attend(pool, geom, layer, batch, q, scale=scale, out=out, lse=lse, workspace=workspace,
                             stream=stream)
    if scale is None and geom.planes == 1:
        warnings.warn("kv_attend: no scale given for a latent pool; 576 ** -0.5 is taken, which is not that of the "
                      "model's heads", stacklevel=2)
    if torch.is_grad_enabled() and (q.requires_grad or pool.requires_grad or (out is not None and out.requires_grad) or
                                    (lse is not None and lse.requires_grad)):
        raise _needs_gradients("kv_attend")
    a, dtype = _attend_desc(geom, q, scale), q.dtype
    a.q = _rows("q", q, batch, dtype)
    if out is None:
        with _on(stream):
            out = torch.empty(q.shape[0], a.q_heads, a.value_dim, dtype=dtype, device=q.device)
    a.out = _rows("out", out, batch, dtype, a.q_heads, a.value_dim, True)
    if lse is not None:
        _need(lse.dtype == torch.float32 and lse.is_contiguous() and lse.shape == q.shape[:2] and
              lse.device == batch.device, "kv_attend: lse is a contiguous float32 [tokens][heads]")
        a.lse = lse.data_ptr()
    desc = _pool(pool, geom, batch, dtype)
    if workspace is not None:
        if workspace.device != batch.device or not workspace.is_contiguous():
            raise MoriError("kv_attend: workspace is contiguous and on the batch's device", M.MORI_EINVAL)
    else:
        rc, n = M.mori_kv_attend_workspace(desc, batch.desc, a)
        check(rc, "mori_kv_attend_workspace")
        with _on(stream):
            workspace = torch.empty(n, dtype=torch.uint8, device=batch.device)
    check(M.mori_kv_attend(desc, int(layer), batch.desc, a, workspace.data_ptr(), workspace.nbytes,
                           batch.error.data_ptr(), _stream_of(batch, stream)), "mori_kv_attend")
    torch.autograd.graph.increment_version((out,) if lse is None else (out, lse))
    return out
