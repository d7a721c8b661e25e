"""Cases of the operators that write and read the paged KV pool for a model.

  append         kv_append on a K/V pool: new keys (rotated) and values into the
                 programs' pages, the queries rotated in the same call
  append_latent  kv_append on a compressed-latent pool (one row: latent, then the
                 rotated key part)
  attend         kv_attend on a K/V pool: causal attention of each program's new
                 tokens over its pages, grouped heads, ragged batches
  attend_latent  kv_attend on a latent pool (rows of 512 + 64, the latent is the
                 value), queries already in the latent space

A case names a batch: ``seqs`` programs with about ``new`` new tokens each behind
about ``ctx`` cached ones (0: whole prompts), and ``decode`` further programs
with one new token.  Token counts and contexts follow from the case alone;
values, page order and the programs' order follow from the seed.  ``own`` chooses
between the plain form (elementary torch operations in 32 bits) and the
framework's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

LATENT, ROPE = 512, 64  # a latent row: the compressed part, then the rotated key part
THETA = 500000.0
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _case(kind, dtype, seqs, new, ctx, q_heads, kv_heads=1, dim=LATENT + ROPE, block=16, ragged=True, decode=0,
          style="half", name=None):
    c = {"kind": kind, "dtype": dtype, "seqs": seqs, "new": new, "ctx": ctx, "q_heads": q_heads,
         "kv_heads": kv_heads, "dim": dim, "block": block, "ragged": ragged, "decode": decode, "style": style}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the tiny workload's eight agents, one token each: launch latency
        _case("append", "fp16", 8, 1, 700, 8, 4, 64, name="append_step_tiny"),
        # a prefill step of five Llama-3-8B programs, ragged chunks
        _case("append", "bf16", 5, 4096, 6000, 32, 8, 128, name="append_chunk_8b"),
        # every program of the compressed-latent workload takes one token
        _case("append_latent", "bf16", 256, 1, 1024, 128, block=64, style="pairs", name="append_latent_step"),
        # the tiny workload's decode step
        _case("attend", "fp16", 8, 1, 700, 8, 4, 64, name="step_tiny"),
        # decode step of the Llama-3-8B workload's 64 programs (lognormal contexts)
        _case("attend", "bf16", 64, 1, 16384, 32, 8, 128, name="step_8b"),
        # one agent with a long context on one rank at tensor parallelism 8: a single key head
        _case("attend", "bf16", 1, 1, 65501, 8, 1, 128, name="step_long_tp8"),
        # resumed agents send a tool's output: chunks of hundreds of tokens behind long contexts
        _case("attend", "bf16", 4, 512, 12000, 32, 8, 128, name="chunk_8b"),
        # one chunk of a prompt scheduled with 31 decoding programs, tensor parallelism 2 of Llama-3-70B
        _case("attend", "bf16", 1, 777, 6144, 32, 4, 128, decode=31, name="mixed_70b_tp2"),
        # whole prompts of programs admitted from Waiting, packed
        _case("attend", "bf16", 3, 8192, 0, 32, 8, 128, name="prompt_8b"),
        # decode step over the latent pool, one rank's 16 heads
        _case("attend_latent", "bf16", 256, 1, 8192, 16, block=64, name="latent_step_16"),
        # the same with all 128 heads on one GPU
        _case("attend_latent", "bf16", 48, 1, 8192, 128, block=64, name="latent_step_128"),
        # chunks of two programs over the latent pool
        _case("attend_latent", "bf16", 2, 384, 4096, 32, block=64, name="latent_chunk_32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(8, 4, 64), (12, 4, 64), (16, 16, 64), (32, 8, 128), (64, 8, 128), (32, 4, 128), (16, 2, 128), (8, 1, 128),
         (10, 2, 128), (16, 16, 128)]


def draw(rng):
    while True:
        kind = rng.choice(["append"] * 2 + ["append_latent"] + ["attend"] * 5 + ["attend_latent"] * 3)
        latent = kind.endswith("latent")
        q, kv, dim = (rng.choice([16, 32, 64, 128]), 1, LATENT + ROPE) if latent else rng.choice(HEADS)
        seqs = _log_int(rng, 1, 256 if latent else 64)
        if kind.startswith("append"):
            new, ctx = _log_int(rng, 1, 4096), _log_int(rng, 16, 8192)
        else:
            shape = rng.choice(["step", "step", "few", "chunk", "prompt"])
            new = {"step": 1, "few": rng.randint(2, 16)}.get(shape) or _log_int(rng, 17, 2048 if latent else 8192)
            ctx = 0 if shape == "prompt" else _log_int(rng, 64, 65536)
        decode = rng.choice([0, 0, _log_int(rng, 1, 64)]) if new > 1 else 0
        case = _case(kind, rng.choice(["bf16", "bf16", "fp16"]), seqs, new, ctx, q, kv, dim,
                     rng.choice([64, 64, 16] if latent else [16, 16, 32, 64]), rng.random() < 0.8, decode,
                     rng.choice(["half", "pairs"]))
        n, length = _lengths(case)
        w = work(case)
        pool = int(length.sum()) * _row(case) * _planes(case)
        if w["flops"] > 8e11 or w["bytes"] > 4e9 or pool > (4e8 if kind.startswith("append") else 4e9):
            continue
        return case


# --------------------------------------------------------------------------
# shapes
# --------------------------------------------------------------------------
def _lengths(case):
    """New tokens of each program and its length in the pool with them."""
    rng = np.random.default_rng([case[k] for k in ("seqs", "new", "ctx", "q_heads", "decode", "block")])
    seqs, extra = case["seqs"], case["decode"]
    n = np.full(seqs, case["new"], np.int64)
    if case["ragged"] and case["new"] > 1:
        n = np.maximum(1, (case["new"] * np.exp(-0.7 * rng.random(seqs))).astype(np.int64))
        n[0] = case["new"]
    n = np.concatenate([n, np.ones(extra, np.int64)])
    base = case["ctx"] or (case["new"] if extra else 0)
    cached = np.full(n.size, base, np.int64)
    if case["ragged"] and n.size > 1:
        cached = np.clip(base * np.exp(0.5 * rng.standard_normal(n.size)), base // 4, 4 * base).astype(np.int64)
    if not case["ctx"]:
        cached[:seqs] = 0
    return n, cached + n


def _latent(case):
    return case["kind"].endswith("latent")


def _planes(case):
    return 1 if _latent(case) else 2


def _row(case):
    return 2 * case["kv_heads"] * case["dim"]


def _rot(case):
    return ROPE if _latent(case) else case["dim"]


def work(case):
    n, length = _lengths(case)
    T, q, kv, dim = int(n.sum()), case["q_heads"], case["kv_heads"], case["dim"]
    if case["kind"].startswith("append"):
        row = dim if _latent(case) else 2 * kv * dim
        turned = (q + kv) * _rot(case)
        return {"bytes": 2 * 2 * T * (row + q * _rot(case)) + 4 * T * _rot(case), "flops": 3 * T * turned}
    value = LATENT if _latent(case) else dim
    pairs = sum(int(a) * int(l) - int(a) * (int(a) - 1) // 2 for a, l in zip(n, length))
    read = int(length.sum()) * _row(case) * _planes(case)
    return {"bytes": read + 2 * T * q * (dim + value), "flops": 2 * (dim + value) * q * pairs}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
class Geometry:
    """Of the pool: one layer of a model's."""

    def __init__(self, planes, block_tokens, row_bytes, num_blocks):
        self.layers, self.planes = 1, planes
        self.block_tokens, self.row_bytes, self.num_blocks = block_tokens, row_bytes, num_blocks


class State:
    pass


def _normal(gen, shape, dtype, scale=1.0):
    x = torch.empty(shape, dtype=dtype, device="cuda").normal_(generator=gen)
    return x if scale == 1.0 else x.mul_(scale)


def _pages(rng, count):
    """Page ids of a used pool: chunks of mean 4 consecutive pages, shuffled."""
    cuts = np.cumsum(rng.geometric(0.25, size=count))
    cuts = np.concatenate([[0], cuts[cuts < count], [count]])
    order = rng.permutation(cuts.size - 1)
    return np.concatenate([np.arange(cuts[i], cuts[i + 1]) for i in order]).astype(np.int32)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def prepare(case, seed):
    st = State()
    st.case = case
    st.n, st.length = _lengths(case)
    rng = np.random.default_rng([seed, 0x6B76])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype, B, T = DTYPES[case["dtype"]], st.n.size, int(st.n.sum())
    q, kv, dim, bt = case["q_heads"], case["kv_heads"], case["dim"], case["block"]
    # tables: programs in another order than the batch, some blocks to grow into, free pages between
    blocks = -(-st.length // bt) + np.arange(B) % 3
    st.prog = rng.permutation(B).astype(np.int32)
    per_program = np.empty(B, np.int64)
    per_program[st.prog] = blocks
    st.tbl_off = np.concatenate([[0], np.cumsum(per_program)]).astype(np.int32)
    total = int(blocks.sum())
    st.pages = _pages(rng, total + total // 16 + 1)[:total]
    nb = total + total // 16 + 1
    st.geom = Geometry(_planes(case), bt, _row(case), nb)
    st.pool = _normal(gen, (_planes(case), nb, bt, kv, dim), dtype)
    st.seq_off = np.concatenate([[0], np.cumsum(st.n)]).astype(np.int32)
    st.d_tbl, st.d_tbl_off, st.d_prog = _dev(st.pages), _dev(st.tbl_off), _dev(st.prog)
    st.d_seq_off, st.d_length = _dev(st.seq_off), _dev(st.length.astype(np.int32))
    if case["kind"].startswith("append"):
        r = _rot(case)
        angle = torch.arange(int(st.length.max()), dtype=torch.float64)[:, None] * \
            THETA ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
        st.rope = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
        if _latent(case):
            # the down-projection's output holds latent and key part side by side
            row = _normal(gen, (T, 1, dim), dtype)
            st.k, st.v = row[..., :LATENT], row[..., LATENT:]
            st.q = _normal(gen, (T, q, r), dtype)
            st.q_out = _normal(gen, (T, q, dim), dtype)  # its latent part is another product's output
        else:
            # the fused projection's output: queries, keys, values side by side
            x = _normal(gen, (T, q + 2 * kv, dim), dtype)
            st.q, st.k, st.v = x[:, :q], x[:, q:q + kv], x[:, q + kv:]
            st.q_out = torch.empty(T, q, dim, dtype=dtype, device="cuda")
    else:
        st.q = _normal(gen, (T, q, dim), dtype, 2.5)
        st.out = torch.empty(T, q, LATENT if _latent(case) else dim, dtype=dtype, device="cuda")
    st.scale = (192 if _latent(case) else dim) ** -0.5  # latent: of the 128 + 64 dimensions before compression
    if own:
        _plan(st)
    return st


def _plan(st):
    from paper_2606_00866_amd import attention as A

    st.batch = A.TokenBatch(st.geom, st.d_tbl_off, st.d_tbl, st.d_seq_off, st.d_length, program=st.d_prog,
                            num_tokens=int(st.n.sum()), max_new=int(st.n.max()), max_kv=int(st.length.max()))
    if not st.case["kind"].startswith("append"):
        st.workspace = A.kv_attend_workspace(st.geom, st.batch, st.q)


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(state):
    st, kind = state, state.case["kind"]
    if not own:
        return _plain_append(st) if kind.startswith("append") else _plain_attend(st)
    from paper_2606_00866_amd import attention as A

    if kind == "append":
        A.kv_append(st.pool, st.geom, 0, st.batch, st.k, st.v, q=st.q, q_out=st.q_out, rope=st.rope,
                    style=st.case["style"])
        return {"pool": st.pool, "q": st.q_out}
    if kind == "append_latent":
        A.kv_append(st.pool, st.geom, 0, st.batch, st.k, st.v, q=st.q, q_out=st.q_out[..., LATENT:], rope=st.rope,
                    style=st.case["style"])
        return {"pool": st.pool, "q": st.q_out}
    A.kv_attend(st.pool, st.geom, 0, st.batch, st.q, scale=st.scale, out=st.out, workspace=st.workspace)
    return st.out


def _slots(st):
    """Page and row of every new token, and its position."""
    bt = st.case["block"]
    n = st.d_seq_off[1:] - st.d_seq_off[:-1]
    T = int(st.n.sum())
    seq = torch.repeat_interleave(torch.arange(st.n.size, device="cuda"), n.long(), output_size=T)
    pos = (st.d_length - n)[seq] + torch.arange(T, device="cuda") - st.d_seq_off[seq]
    page = st.d_tbl[(st.d_tbl_off[st.d_prog.long()][seq] + pos // bt).long()]
    return page.long(), (pos % bt).long(), pos.long()


def _rotate(x, table, style):
    """x [T][H][r] in 32 bits, table [T][r]: cosines, then sines."""
    r = x.shape[-1]
    c, s = table[:, None, :r // 2], table[:, None, r // 2:]
    if style == "half":
        a, b = x[..., :r // 2], x[..., r // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)


def _plain_append(st):
    page, row, pos = _slots(st)
    table, style = st.rope[pos], st.case["style"]
    q = _rotate(st.q.float(), table, style).to(st.q.dtype)
    if _latent(st.case):
        st.pool[0, page, row, :, :LATENT] = st.k
        st.pool[0, page, row, :, LATENT:] = _rotate(st.v.float(), table, style).to(st.v.dtype)
        st.q_out[..., LATENT:] = q
    else:
        st.pool[0, page, row] = _rotate(st.k.float(), table, style).to(st.k.dtype)
        st.pool[1, page, row] = st.v
        st.q_out.copy_(q)
    return {"pool": st.pool, "q": st.q_out}


def _plain_attend(st):
    case = st.case
    H, kv, bt = case["q_heads"], case["kv_heads"], case["block"]
    G = H // kv
    for b in range(st.n.size):
        n, L, p = int(st.n[b]), int(st.length[b]), int(st.prog[b])
        t0, off = int(st.seq_off[b]), int(st.tbl_off[p])
        pages = st.d_tbl[off:off + -(-L // bt)].long()
        rows = [st.pool[i, pages].flatten(0, 1)[:L].float().transpose(0, 1) for i in range(_planes(case))]
        keys = rows[0].transpose(1, 2).contiguous()  # [kv][dim][L]
        values = (rows[0][..., :LATENT] if _latent(case) else rows[1]).contiguous()  # [kv][L][value]
        limit = torch.arange(L - n, L, device="cuda")
        at = torch.arange(L, device="cuda")
        step = max(1, (1 << 28) // (H * L))
        for i in range(0, n, step):
            m = min(step, n - i)
            q = st.q[t0 + i:t0 + i + m].float().unflatten(1, (kv, G)).transpose(0, 1).flatten(1, 2)  # [kv][m * G][dim]
            s = torch.bmm(q.contiguous(), keys).mul_(st.scale)
            masked = at[None, :] > limit[i:i + m, None]
            s.unflatten(1, (m, G)).masked_fill_(masked[None, :, None, :], -math.inf)
            s.sub_(s.amax(-1, keepdim=True)).exp_()
            o = torch.bmm(s, values) / s.sum(-1, keepdim=True)
            st.out[t0 + i:t0 + i + m] = o.unflatten(1, (m, G)).transpose(0, 1).flatten(1, 2).to(st.out.dtype)
        del keys, values, rows
    return st.out


# --------------------------------------------------------------------------
# the definition in 64 bits
# --------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    return _exact_append(st) if case["kind"].startswith("append") else _exact_attend(st)


def _exact_append(st):
    """Token by token of the batch's numbering, the rotation as a product of complex numbers."""
    case, r = st.case, _rot(st.case)
    T, bt = int(st.n.sum()), case["block"]
    seq = np.repeat(np.arange(st.n.size), st.n)
    pos = st.length[seq] - st.n[seq] + np.arange(T) - st.seq_off[seq]
    page = st.pages[st.tbl_off[st.prog[seq]] + pos // bt]
    at, row = _dev(page.astype(np.int64)), _dev(pos % bt)
    half = r // 2
    turn = torch.complex(st.rope[_dev(pos), :half].double(), st.rope[_dev(pos), half:].double())[:, None]

    def rotated(x):
        x = x.double()
        if case["style"] == "half":
            z = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * turn
            return torch.cat([z.real, z.imag], -1)
        return torch.view_as_real(torch.view_as_complex(x.contiguous().unflatten(-1, (half, 2))) * turn).flatten(-2)

    pool, q = st.pool.double(), st.q_out.double()
    if _latent(case):
        pool[0, at, row] = torch.cat([st.k.double(), rotated(st.v)], -1)
        q[..., LATENT:] = rotated(st.q)
    else:
        pool[0, at, row] = rotated(st.k)
        pool[1, at, row] = st.v.double()
        q = rotated(st.q)
    return {"pool": pool, "q": q}


def _exact_attend(st):
    """Head by head: the logarithm of each row's sum, then the weighted values."""
    case, w = st.case, work(st.case)
    if w["flops"] > 2e12:
        return None
    H, G = case["q_heads"], case["q_heads"] // case["kv_heads"]
    out = torch.empty(st.out.shape, dtype=torch.float64, device="cuda")
    for b in range(st.n.size):
        n, L, p = int(st.n[b]), int(st.length[b]), int(st.prog[b])
        t0 = int(st.seq_off[b])
        j = np.arange(L)
        page = _dev(st.pages[st.tbl_off[p] + j // case["block"]].astype(np.int64))
        row = _dev(j % case["block"])
        shared = range(0, H, G) if n * G <= 4096 else range(H)  # heads of a group together, or one by one
        for h in shared:
            g = G if len(shared) < H else 1
            k = st.pool[0, page, row, h // G].double()
            v = k[:, :LATENT] if _latent(case) else st.pool[1, page, row, h // G].double()
            part = max(1, (1 << 27) // (g * L))
            for i in range(0, n, part):
                m = min(part, n - i)
                s = st.q[t0 + i:t0 + i + m, h:h + g].double().flatten(0, 1) @ k.t() * st.scale
                behind = torch.ones(m, L, dtype=torch.bool, device="cuda").triu(L - n + i + 1)
                s = s.masked_fill(behind.repeat_interleave(g, 0), -math.inf)
                out[t0 + i:t0 + i + m, h:h + g] = (torch.exp(s - torch.logsumexp(s, 1, keepdim=True)) @ v) \
                    .unflatten(0, (m, g))
    return out
