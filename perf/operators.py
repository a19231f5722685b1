"""The operators behind the embedding cache: what a sequence model does with the rows of a history.

A ranking model that reads histories keeps the keys and values of their tokens in pages, and scores
candidates against them.  Three operators carry that, each reached through
paper_2210_08804_amd.binding:

  extend   hps_seq_extend: pages for the tokens that the requests add, where each of them goes
  rotate   hps_seq_append / hps_seq_rope: queries and keys turned by their positions, keys and values
           written to their pages; the gradient of the turning
  attend   hps_seq_attention: every candidate's tokens against the history that its group shares and
           against its own tokens

A case is a dict of plain values, `prepare` builds what a program holds before the call, `run` is one
pass, `exact` the definition in 64 bits.  Lengths are a fixed set of numbers in an order that the seed
deals, so that the work of a case is known from the case.
"""
import math

import numpy as np
import torch

own = False

OPS = ("extend", "rotate", "attend")
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
BASE = 10000.0


def listed():
    return [
        # one decoding step of a small batch: a token per request
        dict(name="extend_decode_64", op="extend", requests=64, past=512, new=1, share=1.0, block=16),
        # a scheduler's ordinary step: most requests add a token, some a chunk of their prompt
        dict(name="extend_mixed_1000", op="extend", requests=1000, past=4096, new=511, share=0.1, block=32),
        # histories of many users taken in at once
        dict(name="extend_histories_8192", op="extend", requests=8192, past=64, new=255, share=1.0, block=64),
        # one decoding step of a small batch, full rotation
        dict(name="append_decode_26", op="rotate", tokens=26, q_heads=16, kv_heads=4, dim=128, rot=128, pairs="half", dtype="bf16", block=16, grad=False),
        # a chunk of prompts, half of each head is turned, pairs are neighbours
        dict(name="append_prompts_8192", op="rotate", tokens=8192, q_heads=32, kv_heads=8, dim=128, rot=64, pairs="neighbours", dtype="bf16", block=32, grad=False),
        # odd head sizes and an odd number of tokens
        dict(name="append_ragged_5003_d96", op="rotate", tokens=5003, q_heads=12, kv_heads=12, dim=96, rot=96, pairs="half", dtype="f16", block=64, grad=False),
        # the gradient of queries and keys of a training batch in 32 bits
        dict(name="rotate_gradient_16384", op="rotate", tokens=16384, q_heads=16, kv_heads=16, dim=64, rot=64, pairs="half", dtype="f32", block=64, grad=True),
        # the smallest request: eight candidates of one user with a short history
        dict(name="score_8_candidates", op="attend", groups=1, requests=8, new=1, prefix=500, length=16, q_heads=8, kv_heads=8, dim=64, dtype="bf16", block=16),
        # an ordinary one: a few hundred candidates, thousands of events
        dict(name="score_256_candidates", op="attend", groups=1, requests=256, new=1, prefix=8192, length=64, q_heads=16, kv_heads=4, dim=128, dtype="bf16", block=32),
        # a batch of users with ragged histories, candidates of one to five tokens
        dict(name="score_26_users", op="attend", groups=26, requests=39, new=5, prefix=3000, length=37, q_heads=8, kv_heads=2, dim=64, dtype="f16", block=16),
        # few requests behind a very long context: bound by reading it
        dict(name="decode_4_long_prefix", op="attend", groups=1, requests=4, new=1, prefix=200003, length=700, q_heads=32, kv_heads=8, dim=128, dtype="bf16", block=64),
        # the largest: a whole candidate set against a long history
        dict(name="score_512_long_history", op="attend", groups=1, requests=512, new=1, prefix=32768, length=128, q_heads=32, kv_heads=8, dim=128, dtype="bf16", block=64),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, no dearer than the largest listed one of its kind."""
    op = rng.choices(OPS, weights=(2, 3, 5))[0]
    block = rng.choice((16, 32, 64))
    if op == "extend":
        c = dict(op=op, requests=_log_uniform(rng, 1, 8192), past=_log_uniform(rng, 1, 4096), new=_log_uniform(rng, 1, 512), share=rng.choice((0.1, 0.5, 1.0)), block=block)
        c["new"] = max(1, min(c["new"], (1 << 20) // max(1, int(c["requests"] * c["share"]))))
        c["past"] = max(1, min(c["past"], (1 << 22) // c["requests"]))
        return c
    dim = rng.choice((32, 64, 64, 96, 128, 128))
    q_heads, kv_heads = rng.choice(((8, 8), (8, 2), (16, 4), (32, 8), (12, 12), (16, 1), (5, 5)))
    if op == "rotate":
        grad = rng.random() < 0.4
        return dict(op=op, tokens=_log_uniform(rng, 1, 8192), q_heads=q_heads, kv_heads=kv_heads, dim=dim, rot=dim if rng.random() < 0.6 else dim // 2,
                    pairs=rng.choice(("half", "neighbours")), dtype=rng.choice(("f32", "f16", "bf16") if grad else ("f16", "bf16", "bf16")), block=block, grad=grad)
    c = dict(op=op, groups=rng.choice((1, 1, 1, _log_uniform(rng, 2, 32))), requests=_log_uniform(rng, 1, 512), new=rng.choice((1, 1, 1, 3, 8, 32)), prefix=_log_uniform(rng, 64, 131072),
             length=_log_uniform(rng, 1, 1024), q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=rng.choice(("f16", "bf16", "bf16")), block=block)
    c["requests"] = max(1, min(c["requests"], 1024 // c["groups"]))
    c["length"] = max(c["length"], c["new"])
    most = 1 << 29                                          # scores of the listed cases' largest
    c["prefix"] = max(64, min(c["prefix"], (1 << 19) // c["groups"], most // (c["groups"] * c["requests"] * c["new"] * q_heads)))
    c["length"] = max(c["new"], min(c["length"], (1 << 17) // (c["groups"] * c["requests"])))
    return c


# ---- what a case's lengths are

def _spread(n, least, most):
    """n lengths from `most` down to `least`, evenly."""
    return np.linspace(most, least, n).round().astype(np.int64) if n > 1 else np.array([most])


def _extend_lengths(c):
    n, some = c["requests"], max(1, int(c["requests"] * c["share"]))
    new = np.ones(n, dtype=np.int64)
    new[:some] = _spread(some, 1, c["new"])
    return _spread(n, 0, c["past"]), new


def _attend_lengths(c):
    n = c["groups"] * c["requests"]
    new = _spread(n, 1, c["new"])
    return _spread(c["groups"], max(1, c["prefix"] // 16), c["prefix"]), np.maximum(new, _spread(n, 1, c["length"])), new


def _tables(rng, lens, block, width, blocks):
    """A table of each length's blocks, dealt from the list `blocks`; -1 behind them."""
    need = -(-lens // block)
    table = np.full((len(lens), width), -1, dtype=np.int32)
    inside = np.arange(width)[None, :] < need[:, None]
    table[inside] = blocks[: int(need.sum())]
    return table


# ---- the inputs

def _cos_sin(rot, positions):
    """[positions][rot/2][2] fp32, from angles in 64 bits."""
    angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * torch.pow(BASE, -torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    return torch.stack((angle.cos(), angle.sin()), dim=-1).float().contiguous()


def prepare(case, seed):
    rng = np.random.RandomState(seed % (1 << 32))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    s = dict(case=case)
    if case["op"] == "extend":
        past, new = _extend_lengths(case)
        past, new = rng.permutation(past), rng.permutation(new)
        block, n = case["block"], case["requests"]
        width = -(-(case["past"] + case["new"]) // block)
        kept, need = -(-past // block), -(-(past + new) // block)
        blocks = rng.permutation(int(need.sum()) + 64)
        left = blocks[int(kept.sum()):]
        free = np.concatenate([left, np.zeros(len(blocks) - len(left), dtype=left.dtype)])   # the list has room for every block
        empty = lambda *shape: torch.empty(*shape, dtype=torch.int32, device="cuda")  # noqa: E731
        tokens = int(new.sum())
        s.update(past=i32(past), new=i32(new), start=i32(rng.randint(0, 4096, n)), free=i32(free), n_free=i32([len(left)]), table=i32(_tables(rng, past, block, width, blocks)),
                 offsets=empty(n + 1), lens=empty(n), slots=empty(tokens + tokens // 8), positions=empty(tokens + tokens // 8), info=empty(4))
        return s
    dtype, D = TYPES[case["dtype"]], case["dim"]
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen, dtype=torch.float32).to(dtype)  # noqa: E731
    Hq, Hk, block = case["q_heads"], case["kv_heads"], case["block"]
    if case["op"] == "rotate":
        T = case["tokens"]
        # queries, keys and values as one projection leaves them, side by side in a token's row
        row = normal(T, (Hq + 2 * Hk) * D).view(T, Hq + 2 * Hk, D)
        s.update(q=row[:, :Hq], k=row[:, Hq:Hq + Hk], v=row[:, Hq + Hk:], positions=i32(rng.randint(0, 8192, T)), table=_cos_sin(case["rot"], 8192),
                 q_out=torch.empty(T, Hq, D, device="cuda", dtype=dtype), k_out=torch.empty(T, Hk, D, device="cuda", dtype=dtype))
        if not case["grad"]:
            n_blocks = -(-T // block) + 8
            s.update(slots=i32(rng.permutation(n_blocks * block)[:T]), k_pages=normal(n_blocks, block, Hk, D), v_pages=normal(n_blocks, block, Hk, D))
        return s
    prefix, lens, new = _attend_lengths(case)
    prefix, deal = rng.permutation(prefix), rng.permutation(len(lens))
    lens, new = lens[deal], new[deal]
    n = len(lens)
    need = int((-(-prefix // block)).sum()), int((-(-lens // block)).sum())
    n_blocks = need[0] + need[1] + 8
    blocks = rng.permutation(n_blocks)
    T = int(new.sum())
    group_offsets = np.arange(case["groups"] + 1) * case["requests"]
    offsets = np.concatenate([[0], np.cumsum(new)])
    s.update(q=normal(T, Hq, D) * 1.5, k_pages=normal(n_blocks, block, Hk, D), v_pages=normal(n_blocks, block, Hk, D),
             prefix_table=i32(_tables(rng, prefix, block, -(-case["prefix"] // block), blocks)), prefix_lens=i32(prefix), group_offsets=i32(group_offsets),
             block_table=i32(_tables(rng, lens, block, -(-case["length"] // block), blocks[need[0]:])), lens=i32(lens), offsets=i32(offsets),
             out=torch.empty(T, Hq, D, device="cuda", dtype=dtype), lse=torch.empty(T, Hq, device="cuda"),
             max_group=int(np.diff(offsets[group_offsets]).max()))
    if own:
        s["session"] = _Session(T * Hq, D)
    return s


class _Session:
    """The attention's scratch memory, which a program keeps as long as it runs."""

    def __init__(self, rows, dim):
        from paper_2210_08804_amd import binding
        self.binding, self.handle = binding, binding.hps_seq_attention_create(rows, dim)

    def __del__(self):
        self.binding.hps_seq_attention_destroy(self.handle)


# ---- one pass

def run(s):
    c = s["case"]
    return (_run_own if own else _run_plain)[c["op"]](s, c)


def _own_extend(s, c):
    from paper_2210_08804_amd import binding as B
    B.hps_seq_extend(s["past"], s["new"], c["block"], s["free"], s["n_free"], s["table"], s["offsets"], s["lens"], s["slots"], s["positions"], s["info"], start=s["start"])
    return s["table"], s["offsets"], s["lens"], s["slots"], s["positions"], s["info"]


def _own_rotate(s, c):
    from paper_2210_08804_amd import binding as B
    if c["grad"]:
        B.hps_seq_rope(s["q"], s["q_out"], s["positions"], s["table"], k=s["k"], k_out=s["k_out"], interleaved=c["pairs"] == "neighbours", inverse=True)
        return s["q_out"], s["k_out"]
    B.hps_seq_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["slots"], q=s["q"], q_out=s["q_out"], positions=s["positions"], table=s["table"], interleaved=c["pairs"] == "neighbours")
    return s["q_out"], s["k_pages"], s["v_pages"]


def _own_attend(s, c):
    from paper_2210_08804_amd import binding as B
    B.hps_seq_attention(s["session"].handle, s["q"], s["k_pages"], s["v_pages"], s["block_table"], s["lens"], s["offsets"], s["out"], prefix_table=s["prefix_table"],
                        prefix_lens=s["prefix_lens"], group_offsets=s["group_offsets"], lse=s["lse"], max_new=c["new"], max_len=c["length"], max_prefix=c["prefix"], max_group=s["max_group"])
    return s["out"], s["lse"]


_run_own = {"extend": _own_extend, "rotate": _own_rotate, "attend": _own_attend}


def _plain_extend(s, c):
    block, table = c["block"], s["table"]
    n, width, most = table.shape[0], table.shape[1], s["slots"].numel()
    past, new = s["past"].long(), s["new"].long()
    lens = past + new
    offsets = torch.cat((new.new_zeros(1), new.cumsum(0)))
    kept, need = (past + block - 1) // block, (lens + block - 1) // block
    first = (need - kept).cumsum(0) - (need - kept)             # of the request's new blocks among all new ones
    at = torch.arange(width, device=past.device)[None, :]
    nth = first[:, None] + at - kept[:, None]
    n_free = s["n_free"].long()
    fresh = (at >= kept[:, None]) & (at < need[:, None])
    from_list = s["free"][(n_free - 1 - nth).clamp(0, s["free"].numel() - 1)]
    table.copy_(torch.where(fresh, from_list, table))           # the last blocks of the list go first
    token = torch.arange(most, device=past.device)
    r = torch.searchsorted(offsets[1:], token, right=True).clamp(max=n - 1)
    inside = token < offsets[-1]
    at_own = past[r] + token - offsets[r]
    slot = table[r, (at_own // block).clamp(max=width - 1)].long() * block + at_own % block
    minus = token.new_full((), -1)
    slots, positions = torch.where(inside, slot, minus), torch.where(inside, at_own + s["start"].long()[r], minus)
    taken = (need - kept).sum()
    zero = taken.new_zeros(1)
    info = torch.cat((n_free - taken, offsets[-1:], zero, zero))
    return table, offsets.int(), lens.int(), slots.int(), positions.int(), info.int()


def _turned(x, positions, table, pairs, inverse):
    """x [T, H, D] with its leading 2 * table.shape[1] values turned, pair by pair, in 32 bits."""
    dtype, half = x.dtype, table.shape[1]
    x = x.float()
    cos, sin = table[positions.long(), None, :, 0], table[positions.long(), None, :, 1]
    sin = -sin if inverse else sin
    part = x[..., : 2 * half]
    a, b = (part[..., :half], part[..., half:]) if pairs == "half" else (part[..., 0::2], part[..., 1::2])
    u, v = a * cos - b * sin, a * sin + b * cos
    part = torch.cat((u, v), dim=-1) if pairs == "half" else torch.stack((u, v), dim=-1).flatten(-2)
    return torch.cat((part, x[..., 2 * half:]), dim=-1).to(dtype)


def _plain_rotate(s, c):
    q = _turned(s["q"], s["positions"], s["table"], c["pairs"], c["grad"])
    k = _turned(s["k"], s["positions"], s["table"], c["pairs"], c["grad"])
    if c["grad"]:
        return q, k
    at = s["slots"].long()
    s["k_pages"].view(-1, *k.shape[1:])[at] = k
    s["v_pages"].view(-1, *k.shape[1:])[at] = s["v"]
    return q, s["k_pages"], s["v_pages"]


def _part(q, k_pages, v_pages, table, lens, first, scale):
    """Attention over one table per row of q [N, M, Hq, D], the M-th query seeing the keys below min(lens, first + M): per query its maximum, sum and weighted values."""
    N, M, Hq, D = q.shape
    Hk = k_pages.shape[2]
    k = k_pages[table.long().clamp(min=0)].flatten(1, 2).float().permute(0, 2, 3, 1).contiguous()       # [N, Hk, D, L]
    v = v_pages[table.long().clamp(min=0)].flatten(1, 2).float().transpose(1, 2).contiguous()           # [N, Hk, L, D]
    L = v.shape[2]
    rows = q.float().reshape(N, M, Hk, Hq // Hk, D).permute(0, 2, 1, 3, 4).reshape(N, Hk, M * (Hq // Hk), D)
    scores = torch.matmul(rows, k).mul_(scale).view(N, Hk, M, Hq // Hk, L)
    at = torch.arange(L, device=q.device)
    sees = (at < lens.long()[:, None, None]) & (at <= first.long()[:, None, None] + torch.arange(M, device=q.device)[:, None])      # [N, M, L]
    scores.masked_fill_(~sees[:, None, :, None, :], -math.inf)
    top = scores.amax(-1, keepdim=True)
    scores.sub_(top.clamp(min=torch.finfo(torch.float32).min)).exp_()
    total = scores.sum(-1)
    back = lambda x: x.permute(0, 2, 1, 3, *range(4, x.dim())).reshape(N, M, Hq, *x.shape[4:])  # noqa: E731
    values = torch.matmul(scores.view(N, Hk, M * (Hq // Hk), L), v).view(N, Hk, M, Hq // Hk, D)
    return back(top.squeeze(-1)), back(total), back(values)


def _plain_attend(s, c):
    q, offsets, groups = s["q"], s["offsets"].long(), s["group_offsets"].long()
    T, scale = q.shape[0], 1.0 / math.sqrt(q.shape[2])
    token = torch.arange(T, device=q.device)
    request = torch.searchsorted(offsets[1:].contiguous(), token, right=True)
    group = torch.searchsorted(groups[1:].contiguous(), request, right=True)
    parts = []
    for rows, starts, most, table, lens, first in (
            (group, offsets[groups], s["max_group"], s["prefix_table"], s["prefix_lens"], s["prefix_lens"]),
            (request, offsets, c["new"], s["block_table"], s["lens"], s["lens"].long() - offsets.diff())):
        at = token - starts[rows]
        padded = q.new_zeros(table.shape[0], most, *q.shape[1:])
        padded[rows, at] = q
        parts.append([x[rows, at] for x in _part(padded, s["k_pages"], s["v_pages"], table, lens, first, scale)])
    (m0, l0, o0), (m1, l1, o1) = parts
    top = torch.maximum(m0, m1)
    w0, w1 = (m0 - top).exp(), (m1 - top).exp()
    total = l0 * w0 + l1 * w1
    return ((o0 * w0[..., None] + o1 * w1[..., None]) / total[..., None]).to(q.dtype), top + total.log()


_run_plain = {"extend": _plain_extend, "rotate": _plain_rotate, "attend": _plain_attend}


# ---- what a pass cannot do without

def work(case):
    c = case
    if c["op"] == "extend":
        past, new = _extend_lengths(c)
        n, tokens = c["requests"], int(new.sum())
        fresh = tokens / c["block"]                                   # about: a new block for every `block` new tokens
        return {"bytes": 4 * (3 * n + 2 * n + fresh * 2 + n + 2 * (tokens + tokens // 8)), "flops": 0}
    D, Hq, Hk, size = c["dim"], c["q_heads"], c["kv_heads"], BYTES[c["dtype"]]
    if c["op"] == "rotate":
        T = c["tokens"]
        heads = Hq + Hk + (0 if c["grad"] else Hk)
        table = min(T, 8192) * c["rot"] * 4
        return {"bytes": 2 * T * heads * D * size + table + 8 * T, "flops": 3 * T * (Hq + Hk) * c["rot"]}
    prefix, lens, new = _attend_lengths(c)
    T, keys = int(new.sum()), int(prefix.sum() + lens.sum())
    scores = int((prefix * c["requests"]).sum()) * T / len(lens) + float((new * (lens - (new - 1) / 2)).sum())
    return {"bytes": 2 * T * Hq * D * size + 4 * T * Hq + 2 * keys * Hk * D * size, "flops": 4 * scores * Hq * D}


# ---- the definition in 64 bits

def exact(case, seed):
    c = case
    if c["op"] == "extend":
        return None
    s = _inputs(case, seed)
    if c["op"] == "rotate":
        inverse = c["grad"]
        angle = s["positions"].double()[:, None] * torch.tensor([BASE ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)], device="cuda", dtype=torch.float64)
        turn = torch.polar(torch.ones_like(angle), -angle if inverse else angle)[:, None, :]
        outs = []
        for x in (s["q"], s["k"]):
            x = x.double()
            half = c["rot"] // 2
            if c["pairs"] == "half":
                z = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous()) * turn
                y = torch.cat((z.real, z.imag, x[..., 2 * half:]), dim=-1)
            else:
                z = torch.view_as_complex(x[..., :2 * half].reshape(*x.shape[:2], half, 2).contiguous()) * turn
                y = torch.cat((torch.view_as_real(z).flatten(-2), x[..., 2 * half:]), dim=-1)
            outs.append(y)
        if inverse:
            return tuple(outs)
        pages = []
        for name, new in (("k_pages", outs[1]), ("v_pages", s["v"].double())):
            p = s[name].double()
            p.view(-1, *new.shape[1:]).index_copy_(0, s["slots"].long(), new)
            pages.append(p)
        return outs[0], pages[0], pages[1]
    block, D, Hq, Hk = c["block"], c["dim"], c["q_heads"], c["kv_heads"]
    offsets, lens, prefix = s["offsets"].tolist(), s["lens"].tolist(), s["prefix_lens"].tolist()
    if len(lens) * max(1, c["prefix"] * Hk * D // (1 << 24)) > 4096:
        return None                                                   # over 20 seconds

    def keys_of(pages, table, length):
        blocks = table[: -(-length // block)].long()
        return pages[blocks].reshape(-1, Hk, D)[:length].double()

    out = torch.empty(s["q"].shape, device="cuda", dtype=torch.float64)
    lse = torch.empty(s["q"].shape[:2], device="cuda", dtype=torch.float64)
    for g, shared in enumerate(prefix):
        pk, pv = (keys_of(p, s["prefix_table"][g], shared) for p in (s["k_pages"], s["v_pages"]))
        for r in range(g * c["requests"], (g + 1) * c["requests"]):
            k = torch.cat((pk, keys_of(s["k_pages"], s["block_table"][r], lens[r]))).transpose(0, 1)
            v = torch.cat((pv, keys_of(s["v_pages"], s["block_table"][r], lens[r]))).transpose(0, 1)
            n = offsets[r + 1] - offsets[r]
            q = s["q"][offsets[r]:offsets[r + 1]].double().view(n, Hk, Hq // Hk, D).transpose(0, 1).reshape(Hk, n * (Hq // Hk), D)
            scores = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(D)
            hidden = torch.arange(k.shape[1], device="cuda")[None, :] > shared + lens[r] - n + torch.arange(n, device="cuda").repeat_interleave(Hq // Hk)[:, None]
            scores = scores.masked_fill(hidden, -math.inf)
            p = torch.softmax(scores, dim=-1)
            out[offsets[r]:offsets[r + 1]] = torch.bmm(p, v.contiguous()).view(Hk, n, Hq // Hk, D).transpose(0, 1).reshape(n, Hq, D)
            lse[offsets[r]:offsets[r + 1]] = torch.logsumexp(scores, dim=-1).view(Hk, n, Hq // Hk).transpose(0, 1).reshape(n, Hq)
    return out, lse


def _inputs(case, seed):
    return prepare(case, seed)
