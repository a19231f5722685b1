"""Histories kept in 4 bits: what stands beside the sequence operators where memory holds four times the tokens.

A ranking model with long histories norms its queries and keys head by head, turns them by their positions, and
keeps keys and values as 4-bit numbers with a scale for each 32 of a head.  Reached through
paper_2210_08804_amd.binding:

  norm      hps_seq_norm_rope: every head divided by its root mean square, weighted, turned by its position
  gradient  hps_seq_norm_rope_grad: the gradients of the heads and of the weights, for training
  append    hps_seq_append_packed: the same for queries and keys of new tokens, with keys and values rounded to 4
            bits and written to their pages; hps_seq_read_packed gives the pages' values
  attend    hps_seq_attention_packed: every candidate's tokens against the history that its group shares and
            against its own tokens, from such pages

A packed value is s * v with s = 2^x shared by 32 neighbours of a head and v one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and
their negatives; x is the least integer that leaves the largest of the 32 at most 7 * s, and v the nearest (of two
the one with the even code).  Keys are computed in 64 bits in front of that rounding, so that codes do not depend on
the order of a sum.

A case is a dict of plain values, `prepare` builds what a program holds before the call, `run` is one pass, `exact`
the definition in 64 bits.  Lengths are a fixed set of numbers in an order that the seed deals, so that the work of
a case is known from the case.
"""
import math

import numpy as np
import torch

own = False

OPS = ("norm", "gradient", "append", "attend")
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
LEAST, MOST = {"f32": -126, "f16": -23, "bf16": -126}, {"f32": 125, "f16": 13, "bf16": 125}       # exponents of scales
BASE, EPS = 10000.0, 1e-6
POSITIONS = 8192


def listed():
    return [
        # one decoding step of a small batch
        dict(name="norm_decode_26", op="norm", tokens=26, q_heads=16, kv_heads=4, dim=128, rot=128, pairs="half", dtype="bf16"),
        # a chunk of prompts, half of each head is turned, pairs are neighbours
        dict(name="norm_prompts_8192", op="norm", tokens=8192, q_heads=32, kv_heads=8, dim=128, rot=64, pairs="neighbours", dtype="bf16"),
        # a training batch of ordinary size; odd heads and an odd number of tokens
        dict(name="gradient_2003_d96", op="gradient", tokens=2003, q_heads=12, kv_heads=12, dim=96, rot=96, pairs="half", dtype="bf16"),
        # a large one in 32 bits
        dict(name="gradient_16384", op="gradient", tokens=16384, q_heads=16, kv_heads=16, dim=64, rot=64, pairs="half", dtype="f32"),
        # one decoding step of a small batch: a token per request
        dict(name="append_decode_64", op="append", tokens=64, q_heads=16, kv_heads=4, dim=128, rot=128, pairs="half", dtype="bf16", block=16, norm=True),
        # histories taken in: a chunk of prompts
        dict(name="append_prompts_8192", op="append", tokens=8192, q_heads=32, kv_heads=8, dim=128, rot=128, pairs="half", dtype="bf16", block=32, norm=True),
        # the smallest request: eight candidates of one user with a short history
        dict(name="score_8_candidates", op="attend", groups=1, requests=8, new=1, prefix=500, length=16, q_heads=8, kv_heads=8, dim=64, dtype="bf16", block=16),
        # an ordinary one: a few hundred candidates, thousands of events
        dict(name="score_256_candidates", op="attend", groups=1, requests=256, new=1, prefix=8192, length=64, q_heads=16, kv_heads=4, dim=128, dtype="bf16", block=32),
        # a batch of users with ragged histories, candidates of one to five tokens
        dict(name="score_26_users", op="attend", groups=26, requests=39, new=5, prefix=3000, length=37, q_heads=8, kv_heads=2, dim=64, dtype="f16", block=16),
        # single tokens of many requests, each behind a context of its own
        dict(name="decode_64_own_contexts", op="attend", groups=0, requests=64, new=1, prefix=0, length=8001, q_heads=32, kv_heads=8, dim=128, dtype="bf16", block=32),
        # few requests behind a very long context: bound by reading it
        dict(name="decode_4_long_prefix", op="attend", groups=1, requests=4, new=1, prefix=200003, length=700, q_heads=32, kv_heads=8, dim=128, dtype="bf16", block=64),
        # the largest: a whole candidate set against a long history
        dict(name="score_512_long_history", op="attend", groups=1, requests=512, new=1, prefix=32768, length=128, q_heads=32, kv_heads=8, dim=128, dtype="bf16", block=64),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, no dearer than the largest listed one of its kind."""
    op = rng.choices(OPS, weights=(2, 2, 2, 5))[0]
    dim = rng.choice((32, 64, 64, 96, 128, 128))
    q_heads, kv_heads = rng.choice(((8, 8), (8, 2), (16, 4), (32, 8), (12, 12), (16, 1), (5, 5)))
    block = rng.choice((16, 32, 64))
    if op != "attend":
        c = dict(op=op, tokens=_log_uniform(rng, 1, 8192), q_heads=q_heads, kv_heads=kv_heads, dim=dim, rot=dim if rng.random() < 0.6 else dim // 2,
                 pairs=rng.choice(("half", "neighbours")), dtype=rng.choice(("f16", "bf16", "bf16") if op == "append" else ("f32", "f16", "bf16")))
        return dict(c, block=block, norm=rng.random() < 0.7) if op == "append" else c
    c = dict(op=op, groups=rng.choice((0, 1, 1, 1, _log_uniform(rng, 2, 32))), requests=_log_uniform(rng, 1, 512), new=rng.choice((1, 1, 1, 3, 8, 32)), prefix=_log_uniform(rng, 64, 131072),
             length=_log_uniform(rng, 1, 1024), q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=rng.choice(("f16", "bf16", "bf16")), block=block)
    groups = max(1, c["groups"])
    c["requests"] = max(1, min(c["requests"], 1024 // groups))
    most = 1 << 29                                          # scores of the listed cases' largest
    c["prefix"] = 0 if c["groups"] == 0 else max(64, min(c["prefix"], (1 << 19) // groups, most // (groups * c["requests"] * c["new"] * q_heads)))
    if c["groups"] == 0:
        c["length"] = _log_uniform(rng, 1, 16384)
    c["length"] = max(c["new"], min(c["length"], (1 << (17 if c["groups"] else 19)) // (groups * c["requests"])))
    return c


# ---- what a case's lengths are

def _spread(n, least, most):
    """n lengths from `most` down to `least`, evenly."""
    return np.linspace(most, least, n).round().astype(np.int64) if n > 1 else np.array([most])


def _attend_lengths(c):
    n = max(1, c["groups"]) * c["requests"]
    new = _spread(n, 1, c["new"])
    prefix = _spread(c["groups"], max(1, c["prefix"] // 16), c["prefix"]) if c["groups"] else np.zeros(0, dtype=np.int64)
    return prefix, np.maximum(new, _spread(n, 1, c["length"])), new


def _tables(lens, block, width, blocks):
    """A table of each length's blocks, dealt from the list `blocks`; -1 behind them."""
    need = -(-lens // block)
    table = np.full((len(lens), width), -1, dtype=np.int32)
    inside = np.arange(width)[None, :] < need[:, None]
    table[inside] = blocks[: int(need.sum())]
    return table


# ---- 4-bit pages: a tile of [keys' codes | values' codes | keys' scales | values' scales] for each block and head

def _tile_bytes(block, dim):
    return block * dim * 17 // 16


def _quantised(x, dtype):
    """(codes, scale exponents) of x [..., dim] in 64 bits: uint8 [..., dim], int16 [..., dim / 32]."""
    g = x.unflatten(-1, (-1, 32))
    top = g.abs().amax(-1)
    mantissa, exponent = torch.frexp(top)                   # top = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = (exponent - 3 + (mantissa > 0.875).to(exponent.dtype)).clamp(LEAST[dtype], MOST[dtype])
    e = torch.where(top > 0, e, torch.full_like(e, LEAST[dtype]))
    v = torch.ldexp(g.abs(), -e[..., None])
    step = torch.where(v < 2, 0.5, torch.where(v < 4, 1.0, 2.0)).to(v.dtype)
    v = (torch.round(v / step) * step).clamp(max=6)
    code = torch.where(v < 2, v * 2, torch.where(v < 4, v + 2, v / 2 + 4)).to(torch.uint8)
    code = code | (torch.signbit(g).to(torch.uint8) << 3)
    return code.flatten(-2), e.to(torch.int16)


def _packed(k, v, dtype):
    """Tiles of whole blocks: k, v [blocks, heads, block, dim] -> uint8 [blocks, heads, bytes]."""
    block, dim = k.shape[2:]
    groups = dim // 32
    kc, ke = _quantised(k, dtype)
    vc, ve = _quantised(v, dtype)
    pairs = lambda c: c[..., 0::2] | (c[..., 1::2] << 4)  # noqa: E731
    vb = pairs(vc).unflatten(-1, (16, groups)).unflatten(2, (block // 8, 8)).permute(0, 1, 2, 4, 3, 5)
    vs = (ve + 127).to(torch.uint8).unflatten(2, (block // 8, 8)).transpose(-1, -2)
    return torch.cat((pairs(kc).flatten(2), vb.flatten(2), (ke + 127).to(torch.uint8).flatten(2), vs.flatten(2)), dim=-1).contiguous()


def _values(code, scale):
    """codes [..., dim] and scale bytes [..., dim / 32] as 32-bit numbers."""
    m = (code & 7).float()
    m = torch.where(m < 4, m * 0.5, torch.where(m < 6, m - 2, 2 * m - 8))
    m = torch.where(code > 7, -m, m)
    return (torch.ldexp(m.unflatten(-1, (-1, 32)), scale[..., None].int() - 127)).flatten(-2)


def _unpacked(tiles, block, dim):
    """uint8 [..., bytes] -> k, v [..., block, dim] in 32 bits."""
    groups, half = dim // 32, block * dim // 2
    both = lambda b: torch.stack((b & 15, b >> 4), dim=-1).flatten(-2)  # noqa: E731
    kc, vb, ks, vs = tiles.split((half, half, block * groups, block * groups), dim=-1)
    vb = vb.unflatten(-1, (block // 8, 16, 8, groups)).transpose(-3, -2).flatten(-2).flatten(-3, -2)
    vs = vs.unflatten(-1, (block // 8, groups, 8)).transpose(-1, -2).flatten(-3, -2)
    return _values(both(kc.unflatten(-1, (block, -1))), ks.unflatten(-1, (block, groups))), _values(both(vb), vs)


# ---- the inputs

def _cos_sin(rot):
    """[positions][rot/2][2] fp32, from angles in 64 bits."""
    angle = torch.arange(POSITIONS, device="cuda", dtype=torch.float64)[:, None] * torch.pow(BASE, -torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    return torch.stack((angle.cos(), angle.sin()), dim=-1).float().contiguous()


def prepare(case, seed):
    rng = np.random.RandomState(seed % (1 << 32))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()  # noqa: E731
    c, s = case, dict(case=case)
    dtype, D, Hq, Hk = TYPES[c["dtype"]], c["dim"], c["q_heads"], c["kv_heads"]
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=gen, dtype=torch.float32)  # noqa: E731
    empty = lambda *shape: torch.empty(*shape, device="cuda", dtype=dtype)  # noqa: E731

    def pages(n, block):
        tiles = torch.empty(n, Hk, _tile_bytes(block, D), dtype=torch.uint8, device="cuda")
        per = max(1, (1 << 24) // (Hk * block * D))
        for at in range(0, n, per):
            m = min(per, n - at)
            tiles[at:at + m] = _packed(normal(m, Hk, block, D), normal(m, Hk, block, D), c["dtype"])
        return tiles

    if c["op"] != "attend":
        T = c["tokens"]
        # queries, keys and values as one projection leaves them, side by side in a token's row
        row = (normal(T, (Hq + 2 * Hk) * D) * 1.5).to(dtype).view(T, Hq + 2 * Hk, D)
        s.update(q=row[:, :Hq], k=row[:, Hq:Hq + Hk], v=row[:, Hq + Hk:], positions=i32(rng.randint(0, POSITIONS, T)), table=_cos_sin(c["rot"]),
                 q_weight=1 + 0.2 * normal(D), k_weight=1 + 0.2 * normal(D), q_out=empty(T, Hq, D), k_out=empty(T, Hk, D))
        if c["op"] == "gradient":
            s.update(q_back=normal(T, Hq, D).to(dtype), k_back=normal(T, Hk, D).to(dtype), q_weight_grad=torch.empty(D, device="cuda"), k_weight_grad=torch.empty(D, device="cuda"))
            if own:
                from paper_2210_08804_amd import binding
                s["parts"] = torch.empty(binding.HPS_SEQ_NORM_PARTS * 2 * D, device="cuda")
        if c["op"] == "append":
            n_blocks = -(-T // c["block"]) + 8
            slots = rng.permutation(n_blocks)[:, None] * c["block"] + np.arange(c["block"])
            s.update(pages=pages(n_blocks, c["block"]), slots=i32(slots.reshape(-1)[:T]), every=i32(np.arange(n_blocks * c["block"])),
                     k_read=empty(n_blocks * c["block"], Hk, D), v_read=empty(n_blocks * c["block"], Hk, D))
        return s
    block = c["block"]
    prefix, lens, new = _attend_lengths(c)
    prefix, deal = rng.permutation(prefix), rng.permutation(len(lens))
    lens, new = lens[deal], new[deal]
    need = int((-(-prefix // block)).sum()), int((-(-lens // block)).sum())
    n_blocks = need[0] + need[1] + 8
    blocks = rng.permutation(n_blocks)
    T = int(new.sum())
    group_offsets = np.arange(c["groups"] + 1) * c["requests"]
    offsets = np.concatenate([[0], np.cumsum(new)])
    s.update(q=(normal(T, Hq, D) * 1.5).to(dtype), pages=pages(n_blocks, block),
             block_table=i32(_tables(lens, block, -(-c["length"] // block), blocks[need[0]:])), lens=i32(lens), offsets=i32(offsets), out=empty(T, Hq, D),
             lse=torch.empty(T, Hq, device="cuda"), max_group=0)
    if c["groups"]:
        s.update(prefix_table=i32(_tables(prefix, block, -(-c["prefix"] // block), blocks)), prefix_lens=i32(prefix), group_offsets=i32(group_offsets),
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


def _own_norm(s, c):
    from paper_2210_08804_amd import binding as B
    B.hps_seq_norm_rope(s["q"], s["q_out"], q_weight=s["q_weight"], k=s["k"], k_out=s["k_out"], k_weight=s["k_weight"], positions=s["positions"], table=s["table"], eps=EPS,
                        interleaved=c["pairs"] == "neighbours")
    return s["q_out"], s["k_out"]


def _own_gradient(s, c):
    from paper_2210_08804_amd import binding as B
    B.hps_seq_norm_rope_grad(s["q"], s["q_back"], s["q_out"], q_weight=s["q_weight"], q_weight_grad=s["q_weight_grad"], k=s["k"], k_out_grad=s["k_back"], k_grad=s["k_out"],
                             k_weight=s["k_weight"], k_weight_grad=s["k_weight_grad"], positions=s["positions"], table=s["table"], eps=EPS,
                             interleaved=c["pairs"] == "neighbours", parts=s["parts"])
    return s["q_out"], s["k_out"], s["q_weight_grad"], s["k_weight_grad"]


def _own_append(s, c):
    from paper_2210_08804_amd import binding as B
    B.hps_seq_append_packed(s["k"], s["v"], s["pages"], s["slots"], q=s["q"], q_out=s["q_out"], positions=s["positions"], table=s["table"], interleaved=c["pairs"] == "neighbours",
                            norm=c["norm"], q_weight=s["q_weight"] if c["norm"] else None, k_weight=s["k_weight"] if c["norm"] else None, eps=EPS)
    B.hps_seq_read_packed(s["pages"], s["every"], s["k_read"], s["v_read"])
    return s["q_out"], s["k_read"], s["v_read"]


def _own_attend(s, c):
    from paper_2210_08804_amd import binding as B
    B.hps_seq_attention_packed(s["session"].handle, s["q"], s["pages"], s["block_table"], s["lens"], s["offsets"], s["out"], prefix_table=s.get("prefix_table"),
                               prefix_lens=s.get("prefix_lens"), group_offsets=s.get("group_offsets"), lse=s["lse"], max_new=c["new"], max_len=c["length"], max_prefix=c["prefix"],
                               max_group=s["max_group"])
    return s["out"], s["lse"]


_run_own = {"norm": _own_norm, "gradient": _own_gradient, "append": _own_append, "attend": _own_attend}


def _turned(x, positions, table, pairs, inverse=False):
    """x [T, H, D] with its leading 2 * table.shape[1] values turned, pair by pair, in x's type."""
    half = table.shape[1]
    cos, sin = table[positions.long(), None, :, 0].to(x.dtype), table[positions.long(), None, :, 1].to(x.dtype)
    sin = -sin if inverse else sin
    part = x[..., : 2 * half]
    a, b = (part[..., :half], part[..., half:]) if pairs == "half" else (part[..., 0::2], part[..., 1::2])
    u, v = a * cos - b * sin, a * sin + b * cos
    part = torch.cat((u, v), dim=-1) if pairs == "half" else torch.stack((u, v), dim=-1).flatten(-2)
    return torch.cat((part, x[..., 2 * half:]), dim=-1)


def _normed(x, weight):
    """Every head over its root mean square, weighted, in x's type."""
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.to(x.dtype)


def _plain_norm(s, c):
    return tuple(_turned(_normed(x.float(), w), s["positions"], s["table"], c["pairs"]).to(x.dtype) for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])))


def _plain_gradient(s, c):
    grads, weights = [], []
    for x, back, w in ((s["q"], s["q_back"], s["q_weight"]), (s["k"], s["k_back"], s["k_weight"])):
        dz = _turned(back.float(), s["positions"], s["table"], c["pairs"], inverse=True)
        r = torch.rsqrt(x.float().square().mean(-1, keepdim=True) + EPS)
        n = x.float() * r
        weights.append((dz * n).sum((0, 1)))
        dn = dz * w
        grads.append((r * (dn - n * (dn * n).mean(-1, keepdim=True))).to(x.dtype))
    return (*grads, *weights)


def _plain_append(s, c):
    block, pages, slots = c["block"], s["pages"], s["slots"].long()
    turn = lambda x, w: _turned(_normed(x, w) if c["norm"] else x, s["positions"], s["table"], c["pairs"])  # noqa: E731
    q = turn(s["q"].float(), s["q_weight"]).to(s["q"].dtype)
    k, v = turn(s["k"].double(), s["k_weight"]), s["v"].double()             # in front of a rounding to 4 bits: in 64
    D, groups = c["dim"], c["dim"] // 32
    bytes_of = lambda code: code[..., 0::2] | (code[..., 1::2] << 4)  # noqa: E731
    (kc, ke), (vc, ve) = _quantised(k, c["dtype"]), _quantised(v, c["dtype"])
    at, place = slots // block, slots % block
    n, half = pages.shape[0], block * D // 2
    keys, values = pages[..., :half].view(n, -1, block, D // 2), pages[..., half:2 * half].view(n, -1, block // 8, 16, 8, groups)
    key_scales = pages[..., 2 * half:2 * half + block * groups].view(n, -1, block, groups)
    value_scales = pages[..., 2 * half + block * groups:].view(n, -1, block // 8, groups, 8)
    keys[at, :, place] = bytes_of(kc)
    values[at, :, place // 8, :, place % 8] = bytes_of(vc).unflatten(-1, (16, groups))
    key_scales[at, :, place] = (ke + 127).to(torch.uint8)
    value_scales[at, :, place // 8, :, place % 8] = (ve + 127).to(torch.uint8)
    k_all, v_all = _unpacked(pages, block, D)
    return q, *(x.transpose(1, 2).flatten(0, 1).to(q.dtype) for x in (k_all, v_all))


def _part(q, pages, block, dim, table, lens, first, scale):
    """Attention over one table per row of q [N, M, Hq, D], the M-th query seeing the keys below min(lens, first + M): per query its maximum, sum and weighted values."""
    N, M, Hq, D = q.shape
    Hk = pages.shape[1]
    k, v = _unpacked(pages[table.long().clamp(min=0)], block, dim)                  # [N, blocks, Hk, block, D]
    k, v = k.transpose(1, 2).flatten(2, 3).transpose(2, 3).contiguous(), v.transpose(1, 2).flatten(2, 3).contiguous()
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
    q, offsets = s["q"], s["offsets"].long()
    T, scale = q.shape[0], 1.0 / math.sqrt(q.shape[2])
    token = torch.arange(T, device=q.device)
    request = torch.searchsorted(offsets[1:].contiguous(), token, right=True)
    stretches = [(request, offsets, c["new"], s["block_table"], s["lens"], s["lens"].long() - offsets.diff())]
    if c["groups"]:
        groups = s["group_offsets"].long()
        group = torch.searchsorted(groups[1:].contiguous(), request, right=True)
        stretches.append((group, offsets[groups], s["max_group"], s["prefix_table"], s["prefix_lens"], s["prefix_lens"]))
    parts = []
    for rows, starts, most, table, lens, first in stretches:
        at = token - starts[rows]
        padded = q.new_zeros(table.shape[0], most, *q.shape[1:])
        padded[rows, at] = q
        parts.append([x[rows, at] for x in _part(padded, s["pages"], c["block"], c["dim"], table, lens, first, scale)])
    top = torch.stack([p[0] for p in parts]).amax(0)
    weights = [(p[0] - top).exp() for p in parts]
    total = sum(p[1] * w for p, w in zip(parts, weights))
    return (sum(p[2] * w[..., None] for p, w in zip(parts, weights)) / total[..., None]).to(q.dtype), top + total.log()


_run_plain = {"norm": _plain_norm, "gradient": _plain_gradient, "append": _plain_append, "attend": _plain_attend}


# ---- what a pass cannot do without

def work(case):
    c = case
    D, Hq, Hk, size = c["dim"], c["q_heads"], c["kv_heads"], BYTES[c["dtype"]]
    if c["op"] != "attend":
        T = c["tokens"]
        heads, table = Hq + Hk, min(T, POSITIONS) * c["rot"] * 4 + 4 * T + 8 * D
        if c["op"] == "norm":
            return {"bytes": 2 * T * heads * D * size + table, "flops": T * heads * (4 * D + 3 * c["rot"])}
        if c["op"] == "gradient":
            return {"bytes": 3 * T * heads * D * size + table + 8 * D, "flops": T * heads * (11 * D + 3 * c["rot"])}
        slots = (-(-T // c["block"]) + 8) * c["block"]
        packed = Hk * D * 17 // 16                                    # of a token, keys and values
        return {"bytes": T * (2 * Hq + 2 * Hk) * D * size + table + 4 * T + T * packed + slots * (4 + packed + 2 * Hk * D * size),
                "flops": T * (heads * 3 * c["rot"] + (heads * 4 * D if c["norm"] else 0) + 2 * Hk * 4 * D) + slots * 2 * Hk * D}
    prefix, lens, new = _attend_lengths(c)
    T, keys = int(new.sum()), int(prefix.sum() + lens.sum())
    scores = int((prefix * c["requests"]).sum()) * T / len(lens) + float((new * (lens - (new - 1) / 2)).sum())
    return {"bytes": 2 * T * Hq * D * size + 4 * T * Hq + keys * Hk * D * 17 // 16, "flops": 4 * scores * Hq * D}


# ---- the definition in 64 bits

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_turned(x, c, positions, table, inverse=False):
    turn = torch.complex(table[..., 0].double(), (-1 if inverse else 1) * table[..., 1].double())[positions.long()][:, None, :]
    half = c["rot"] // 2
    if c["pairs"] == "half":
        z = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous()) * turn
        return torch.cat((z.real, z.imag, x[..., 2 * half:]), dim=-1)
    z = torch.view_as_complex(x[..., :2 * half].reshape(*x.shape[:2], half, 2).contiguous()) * turn
    return torch.cat((torch.view_as_real(z).flatten(-2), x[..., 2 * half:]), dim=-1)


def _exact_rounded(x, dtype):
    """x [..., dim] as 4-bit pages hold it: the nearest of the grid, searched for."""
    grid = torch.tensor(_GRID, device=x.device, dtype=torch.float64)
    middle = (grid[1:] + grid[:-1]) / 2
    g = x.reshape(*x.shape[:-1], -1, 32)
    powers = torch.exp2(torch.arange(LEAST[dtype], MOST[dtype] + 1, device=x.device, dtype=torch.float64))
    s = powers[torch.searchsorted(7 * powers, g.abs().amax(-1).contiguous()).clamp(max=len(powers) - 1)][..., None]
    v = (g / s).abs()
    low = torch.searchsorted(middle, v.contiguous())                        # of two as near: the lower, or by their codes
    tie = (low < 7) & (v == middle[low.clamp(max=6)]) & (low % 2 == 1)
    return (torch.copysign(grid[low + tie.long()], g) * s).reshape(x.shape)


def _exact_pages(tiles, block, dim):
    """The values of tiles [n, heads, bytes], byte by byte: k, v [n, block, heads, dim]."""
    n, heads, _ = tiles.shape
    groups = dim // 32
    grid = torch.tensor(_GRID + tuple(-x for x in _GRID), device=tiles.device, dtype=torch.float64)
    p, d = torch.arange(block, device=tiles.device)[:, None], torch.arange(dim, device=tiles.device)[None, :]
    half, width = block * dim // 2, 2 * groups
    at_k, at_v = p * (dim // 2) + d // 2, half + p // 8 * (4 * dim) + d // width * (8 * groups) + p % 8 * groups + d % width // 2
    of_k, of_v = 2 * half + p * groups + d // 32, 2 * half + block * groups + p // 8 * (8 * groups) + d // 32 * 8 + p % 8
    out = []
    for at, of, odd in ((at_k, of_k, d % 2), (at_v, of_v, d % width % 2)):
        code = (tiles[:, :, at.reshape(-1)].long().view(n, heads, block, dim) >> (4 * odd)) & 15
        out.append((grid[code] * torch.exp2(tiles[:, :, of.reshape(-1)].view(n, heads, block, dim).double() - 127)).transpose(1, 2))
    return out


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] != "attend":
        ins = [(s["q"].double(), s["q_weight"].double()), (s["k"].double(), s["k_weight"].double())]
        size = lambda x: torch.sqrt((x * x).sum(-1, keepdim=True) / c["dim"] + EPS)  # noqa: E731
        if c["op"] == "gradient":
            dx, dw = [], []
            for (x, w), back in zip(ins, (s["q_back"], s["k_back"])):
                dz, m = _exact_turned(back.double(), c, s["positions"], s["table"], inverse=True), size(x)
                dw.append((dz * x / m).flatten(0, 1).sum(0))
                dx.append(dz * w / m - x * (dz * w * x).sum(-1, keepdim=True) / (c["dim"] * m ** 3))
            return (*dx, *dw)
        outs = [_exact_turned(x / size(x) * w if c.get("norm", True) else x, c, s["positions"], s["table"]) for x, w in ins]
        if c["op"] == "norm":
            return tuple(outs)
        read = []
        for p, new in zip(_exact_pages(s["pages"], c["block"], c["dim"]), (outs[1], s["v"].double())):
            p = p.reshape(-1, *new.shape[1:]).contiguous()
            p.index_copy_(0, s["slots"].long(), _exact_rounded(new, c["dtype"]))
            read.append(p)
        return outs[0], *read
    block, D, Hq, Hk = c["block"], c["dim"], c["q_heads"], c["kv_heads"]
    offsets, lens = s["offsets"].tolist(), s["lens"].tolist()
    if len(lens) * max(1, max(c["prefix"], c["length"]) * Hk * D // (1 << 24)) > 4096:
        return None                                                   # over 20 seconds

    def keys_of(table, length):
        k, v = _exact_pages(s["pages"][table[: -(-length // block)].long()], block, D)
        return k.reshape(-1, Hk, D)[:length], v.reshape(-1, Hk, D)[:length]

    out = torch.empty(s["q"].shape, device="cuda", dtype=torch.float64)
    lse = torch.empty(s["q"].shape[:2], device="cuda", dtype=torch.float64)
    for g in range(max(1, c["groups"])):
        shared = int(s["prefix_lens"][g]) if c["groups"] else 0
        if shared:
            pk, pv = keys_of(s["prefix_table"][g], shared)
        for r in range(g * c["requests"], (g + 1) * c["requests"]):
            k, v = keys_of(s["block_table"][r], lens[r])
            if shared:
                k, v = torch.cat((pk, k)), torch.cat((pv, v))
            k, v = k.transpose(0, 1), v.transpose(0, 1)
            n = offsets[r + 1] - offsets[r]
            q = s["q"][offsets[r]:offsets[r + 1]].double().view(n, Hk, Hq // Hk, D).transpose(0, 1).reshape(Hk, n * (Hq // Hk), D)
            scores = torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(D)
            hidden = torch.arange(k.shape[1], device="cuda")[None, :] > shared + lens[r] - n + torch.arange(n, device="cuda").repeat_interleave(Hq // Hk)[:, None]
            scores = scores.masked_fill(hidden, -math.inf)
            p = torch.softmax(scores, dim=-1)
            out[offsets[r]:offsets[r + 1]] = torch.bmm(p, v.contiguous()).view(Hk, n, Hq // Hk, D).transpose(0, 1).reshape(n, Hq, D)
            lse[offsets[r]:offsets[r + 1]] = torch.logsumexp(scores, dim=-1).view(Hk, n, Hq // Hk).transpose(0, 1).reshape(n, Hq)
    return out, lse
