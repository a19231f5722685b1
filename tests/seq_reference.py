"""The operators of hps_seq.h from their definitions, in 64 bits on the CPU, and how far results may be from them.  (Test infrastructure only.)"""
import math

import numpy as np
import torch

ROUND = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}      # half a unit in the last place, relative: 24, 11 and 8 significant bits
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}        # and absolute, below the normal numbers


def extend(past, new, start, free, n_free, n_blocks, block, table, max_tokens):
    """(table, token_offsets, total_lens, slots, positions, info); token by token."""
    table = table.copy()
    width, cap = table.shape[1] if table.ndim == 2 else 0, table.shape[1] * block
    n_free = min(max(n_free, 0), n_blocks)
    left, short, over, tokens = n_free, 0, 0, 0
    offsets, lens, slots, positions = [0], [], [], []
    for r in range(len(past)):
        p, n = min(max(int(past[r]), 0), cap), max(int(new[r]), 0)
        fit = min(n, cap - p)
        for j in range(-(-p // block), -(-(p + fit) // block)):
            if left > 0:
                left -= 1
                b = int(free[left])
            else:
                short += 1
                b = -1
            table[r, j] = b if 0 <= b < n_blocks else -1
        for i in range(min(n, max(0, max_tokens - tokens))):
            own = p + i
            b = int(table[r, own // block]) if own < cap else -1
            slots.append(b * block + own % block if 0 <= b < n_blocks else -1)
            positions.append((0 if start is None else int(start[r])) + own)
        tokens += n
        over += n - fit
        offsets.append(min(tokens, 2 ** 31 - 1))
        lens.append(p + fit)
    slots += [-1] * (max_tokens - len(slots))
    positions += [-1] * (max_tokens - len(positions))
    i32 = lambda x: np.asarray(x, dtype=np.int32)  # noqa: E731
    return table, i32(offsets), i32(lens), i32(slots), i32(positions), i32([left, min(tokens, 2 ** 31 - 1), short, min(over, 2 ** 31 - 1)])


def release(lens, finished, block, table, free, n_free, n_blocks):
    """(lens, table, free, info[:3])"""
    lens, table, free = lens.copy(), table.copy(), free.copy()
    cap = table.shape[1] * block
    n = had = min(max(n_free, 0), n_blocks)
    lost = 0
    for r in range(len(lens)):
        if not finished[r]:
            continue
        for j in range(-(-min(max(int(lens[r]), 0), cap) // block)):
            b, table[r, j] = int(table[r, j]), -1
            if not 0 <= b < n_blocks:
                continue
            if n < n_blocks:
                free[n] = b
                n += 1
            else:
                lost += 1
        lens[r] = 0
    return lens, table, free, np.asarray([n, n - had, lost], dtype=np.int32)


def angles(rot, base=10000.0, scale=0, factor=1.0, original=1.0, low=1.0, high=2.0):
    w = base ** (-2.0 * np.arange(rot // 2) / rot)
    if scale == 1:
        w = w / factor
    if scale == 2:
        g = np.clip((original * w / (2 * np.pi) - low) / (high - low), 0, 1)
        w = w * (g + (1 - g) / factor)
    return w


def rope(x, positions, table, interleaved, inverse):
    """x [T, H, D] turned by the rows of table [positions, rot / 2, 2], in 64 bits."""
    x, table = x.double().clone(), table.double()
    half = table.shape[1]
    live = positions >= 0
    row = table[positions.clamp(0, table.shape[0] - 1).long()].clone()
    row[positions >= table.shape[0]] = math.nan
    cos, sin = row[:, None, :, 0], row[:, None, :, 1] * (-1 if inverse else 1)
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    u, v = a * cos - b * sin, a * sin + b * cos
    out = x.clone()
    if interleaved:
        out[..., 0:2 * half:2], out[..., 1:2 * half:2] = u, v
    else:
        out[..., :half], out[..., half:2 * half] = u, v
    return out, live


def rope_bound(x, out, dtype):
    """Products and the sum of two in 32 bits, with one rounding each, then one to the type: each term is at most |x| of its pair's norm, times cosines
    that are themselves given in 32 bits (they are inputs here)."""
    size = x.double().abs().amax() * 1.5
    return ROUND[dtype] * out.abs() * 1.001 + 3 * 2.0 ** -24 * size + TINY[dtype]


def keys_of(pages, table, length, block):
    """[length, heads, dim] in 64 bits; blocks that are none stand for zeros."""
    at = torch.arange(length)
    b = table[at // block].long() if length else at
    ok = (b >= 0) & (b < pages.shape[0])
    x = pages[b.clamp(0, max(pages.shape[0] - 1, 0)), at % block].double() if length else pages.new_zeros((0, *pages.shape[2:])).double()
    return torch.where(ok[:, None, None], x, torch.zeros_like(x)) if length else x


def attention(q, k_pages, v_pages, block_table, lens, offsets, scale, prefix_table=None, prefix_lens=None, group_offsets=None, written=None):
    """(out, lse, bound of out's error, bound of lse's) for tensors on the CPU."""
    T, H, D = q.shape
    hk, block, dtype = k_pages.shape[2], k_pages.shape[1], q.dtype
    out, lse = torch.full((T, H, D), math.nan, dtype=torch.float64), torch.full((T, H), math.nan, dtype=torch.float64)
    bound, lse_bound = torch.zeros(T, H, D, dtype=torch.float64), torch.zeros(T, H, dtype=torch.float64)
    for r in range(len(lens)):
        group = [g for g in range(0 if prefix_lens is None else len(prefix_lens)) if group_offsets[g] <= r < group_offsets[g + 1]]
        parts = [(prefix_table[g], int(prefix_lens[g])) for g in group] + [(block_table[r], int(lens[r]))]
        k = torch.cat([keys_of(k_pages, t, n, block) for t, n in parts])
        v = torch.cat([keys_of(v_pages, t, n, block) for t, n in parts])
        shared, n = sum(n for _, n in parts[:-1]), int(offsets[r + 1] - offsets[r])
        for i in range(n):
            t = int(offsets[r]) + i
            sees = shared + max(0, int(lens[r]) - n + i + 1)
            kk, vv = (x[:sees].repeat_interleave(H // hk, dim=1).transpose(0, 1) for x in (k, v))        # [H, sees, D]
            if sees == 0:
                out[t], lse[t] = 0, -math.inf
                continue
            qq = q[t].double()
            s = (kk @ qq[:, :, None]).squeeze(-1) * scale
            top = s.amax(-1, keepdim=True)
            top = torch.where(top == -math.inf, torch.zeros_like(top), top)
            w = (s - top).exp()
            total = w.sum(-1, keepdim=True)
            p = torch.where(total == 0, torch.zeros_like(w), w / total)
            weighed = torch.where(p[:, :, None] == 0, torch.zeros_like(vv), p[:, :, None] * vv) if not torch.isfinite(vv).all() else p[:, :, None] * vv
            out[t] = weighed.sum(1)
            lse[t] = (top + total.log()).squeeze(-1)
            # scores: a sum of D products in 32 bits, scaled, an exponent of it; twice (the weight and the sum of weights)
            e = (scale * (kk.abs() @ qq.abs()[:, :, None]).amax(1).squeeze(-1) * (D + 8) * 2.0 ** -24 + 2.0 ** -21)[:, None]
            mass = weighed.abs().sum(1)
            # a weight is rounded to the type (relative, and for halves absolute: weights are given against a sum of at least 1), sums are in 32 bits
            bound[t] = ROUND[dtype] * 1.01 * (out[t].abs() + mass) + mass * (2 * e + (sees + 64) * 2.0 ** -24) + sees * TINY[dtype] * vv.abs().amax(1) + TINY[dtype]
            lse_bound[t] = e.squeeze(-1) + sees * 2.0 ** -24 + lse[t].abs() * 2.0 ** -21 + 1e-6
    return out, lse, bound, lse_bound


def close(got, want, bound):
    """Finite where it should be, within the bound there, and the same infinities and NaN elsewhere."""
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    odd = ~fine & ~torch.isnan(want)
    assert torch.equal(got[odd], want[odd])
    off = (got - want).abs()[fine] - bound.expand_as(want)[fine]
    assert off.numel() == 0 or off.max() <= 0, f"{int((off > 0).sum())} of {off.numel()} values beyond their bound, by {float(off.max()):.3g}"
