"""Head norms and packed pages of hps_seq.h from their definitions, in 64 bits on the CPU, and how far results may be from them.  (Test infrastructure only.)"""
import torch

import seq_reference as R

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
U = 2.0 ** -24                                         # a rounding to 32 bits, relative


def normed(x, weight, eps):
    y = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    return y if weight is None else y * weight.double()


def turned(x, positions, table, interleaved, inverse=False):
    """x in 64 bits; rows of negative positions as they are."""
    if table is None:
        return x
    half = table.shape[1]
    row = table.double()[positions.clamp(0, table.shape[0] - 1).long()].clone()
    row[positions >= table.shape[0]] = float("nan")
    cos, sin = row[:, None, :, 0], row[:, None, :, 1] * (-1 if inverse else 1)
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    u, v = a * cos - b * sin, a * sin + b * cos
    part = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((part, x[..., 2 * half:]), -1)


def live(positions, table, T):
    return torch.ones(T, dtype=torch.bool) if table is None else positions >= 0


def pair_size(x, table, interleaved):
    """|a| + |b| of the pair that a value is turned with, its own size where it is not."""
    x = x.abs()
    if table is None:
        return x
    half = table.shape[1]
    both = x[..., 0:2 * half:2] + x[..., 1:2 * half:2] if interleaved else x[..., :half] + x[..., half:2 * half]
    part = torch.stack((both, both), -1).flatten(-2) if interleaved else torch.cat((both, both), -1)
    return torch.cat((part, x[..., 2 * half:]), -1)


def norm_rope(x, weight, positions, table, eps, interleaved):
    """(out, bound): the squares' sum is off by D roundings at most, its root by half of that; the root, the division, eps, two products and a pair's
    three operations add a dozen; one rounding to the type."""
    z = normed(x.double(), weight, eps)
    out = turned(z, positions, table, interleaved)
    return out, R.ROUND[x.dtype] * 1.01 * out.abs() + pair_size(z, table, interleaved) * (x.shape[-1] / 2 + 12) * U + R.TINY[x.dtype]


def norm_rope_grad(x, weight, back, positions, table, eps, interleaved):
    """(dx, its bound, dweight, its bound), by differentiation of the definition."""
    T, H, D = x.shape
    keep = live(positions, table, T)
    xd = x.double().clone().requires_grad_(True)
    w = (torch.ones(D) if weight is None else weight).double().clone().requires_grad_(True)
    out = turned(normed(xd, w, eps), positions, table, interleaved)
    dx, dw = torch.autograd.grad(out[keep], (xd, w), back.double()[keep], allow_unused=True) if keep.any() and H else (torch.zeros_like(xd), torch.zeros_like(w))
    xd, w = xd.detach(), w.detach()
    # dx = r (w dz - n mean(w dz n)): dz is off by 3 roundings of its pair's size, sums by D, r by D / 2, and each product by one
    r = 1 / (xd.square().mean(-1, keepdim=True) + eps).sqrt()
    n, z = xd * r, pair_size(back.double(), table, interleaved)
    mean = (z * w.abs() * n.abs()).mean(-1, keepdim=True)
    bound = R.ROUND[x.dtype] * 1.01 * dx.abs() + r * (z * w.abs() + n.abs() * mean) * (2 * D + 32) * U + R.TINY[x.dtype]
    # a weight's sum has T * H terms, each off by D / 2 + 10, in chains of no more than all of them, 256 rows and 80 parts
    terms = (z * n.abs())[keep].sum((0, 1))
    return dx, bound, dw, terms * (D / 2 + 10 + min(T * H, 4096) + 336) * U + R.TINY[torch.float32]


# ---- packed pages

LEAST, MOST = {torch.float32: -126, torch.float16: -23, torch.bfloat16: -126}, {torch.float32: 125, torch.float16: 13, torch.bfloat16: 125}


def quantised(x, dtype):
    """(codes [..., D], scale bytes [..., D / 32]) of x in 64 bits, as int64: by looking at every code."""
    g = x.double().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1)
    e = torch.full(top.shape, LEAST[dtype], dtype=torch.int64)
    for k in range(LEAST[dtype], MOST[dtype]):
        e = torch.where(top > 7 * 2.0 ** k, torch.full_like(e, k + 1), e)
    v = g.abs() / torch.exp2(e.double())[..., None]
    grid = torch.tensor(GRID, dtype=torch.float64)
    off = (v[..., None] - grid).abs()
    near = off == off.amin(-1, keepdim=True)           # one, or two neighbours: of these the even one
    even = torch.tensor([i % 2 == 0 for i in range(8)])
    code = torch.where(near.sum(-1) == 1, near.long().argmax(-1), (near & even).long().argmax(-1))
    code = code + 8 * torch.signbit(g).long()
    odd = ~torch.isfinite(g).all(-1)
    return torch.where(odd[..., None], torch.full_like(code, -1), code).flatten(-2), torch.where(odd, torch.full_like(e, 255), e + 127)


def places(block, D):
    """Byte and half of every value (place, d) in a tile: codes of keys, codes of values, scales of keys, scales of values."""
    h = D // 32
    p, d = torch.arange(block)[:, None], torch.arange(D)[None, :]
    g = torch.arange(h)[None, :]
    return ((p * (D // 2) + d // 2, d % 2), (block * D // 2 + p // 8 * 4 * D + d // (2 * h) * 8 * h + p % 8 * h + d % (2 * h) // 2, d % 2),
            block * D + p * h + g, block * (D + h) + p // 8 * 8 * h + g * 8 + p % 8)


def values(code, scale, dtype=torch.float32):
    """What codes and scale bytes stand for, in 64 bits, read as `dtype`."""
    grid = torch.tensor(GRID + tuple(-x for x in GRID), dtype=torch.float64)
    s = torch.exp2(scale.double() - 127)
    s = torch.where(scale > (140 if dtype == torch.float16 else 252), torch.full_like(s, float("nan")), s)
    return (grid[code.clamp(min=0)].unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def unpacked(tiles, block, D, dtype=torch.float32):
    """tiles uint8 [..., bytes] -> keys, values [..., block, D] in 64 bits."""
    (kb, kh), (vb, vh), ks, vs = places(block, D)
    t = tiles.long()
    return tuple(values(t[..., b] >> (4 * h) & 15, t[..., s], dtype) for b, h, s in ((kb, kh, ks), (vb, vh, vs)))


def store(tiles, block, D, slot, head, which, code, scale):
    """Writes a token's codes [D] (-1: not compared) and scale bytes of one head into tiles uint8 [blocks, heads, bytes]; returns the bytes whose codes are none."""
    (kb, kh), (vb, vh), ks, vs = places(block, D)
    b, h, s = ((kb, kh, ks), (vb, vh, vs))[which]
    b, h, s = b[slot % block], h[slot % block if h.shape[0] > 1 else 0], s[slot % block]
    tile = tiles[slot // block, head]
    for half in (0, 1):
        at = b[h == half]
        c = code[h == half].clamp(min=0)
        tile[at] = ((tile[at].long() & (0xF0 if half == 0 else 0x0F)) | (c << (4 * half))).to(torch.uint8)
    tile[s] = scale.to(torch.uint8)
    return b[code < 0]


def packed(k, v, dtype):
    """Tiles uint8 [blocks, heads, bytes] of pages k, v [blocks, block, heads, D]; the codes of groups that are no numbers are 0."""
    n, block, K, D = k.shape
    (kb, kh), (vb, vh), ks, vs = places(block, D)
    tiles = torch.zeros(n, K, block * D * 17 // 16, dtype=torch.int64)
    for x, b, h, s in ((k, kb, kh, ks), (v, vb, vh, vs)):
        code, scale = quantised(x.transpose(1, 2), dtype)                   # [n, K, block, D]
        code = code.clamp(min=0) << (4 * h)
        tiles.scatter_add_(2, b.expand(n, K, block, D).flatten(2), code.flatten(2))
        tiles.scatter_(2, s.expand(n, K, *s.shape).flatten(2), scale.flatten(2))
    return tiles.to(torch.uint8)
