"""Packed pages (hps_seq_append_packed, hps_seq_read_packed) against their definition, byte by byte."""
import math

import pytest
import torch

import packed_reference as P
import seq_reference as R
from paper_2210_08804_amd import binding as B
from test_gpu_seq_norm import table_of

pytestmark = pytest.mark.gpu
F32, HF, BF = torch.float32, torch.float16, torch.bfloat16


class Case:
    def __init__(self, dtype, T, H, K, D, block, rot=None, norm=True, weights=True, seed=0, lead=0, spare=2, size=1.5):
        g = torch.Generator().manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        self.row = (normal(T, (H + 2 * K) * D + lead) * size).to(dtype)
        self.dtype, self.T, self.H, self.K, self.D, self.block, self.norm, self.lead = dtype, T, H, K, D, block, norm, lead
        self.n_blocks = -(-T // block) + spare
        self.slots = torch.randperm(self.n_blocks * block, generator=g)[:T].int()
        self.table, self.positions = table_of(50, rot) if rot else None, torch.randint(0, 50, (T,), generator=g).int()
        self.qw, self.kw = (1 + 0.3 * normal(D), 1 + 0.3 * normal(D)) if weights and norm else (None, None)
        self.size = B.hps_seq_packed_bytes(block, D)
        self.before = torch.randint(0, 256, (self.n_blocks, K, self.size), generator=g).to(torch.uint8)

    def heads(self, row):
        H, K, D, lead = self.H, self.K, self.D, self.lead
        cut = lambda a, n: row[:, lead + a * D:lead + (a + n) * D].unflatten(1, (n, D)) if n else row.new_zeros(self.T, 0, D)  # noqa: E731
        return cut(0, H), cut(H, K), cut(H + K, K)

    def run(self, interleaved=False, eps=1e-6, pages=None, q_out=None, stream=None):
        cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
        q, k, v = self.heads(self.row.cuda())
        pages = self.before.cuda() if pages is None else pages
        q_out = torch.full((self.T, self.H, self.D), 9.0, dtype=self.dtype, device="cuda") if q_out is None else q_out
        args = dict(q=q if self.H else None, q_out=q_out if self.H else None, positions=cuda(self.positions) if self.table is not None else None, table=cuda(self.table),
                    interleaved=interleaved, norm=self.norm, q_weight=cuda(self.qw), k_weight=cuda(self.kw), eps=eps)
        slots = self.slots.cuda()
        torch.cuda.synchronize()
        B.hps_seq_append_packed(k, v, pages, slots, stream=stream, **args)
        torch.cuda.synchronize()
        return q_out.cpu(), pages.cpu()

    def want(self, interleaved=False, eps=1e-6):
        """(q, its bound, pages, mask of bytes that are compared)"""
        q, k, v = self.heads(self.row)
        if self.norm:
            q_out, bound = P.norm_rope(q, self.qw, self.positions, self.table, eps, interleaved)
        else:
            q_out = P.turned(q.double(), self.positions, self.table, interleaved)
            bound = R.ROUND[self.dtype] * 1.01 * q_out.abs() + P.pair_size(q.double(), self.table, interleaved) * 3 * P.U + R.TINY[self.dtype]
        k = k.double()
        k = P.turned(P.normed(k, self.kw, eps) if self.norm else k, self.positions, self.table, interleaved)
        pages, mask = self.before.clone(), torch.ones_like(self.before, dtype=torch.bool)
        keep = P.live(self.positions, self.table, self.T)
        for which, x in ((0, k), (1, v.double())):
            code, scale = P.quantised(x, self.dtype)
            for t in range(self.T):
                if keep[t] and 0 <= self.slots[t] < self.n_blocks * self.block:
                    for h in range(self.K):
                        s = int(self.slots[t])
                        none = P.store(pages, self.block, self.D, s, h, which, code[t, h], scale[t, h])
                        mask[s // self.block, h, none] = False
        return q_out, bound, pages, mask

    def check(self, interleaved=False, eps=1e-6, **kw):
        q, pages = self.run(interleaved, eps, **kw)
        want, bound, want_pages, mask = self.want(interleaved, eps)
        keep = P.live(self.positions, self.table, self.T)
        R.close(q[keep], want[keep], bound[keep])
        assert (q[~keep] == 9).all()
        bad = ((pages != want_pages) & mask).nonzero()
        assert len(bad) == 0, f"{len(bad)} bytes, the first at {bad[0].tolist()}: {int(pages[tuple(bad[0])])} where {int(want_pages[tuple(bad[0])])}"
        return pages


@pytest.mark.parametrize("dtype", [F32, HF, BF])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 256])
def test_head_dims(D, dtype):
    for rot, interleaved in ((D, False), (D, True), (D // 2, False), (2, True), (10, False), (None, False)):
        Case(dtype, 37, 4, 2, D, 16, rot, seed=D).check(interleaved)
        Case(dtype, 5, 3, 3, D, 32, rot, norm=False, seed=D + 1).check(interleaved)


@pytest.mark.parametrize("block", [16, 32, 64, 128, 1024])
def test_block_sizes(block):
    for D in (64, 96, 128):
        Case(BF, 70, 2, 1, D, block, D, seed=block, spare=1).check()


@pytest.mark.parametrize("T,H,K", [(0, 2, 1), (1, 8, 2), (2, 0, 3), (8, 5, 5), (9, 16, 1), (133, 33, 11)])
def test_tokens_and_heads(T, H, K):
    Case(BF, T, H, K, 64, 16, 64, seed=T + 1).check()


def test_many_tokens():
    """Enough of them for work-groups that go through all heads."""
    c = Case(BF, 8200, 1, 2, 128, 32, 128, seed=5)
    q, pages = c.run()
    few = torch.cat((torch.arange(40), torch.arange(8160, 8200)))
    _, k, v = c.heads(c.row)
    k = P.turned(P.normed(k[few].double(), c.kw, 1e-6), c.positions[few], c.table, False)
    read = [x.transpose(1, 2).flatten(0, 1)[c.slots[few].long()] for x in P.unpacked(pages, 32, 128)]
    for x, got in ((k, read[0]), (v[few].double(), read[1])):
        assert torch.equal(P.values(*P.quantised(x, BF)), got)
    other = torch.ones(c.n_blocks * 32, dtype=torch.bool)
    other[c.slots.long()] = False
    for now, then in zip(P.unpacked(pages, 32, 128), P.unpacked(c.before, 32, 128)):
        now, then = (x.transpose(1, 2).flatten(0, 1)[other] for x in (now, then))
        assert torch.equal(now.nan_to_num(7.25), then.nan_to_num(7.25))


@pytest.mark.parametrize("dtype", [F32, HF, BF])
@pytest.mark.parametrize("lead", [1, 4])
def test_rows_that_start_anywhere(lead, dtype):
    for D, rot, interleaved in ((64, 32, False), (96, 96, True), (128, 100, False)):
        Case(dtype, 11, 3, 2, D, 16, rot, seed=lead, lead=lead).check(interleaved)


def test_slots_and_positions_that_are_none():
    c = Case(BF, 40, 2, 2, 64, 16, 64, seed=6)
    c.slots[3], c.slots[11], c.slots[12], c.slots[13] = -1, c.n_blocks * 16, 2 ** 31 - 1, -2 ** 31
    c.positions[20], c.positions[21] = -1, -7
    c.check()
    c.positions[22] = 50                               # behind the table: its keys are no numbers
    q, pages = c.run()
    k, v = (x.transpose(1, 2).flatten(0, 1)[int(c.slots[22])] for x in P.unpacked(pages, 16, 64))
    assert torch.isnan(k).all() and torch.isfinite(v).all() and torch.isnan(q[22]).all()


def test_pages_in_strides():
    c = Case(BF, 50, 2, 3, 96, 16, 96, seed=7)
    wide = torch.full((3, c.n_blocks, c.size + 48), 77, dtype=torch.uint8, device="cuda")
    pages = wide[:, :, 16:16 + c.size].transpose(0, 1)
    pages.copy_(c.before)
    c.check(pages=pages)
    assert (wide[:, :, :16] == 77).all() and (wide[:, :, 16 + c.size:] == 77).all()


def test_roundings():
    """Every code's neighbourhood, ties, signed zeros, the largest of a group at and behind 7 times a power of two."""
    steps = torch.tensor([0, .2, .25, .26, .5, .74, .75, .76, 1, 1.25, 1.5, 1.75, 2, 2.25, 2.5, 2.75, 3, 3.5, 3.75, 4, 4.5, 5, 5.25, 5.5, 6, 6.5])
    for dtype in (F32, HF, BF):
        for largest in (4.0, 6.0, 7.0, 7.0 * (1 + 2.0 ** -7), 7.5, 7.9):
            for power in (0, -9, 7):
                c = Case(dtype, 2, 0, 2, 64, 16, None, norm=False, seed=8)
                x = torch.cat((steps, -steps[:5], torch.tensor([largest])))
                c.row = (torch.stack([x * 2.0 ** power, -x * 2.0 ** power]).repeat(1, 8)).to(dtype)
                c.check()


@pytest.mark.parametrize("interleaved", [False, True])
def test_keys_next_to_a_border(interleaved):
    """Keys that lie 2^-28 and less beside the middle of two codes, or of two scales, further than 32 bits tell: rounded as in 64."""
    D, middles = 64, torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
    for largest in (6.0, 7.0):                         # 7 with something more has the next scale
        for off in (2.0 ** -28, -2.0 ** -28, 2.0 ** -40, -2.0 ** -40, 2.0 ** -52, 0.0):
            c = Case(BF, 1, 0, 1, D, 16, D, norm=False, seed=11)
            c.row[:] = 1
            cos = middles.repeat(4).clamp(max=largest)
            c.table = torch.stack((cos, torch.full_like(cos, off)), -1)[None]           # values middle - off, and middle + off of the partners
            c.positions[:] = 0
            c.check(interleaved)


@pytest.mark.parametrize("dtype", [F32, HF, BF])
def test_sizes_of_values(dtype):
    """Groups at the ends of what a type holds; one that is not finite leaves its neighbours alone."""
    largest, least = torch.finfo(dtype).max, torch.finfo(dtype).tiny * torch.finfo(dtype).eps
    c = Case(dtype, 12, 0, 1, 96, 16, None, norm=False, seed=9, size=1.0)
    c.row[0] = 0
    c.row[1] = largest
    c.row[2] = -largest
    c.row[3, ::2] = least
    c.row[4, 7] = least
    c.row[5] = (c.row[5].float().clamp(-3, 3) * (largest / 4)).to(dtype)
    c.row[6, 10], c.row[7, 40], c.row[8, 80], c.row[9, 100] = math.inf, math.nan, -math.inf, math.nan
    pages = c.check()
    k, v = (x.transpose(1, 2).flatten(0, 1)[c.slots.long()][:, 0] for x in P.unpacked(pages, 16, 96, dtype))
    assert torch.isnan(k[6, :32]).all() and torch.isfinite(k[6, 32:]).all() and torch.isnan(v[9, :32]).all() and torch.isfinite(v[9, 32:]).all()
    assert torch.isfinite(k[:6]).all() and torch.isfinite(v[:6]).all()


@pytest.mark.parametrize("dtype", [F32, HF, BF])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 256])
def test_reading(D, dtype):
    """Every byte of tiles at random, scales that are none among them; slots that are none leave their rows alone."""
    g = torch.Generator().manual_seed(D)
    n, K, block = 5, 3, 32
    tiles = torch.randint(0, 256, (n, K, B.hps_seq_packed_bytes(block, D)), generator=g).to(torch.uint8)
    tiles[:3, :, block * D:] = (tiles[:3, :, block * D:] % 30 + 112).to(torch.uint8)
    tiles[3, :, block * D:] = (tiles[3, :, block * D:] % 8 + 248).to(torch.uint8)
    slots = torch.cat((torch.randperm(n * block, generator=g), torch.tensor([3, 3, -1, n * block, 2 ** 31 - 1]))).int()
    ok = (slots >= 0) & (slots < n * block)
    want = [x.transpose(1, 2).flatten(0, 1)[slots.long().clamp(0, n * block - 1)] for x in P.unpacked(tiles, block, D, dtype)]
    for strided in (False, True):
        outs = [torch.full((len(slots), K, D + 1) if strided else (len(slots), K, D), 9.0, dtype=dtype, device="cuda")[..., :D] for _ in range(2)]
        B.hps_seq_read_packed(tiles.cuda(), slots.cuda(), *outs)
        torch.cuda.synchronize()
        for got, x in zip(outs, want):
            x = x.to(dtype)
            assert torch.equal(got.cpu()[ok].nan_to_num(7.25), x[ok].nan_to_num(7.25)) and torch.equal(torch.isnan(got.cpu()[ok]), torch.isnan(x[ok]))
            assert (got[~ok] == 9).all()
    only = torch.full((len(slots), K, D), 9.0, dtype=dtype, device="cuda")
    B.hps_seq_read_packed(tiles.cuda(), slots.cuda(), v_out=only)
    torch.cuda.synchronize()
    assert torch.equal(only.cpu().nan_to_num(7.25), outs[1].cpu().nan_to_num(7.25))


def test_stream_of_its_own_and_graphs():
    c = Case(BF, 300, 4, 2, 128, 16, 128, seed=10)
    want = c.run()
    s = torch.cuda.Stream()
    got = c.run(stream=s)
    assert all(torch.equal(x, y) for x, y in zip(want, got))
    q, k, v = c.heads(c.row.cuda())
    pages, q_out, slots = c.before.cuda(), torch.empty_like(q), c.slots.cuda()
    read = [torch.empty(300, 2, 128, dtype=BF, device="cuda") for _ in range(2)]
    args = dict(q=q, q_out=q_out, positions=c.positions.cuda(), table=c.table.cuda(), norm=True, q_weight=c.qw.cuda(), k_weight=c.kw.cuda())
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        B.hps_seq_append_packed(k, v, pages, slots, **args)
        B.hps_seq_read_packed(pages, slots, *read)
    for i in range(3):
        c.row *= 1.5
        q.copy_(c.heads(c.row)[0]), k.copy_(c.heads(c.row)[1]), v.copy_(c.heads(c.row)[2])
        g.replay()
        torch.cuda.synchronize()
        eager_q, eager_pages = c.run()
        assert torch.equal(q_out.cpu(), eager_q) and torch.equal(pages.cpu(), eager_pages)
        for x, w in zip(read, P.unpacked(eager_pages, 16, 128)):
            assert torch.equal(x.cpu().double(), w.transpose(1, 2).flatten(0, 1)[c.slots.long()])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_keys_next_to_a_border_of_the_least_scale(dtype, interleaved):
    """Keys beside the middle of two codes where the scale is the least: numbers below 2^-126, of which 32 bits tell less the smaller they are."""
    middles = torch.tensor([.25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0]) * 2.0 ** -126
    for off in (2.0 ** -22, 2.0 ** -24, 2.0 ** -40, 2.0 ** -49, 0.0):
        for sign in (1, -1):
            c = Case(dtype, 1, 0, 1, 64, 16, 64, norm=False, seed=12)
            c.row[:] = 2.0 ** -60
            cos = middles.repeat(4) * 2.0 ** 60
            c.table = torch.stack((cos, torch.full_like(cos, sign * off * 2.0 ** -66)), -1)[None]
            c.positions[:] = 0
            c.check(interleaved)


@pytest.mark.parametrize("odd", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("D", [64, 96, 256])
def test_normed_keys_that_are_infinite(D, odd):
    """An infinite key divides the others of its head by infinity, to zeros of either sign; one that is no number spoils its head."""
    for rot, at in ((None, 3), (D, 40), (D // 2, D - 1)):
        c = Case(BF, 5, 2, 2, D, 16, rot, seed=13)
        c.row[2, 2 * D + at] = odd
        _, pages = c.run()
        _, _, want, mask = c.want()
        for got, expected in zip(P.unpacked(pages, 16, D), P.unpacked(want, 16, D)):
            assert torch.equal(torch.isnan(got), torch.isnan(expected)) and torch.equal(got.nan_to_num(7.25), expected.nan_to_num(7.25))


def test_queries_and_keys_of_any_size():
    for size in (1e-30, 1e-22, 1e20):
        c = Case(BF, 9, 2, 2, 64, 16, 64, seed=18)
        c.row[:, :] = (c.row.double() * size).to(BF)
        c.check(eps=0.0)
