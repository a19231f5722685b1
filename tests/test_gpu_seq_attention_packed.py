"""Attention over packed pages (hps_seq_attention_packed) against the definition in 64 bits, on what the pages hold."""
import math

import pytest
import torch

import packed_reference as P
import seq_reference as R
from paper_2210_08804_amd import binding as B
from test_gpu_seq_attention import MIXED, Problem

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


class Packed(Problem):
    """The same problems, their keys and values rounded to packed pages; unused places are no numbers (`junk`)."""

    def tiles(self):
        return P.packed(self.k.double(), self.v.double(), self.dtype)

    def want(self):
        k, v = (x.transpose(1, 2) for x in P.unpacked(self.tiles(), self.block, self.D, self.dtype))
        return R.attention(self.q, k, v, self.block_table, self.lens, self.offsets, self.scale or self.D ** -0.5,
                           *((self.prefix_table, self.prefix_lens, self.group_offsets) if len(self.prefix_lens) else ()))

    def pages(self):
        t = self.tiles().cuda()
        if self.layout == "heads first":
            return t.transpose(0, 1).contiguous().transpose(0, 1)
        if self.layout == "apart":
            wide = torch.full((t.shape[0], t.shape[1], t.shape[2] + 80), 255, dtype=torch.uint8, device="cuda")
            wide[:, :, 32:32 + t.shape[2]] = t
            return wide[:, :, 32:32 + t.shape[2]]
        return t

    def run(self, bounds=True, strided=False, lse=True, session=None, stream=None):
        T = self.q.shape[0]
        pages = self.pages()
        q, out = self.q.cuda(), torch.full((T, self.H, self.D), 9.0, dtype=self.dtype, device="cuda")
        if strided:
            row = torch.full((T, self.H + 3, self.D), 4.0, dtype=self.dtype, device="cuda")
            row[:, 1:1 + self.H] = q
            q, out = row[:, 1:1 + self.H], torch.full((self.H, T, self.D), 9.0, dtype=self.dtype, device="cuda").transpose(0, 1)
        l = torch.full((T, self.H), 9.0, device="cuda") if lse else None
        s = session or B.hps_seq_attention_create(max(T * self.H, 1), self.D)
        kw = dict(self.bounds) if bounds else {}
        if len(self.prefix_lens):
            kw.update(prefix_table=self.prefix_table.cuda(), prefix_lens=self.prefix_lens.cuda(), group_offsets=self.group_offsets.cuda())
        args = self.block_table.cuda(), self.lens.cuda(), self.offsets.cuda()
        torch.cuda.synchronize()
        B.hps_seq_attention_packed(s, q, pages, *args, out, lse=l, scale=self.scale, stream=stream, **kw)
        torch.cuda.synchronize()
        self.flags = B.hps_seq_attention_flags(s, clear=True)
        if session is None:
            B.hps_seq_attention_destroy(s)
        return out.cpu(), l.cpu() if lse else None


MANY = [(9, 7), (40, 11), (1, 1), (130, 3), (64, 20), (3, 3)]


class Shared(Packed):
    """Bounds that are far beyond the lengths, so that work-groups of many rows, which share keys, are taken for histories and own tokens alike."""

    def run(self, **kw):
        T, near = self.q.shape[0], dict(self.bounds)
        if kw.get("bounds", True):
            self.bounds = dict(max_new=T, max_group=T, max_len=1 << 25, max_prefix=(1 << 25) if len(self.prefix_lens) else 0)
            self.bounds = {**self.bounds, **{k: v for k, v in near.items() if v == 0}}
        try:
            return super().run(**kw)
        finally:
            self.bounds = near


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 256])
def test_head_dims(D, dtype):
    Packed(dtype, D, 4, 2, 16, [(77, 4), (130, 2)], MIXED, seed=D).check()
    Packed(dtype, D, 8, 2, 32, [(300, 3), (45, 3)], [(9, 4), (40, 1), (1, 1), (130, 3), (64, 4), (3, 3)], seed=D + 2).check()        # 17 to 32 rows
    Packed(dtype, D, 8, 1, 32, [(200, 6)], MANY, seed=D + 1).check()
    Shared(dtype, D, 8, 1, 32, [(200, 6)], MANY, seed=D + 1).check()


@pytest.mark.parametrize("H,K", [(1, 1), (5, 5), (8, 2), (12, 3), (16, 1), (32, 8), (40, 1), (33, 11)])
def test_heads(H, K):
    Packed(BF, 64, H, K, 16, [(100, 3), (33, 3)], MIXED, seed=H).check()


@pytest.mark.parametrize("block", [16, 32, 64, 128, 1024])
def test_block_sizes(block):
    for dtype, D in ((BF, 128), (HF, 64), (BF, 96)):
        Packed(dtype, D, 4, 2, block, [(150, 6)], MIXED, seed=block).check()
        for kind in (Packed, Shared):
            kind(dtype, D, 16, 2, block, [(300, 6)], [(100, 9), (20, 20), (65, 7), (1, 1), (300, 2), (64, 5)], seed=block).check()


@pytest.mark.parametrize("n", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000])
def test_lengths(n):
    """Histories and own tokens that end at, in front of and behind the steps of the kernels."""
    for new in (1, 8):
        own = max(n, new)
        Packed(BF, 64, 4, 4, 16, [(n, 2)], [(own, new), (new, new)], seed=n).check()
        Packed(BF, 128, 16, 2, 16, [(n, 2)], [(own, new), (new, new)], seed=n + 1).check()
        Packed(HF, 64, 4, 1, 64, [], [(own, new), (new, 1)], seed=n + 2).check()
    for D in (64, 128):
        Shared(BF, D, 16, 1, 16, [(n, 2)], [(max(n, 8), 8), (8, 8)], seed=n + 3).check()


@pytest.mark.parametrize("rows", [1, 4, 15, 16, 17, 31, 32, 33, 64, 127, 128, 129, 300])
def test_rows(rows):
    Packed(BF, 64, 2, 2, 16, [(270, rows)], [(3, 1)] * rows, seed=rows).check()
    Packed(BF, 64, 2, 1, 16, [(90, 1)], [(rows + 5, rows)], seed=rows).check()
    if rows > 100:
        Shared(BF, 64, 2, 2, 16, [(270, rows)], [(3, 1)] * rows, seed=rows).check()
        Shared(BF, 64, 2, 1, 16, [(90, 1)], [(rows + 5, rows)], seed=rows).check()


@pytest.mark.parametrize("layout", ["heads first", "apart"])
def test_layouts_and_strides(layout):
    Packed(BF, 96, 6, 3, 16, [(140, 6)], MIXED, layout=layout).check(strided=True)
    Packed(HF, 128, 12, 3, 32, [(140, 6)], [(60, 9)] * 6, layout=layout).check(strided=True)
    Shared(HF, 128, 12, 3, 32, [(140, 6)], [(60, 9)] * 6, layout=layout).check(strided=True)


def test_long_prompts_without_a_history():
    for kind in (Packed, Shared):
        kind(BF, 128, 4, 1, 16, [], [(513, 513), (700, 300), (40, 40)]).check()
        kind(HF, 64, 2, 2, 64, [], [(1, 1), (1500, 257)]).check()


def test_long_stretches_are_cut_and_joined():
    Packed(BF, 64, 4, 2, 16, [(9001, 2)], [(5, 1), (1, 1)]).check()
    Packed(BF, 64, 4, 2, 16, [], [(9001, 1), (7777, 2)]).check()
    Packed(HF, 128, 8, 1, 64, [(6000, 3)], [(2500, 8), (3000, 2), (64, 1)]).check()
    Shared(HF, 128, 32, 1, 64, [(6000, 3)], [(2500, 8), (3000, 2), (64, 1)]).check()
    p = Packed(BF, 32, 128, 1, 16, [(40000, 16)], [(3, 1)] * 16)             # 2,048 rows and near bounds: many rows and several chunks
    p.check()


def test_many_groups_and_requests():
    groups = [(n, 1 + i % 4) for i, n in enumerate((0, 3, 500, 64, 65, 1, 200, 31, 90, 100, 7))]
    n = sum(g[1] for g in groups)
    Packed(BF, 64, 8, 2, 16, groups, [(1 + i * 7 % 50, 1 + i % 2) for i in range(n)]).check()
    for kind in (Packed, Shared):
        kind(BF, 64, 8, 2, 16, groups, [(60 + i * 7 % 50, 1 + i * 5 % 40) for i in range(n)]).check()
    Packed(BF, 32, 4, 4, 16, [(70, 300)], [(1 + i % 60, 1) for i in range(300)]).check()      # a wave to a request


@pytest.mark.parametrize("new", [1, 30])
def test_rows_that_attend_to_nothing(new):
    """No history and no own tokens; new tokens that are not all in the length; requests without new tokens; requests of no group; tokens of no request."""
    kind = Shared if new == 30 else Packed
    p = kind(BF, 64, 4, 2, 16, [(0, 2), (40, 2)], [(0, 0), (new, new), (50, 0), (new, new), (4 + new, new), (7 + new, new)], tail=3)
    p.check()
    p = kind(BF, 64, 4, 2, 16, [(0, 1), (40, 1)], [(new, new), (new, new), (new, new)], tail=2)
    p.lens = torch.tensor([0, new // 2, 0], dtype=torch.int32)
    p.check()
    p.group_offsets = torch.tensor([1, 1, 2], dtype=torch.int32)
    p.check()
    p.check(bounds=False)
    p.check(lse=False)
    Packed(BF, 64, 4, 2, 16, [], [(0, 0), (0, 0)], tail=3).check()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [64, 96, 128])
def test_what_is_hidden_has_no_part(D, dtype):
    """Groups of keys and values behind a query's own place that are no numbers (the pool's unused places are in every test)."""
    for kind, H, K, new in ((Packed, 4, 4, 13), (Packed, 4, 2, 13), (Packed, 16, 2, 20), (Shared, 16, 1, 16), (Shared, 32, 2, 24)):      # up to 16 rows, up to 32, more, many
        p = kind(dtype, D, H, K, 16, [(50, 1)], [(40, new)], seed=5)
        for i, d in ((39, 3), (38, 60), (35, 33), (31, D - 1)):
            b = int(p.block_table[0, i // 16])
            p.v[b, i % 16, 0, d] = math.inf if i == 38 else math.nan
        p.v[int(p.block_table[0, 2]), 4, K - 1, 5] = math.nan                # token 36
        out, lse = p.run()
        want, want_lse, bound, lse_bound = p.want()
        assert torch.isnan(out[-1]).any() and torch.isfinite(out[0]).all() and torch.isfinite(lse).all()
        R.close(out, want, bound)
        R.close(lse, want_lse, lse_bound)
        p.k[int(p.block_table[0, 2]), 5] = math.nan                          # token 37, whole
        out, lse = p.run()
        first = 37 - (40 - new)
        assert torch.isnan(out[first:]).all() and torch.isnan(lse[first:]).all()
        R.close(out[:first], want[:first], bound[:first])
        R.close(lse[:first], want_lse[:first], lse_bound[:first])
        p.v[int(p.prefix_table[0, 0]), 3, :, 1] = math.nan                   # of the history: every row sees it
        out, _ = p.run()
        assert torch.isnan(out[:, :, :32]).all() and torch.isfinite(out[0, :, 32:]).all()       # the first query sees none of the others


@pytest.mark.parametrize("kind,H,K,new", [(Packed, 2, 2, 1), (Packed, 16, 1, 9), (Shared, 16, 1, 16)])
def test_scales_beyond_the_type(kind, H, K, new):
    """Scale bytes above the type's last one stand for NaN, as 255 does; 0 stands for 2^-127."""
    for dtype, last in ((BF, 252), (HF, 140)):
        p = kind(dtype, 64, H, K, 16, [(40, 1)], [(new, new)], seed=7)
        tiles = p.tiles()
        vs = P.places(16, 64)[3]
        b = int(p.prefix_table[0, 1])
        tiles[b, 0, vs[3, 0]], tiles[b, 0, vs[4, 1]] = 0, 0
        p.tiles = lambda: tiles
        p.check()
        for byte in (last + 1, 254, 255):
            tiles[b, 0, vs[3, 0]] = byte
            out, _ = p.run()
            want, _, bound, _ = p.want()
            assert torch.isnan(out[:, :H // K, :32]).all() and torch.isfinite(out[:, :, 32:]).all()
            R.close(out, want, bound)


def test_extreme_scores():
    """Scores that grow along the keys, fall, and are far apart: the running reference and what is joined."""
    for kind, H, K, new in ((Packed, 2, 2, 1), (Packed, 8, 2, 6), (Packed, 8, 1, 8), (Shared, 32, 1, 8)):
        for sign in (1, -1):
            p = kind(BF, 64, H, K, 16, [(700, 1)], [(new + 40, new)], seed=2, scale=1.0)
            p.q[:] = 1
            for t, n in ((p.prefix_table[0], 700), (p.block_table[0], new + 40)):
                for i in range(n):
                    p.k[int(t[i // 16]), i % 16] = sign * (i - 300) / 64
            p.check()


@pytest.mark.parametrize("kind,H,K,new", [(Packed, 2, 2, 1), (Packed, 8, 2, 6), (Packed, 16, 1, 9), (Shared, 16, 1, 16)])
def test_large_values_behind_growing_scores(kind, H, K, new):
    """The sums are formed against a reference that may lie behind the largest score: they have room for values of 2^80."""
    p = kind(BF, 64, H, K, 16, [(3000, 1)], [(new + 40, new)], seed=4, scale=1.0)
    p.q[:] = 1
    for i in range(3000):
        p.k[int(p.prefix_table[0, i // 16]), i % 16] = i / 1280
    p.v *= 2.0 ** 80
    p.check()
    p.v *= 2.0 ** -160                                 # and small ones are not lost
    p.check()


@pytest.mark.parametrize("kind,H,K,new", [(Packed, 2, 2, 1), (Packed, 4, 4, 20), (Shared, 16, 1, 20)])
def test_odd_queries_spoil_their_own_rows_only(kind, H, K, new):
    for odd in (math.nan, math.inf):
        p = kind(BF, 64, H, K, 16, [(700, 2)], [(new + 40, new), (new, new)], seed=6)
        p.q[0, 1], p.q[new, 0, 7] = odd, odd
        if new > 1:
            p.q[new - 1, H - 1, 63] = odd
        for offsets in ([0, 2], [0, 0]):               # with and without the history
            p.group_offsets = torch.tensor(offsets, dtype=torch.int32)
            out, lse = p.run()
            clean = torch.ones(2 * new, H, dtype=torch.bool)
            clean[0, 1], clean[new, 0] = False, False
            if new > 1:
                clean[new - 1, H - 1] = False
            want, want_lse, bound, lse_bound = p.want()
            assert torch.isfinite(out[clean]).all() and torch.isfinite(lse[clean]).all()
            R.close(out[clean], want[clean], bound[clean])
            R.close(lse[clean], want_lse[clean], lse_bound[clean])


@pytest.mark.parametrize("kind,H,new", [(Packed, 16, 1), (Shared, 64, 16)])
def test_pages_behind_four_gibibytes(kind, H, new):
    """Blocks that are more than 2^32 bytes from the first one."""
    K, D, block = 8, 128, 64
    p = kind(BF, D, H, K, block, [(500, 2)], [(4 + new, new), (70, new)], spare=0)
    tiles = p.tiles()
    n_blocks = (5 << 30) // (K * tiles.shape[2])
    pool = torch.zeros(n_blocks, K, tiles.shape[2], dtype=torch.uint8, device="cuda")
    shift = n_blocks - p.n_blocks
    pool[shift:] = tiles.cuda()
    want, _, bound, _ = p.want()
    p.pages = lambda: pool
    p.prefix_table, p.block_table = (torch.where(t < 0, t, t + shift) for t in (p.prefix_table, p.block_table))
    out, _ = p.run()
    assert p.flags == 0
    R.close(out, want, bound)


@pytest.mark.parametrize("H,K", [(4, 2), (64, 2)])
def test_flags(H, K):
    p = Packed(BF, 64, H, K, 16, [(100, 2)], [(5, 1), (40, 2)], loose=1)
    p.check(bounds=False)
    bad = dict(max_new=1, max_len=39, max_prefix=99, max_group=2)
    for name, value in bad.items():
        p.bounds = {**dict(max_new=2, max_len=40, max_prefix=100, max_group=3), name: value}
        p.run()
        assert p.flags == B.HPS_SEQ_FLAG_LENGTH, name
        p.bounds = dict(max_new=2, max_len=40, max_prefix=100)
    p.lens[1] = 10 ** 9
    p.run(bounds=False)
    assert p.flags == B.HPS_SEQ_FLAG_LENGTH | B.HPS_SEQ_FLAG_BLOCK     # cut to what the table holds, whose last entry is no block
    for junk in (-1, 10 ** 6):                         # a block that is none stands for zeros
        p = Packed(BF, 64, H, K, 16, [(100, 2)], [(5, 1), (40, 2)])
        p.prefix_table[0, 3], p.block_table[1, 1] = junk, junk
        out, lse = p.run()
        assert p.flags == B.HPS_SEQ_FLAG_BLOCK
        want, want_lse, bound, lse_bound = p.want()
        R.close(out, want, bound)
        R.close(lse, want_lse, lse_bound)
    for junk in (-1, 10 ** 6):                         # to work-groups that share keys too
        p = Shared(BF, 64, 64, 1, 16, [(100, 2)], [(5, 1), (40, 3)])
        p.prefix_table[0, 3], p.block_table[1, 1] = junk, junk
        out, lse = p.run()
        assert p.flags == B.HPS_SEQ_FLAG_BLOCK
        want, want_lse, bound, lse_bound = p.want()
        R.close(out, want, bound)
        R.close(lse, want_lse, lse_bound)
    for bounds in (dict(max_prefix=0), dict(max_group=0)):             # a bound of 0 leaves the histories out, and tells
        p = Packed(BF, 64, H, K, 16, [(100, 2)], [(5, 1), (40, 2)])
        p.bounds.update(bounds)
        p.run()
        assert p.flags == B.HPS_SEQ_FLAG_LENGTH


@pytest.mark.parametrize("kind,H", [(Packed, 4), (Shared, 256)])
def test_no_blocks_at_all(kind, H):
    """Pages without blocks: every token stands for zeros."""
    p = kind(BF, 64, H, 2, 16, [(100, 2)], [(5, 1), (40, 2)])
    p.pages = lambda: torch.empty(0, 2, 16 * 68, dtype=torch.uint8, device="cuda")
    out, lse = p.run()
    assert p.flags == B.HPS_SEQ_FLAG_BLOCK and (out == 0).all()
    keys = torch.tensor([105.0, 139, 140], dtype=torch.float64)
    R.close(lse, keys.log()[:, None].expand(3, H), torch.tensor(1e-5, dtype=torch.float64))


def test_refusals():
    p = Packed(BF, 64, 4, 2, 16, [(100, 2)], [(5, 1), (40, 2)])
    s = B.hps_seq_attention_create(12, 64)
    pages = p.pages()
    args = [p.q.cuda(), pages, p.block_table.cuda(), p.lens.cuda(), p.offsets.cuda(), torch.empty(3, 4, 64, dtype=BF, device="cuda")]
    kw = dict(prefix_table=p.prefix_table.cuda(), prefix_lens=p.prefix_lens.cuda(), group_offsets=p.group_offsets.cuda())

    def refuse(error, at=None, value=None, match=None, **more):
        a = list(args)
        if at is not None:
            a[at] = value
        with pytest.raises(error, match=match):
            B.hps_seq_attention_packed(s, *a, **{**kw, **more})

    refuse(TypeError, 0, args[0].cpu())
    refuse(ValueError, 0, args[0][:, :, :32])
    refuse(ValueError, 0, args[0].transpose(1, 2))
    refuse(TypeError, 1, pages.int())
    refuse(ValueError, 1, pages[0])
    refuse(ValueError, 1, pages[:, :, :-1])
    refuse(ValueError, 1, pages.transpose(1, 2))
    refuse(B.HpsError, 1, torch.zeros(4, 2, 24 * 68, dtype=torch.uint8, device="cuda"), match="block_size")
    refuse(B.HpsError, 1, torch.zeros(4, 2, 8 * 68, dtype=torch.uint8, device="cuda"), match="block_size")
    wide = torch.zeros(4, 2, 16 * 68 + 8, dtype=torch.uint8, device="cuda")
    refuse(B.HpsError, 1, wide[:, :, :16 * 68], match="16")
    refuse(B.HpsError, 1, torch.zeros(8 * 16 * 68 + 8, dtype=torch.uint8, device="cuda")[8:].view(4, 2, 16 * 68), match="16")
    refuse(ValueError, 2, args[2][0])
    refuse(TypeError, 3, args[3].long())
    refuse(ValueError, 4, args[4][:2])
    refuse(ValueError, 5, args[5][:2])
    refuse(ValueError, prefix_table=None)
    refuse(ValueError, lse=torch.empty(3, 3, device="cuda"))
    for scale in (0.0, -1.0, math.inf, math.nan):
        refuse(B.HpsError, scale=scale)
    with pytest.raises(B.HpsError, match="dtype"):
        B.hps_seq_attention_packed(s, args[0].float(), *args[1:5], args[5].float(), **kw)
    odd = torch.zeros(3, 4, 40, dtype=BF, device="cuda")
    with pytest.raises(B.HpsError, match="head_dim"):
        B.hps_seq_attention_packed(s, odd, torch.zeros(4, 2, 16 * 40 * 17 // 16, dtype=torch.uint8, device="cuda"), *args[2:5], odd.clone(), **kw)
    torch.cuda.synchronize()
    assert B.hps_seq_attention_flags(s) == 0
    B.hps_seq_attention_destroy(s)


def test_one_session_for_both_kinds_of_pages_and_another_stream():
    s, st = B.hps_seq_attention_create(4096, 128), torch.cuda.Stream()
    for seed, (groups, requests) in enumerate([([(3000, 3)], [(9, 1)] * 3), ([(5, 2)], [(900, 2), (3, 1)]), ([], [(40, 40)]), ([(64, 40)], [(2, 2)] * 40), ([(0, 1), (7, 1)], [(1, 1)] * 3)]):
        for D in (64, 128):
            Packed(BF, D, 4, 2, 16, groups, requests, seed=seed).check(session=s, stream=st)
            Problem(BF, D, 4, 2, 16, groups, requests, seed=seed).check(session=s, stream=st)
    B.hps_seq_attention_destroy(s)


def test_two_sessions_side_by_side():
    """Two calls at a time on streams of their own."""
    ps = [Packed(BF, 64, 8, 2, 16, [(3000, 3)], [(9, 1)] * 3, seed=1), Packed(BF, 64, 8, 2, 16, [(2000, 30)], [(40, 3)] * 30, seed=2)]
    sessions, streams, outs = [B.hps_seq_attention_create(1024, 64) for _ in ps], [torch.cuda.Stream() for _ in ps], []
    args = [[x.cuda() for x in (p.q, p.tiles(), p.block_table, p.lens, p.offsets)] for p in ps]
    kws = [dict(prefix_table=p.prefix_table.cuda(), prefix_lens=p.prefix_lens.cuda(), group_offsets=p.group_offsets.cuda(), **p.bounds) for p in ps]
    outs = [torch.empty_like(a[0]) for a in args]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, st, a, o, kw in zip(sessions, streams, args, outs, kws):
            B.hps_seq_attention_packed(s, *a, o, stream=st, **kw)
    torch.cuda.synchronize()
    for p, o, s in zip(ps, outs, sessions):
        want, _, bound, _ = p.want()
        R.close(o.cpu(), want, bound)
        B.hps_seq_attention_destroy(s)


@pytest.mark.parametrize("H", [8, 64])
def test_graph_replays_on_new_lengths(H):
    p = Packed(BF, 64, H, 2, 16, [(300, 3), (70, 2)], [(40, 2), (20, 1), (33, 4), (16, 1), (50, 2)])
    if H == 64:                                        # many rows share keys
        p.bounds = dict(max_new=10, max_len=1 << 25, max_prefix=1 << 25)
    pages = p.pages()
    T = p.q.shape[0]
    s, out, lse = B.hps_seq_attention_create(T * H, 64), torch.zeros(T, H, 64, dtype=BF, device="cuda"), torch.zeros(T, H, device="cuda")
    q, lens, prefix, table, offsets, ptable, groups = (x.cuda() for x in (p.q, p.lens, p.prefix_lens, p.block_table, p.offsets, p.prefix_table, p.group_offsets))

    def call():
        B.hps_seq_attention_packed(s, q, pages, table, lens, offsets, out, prefix_table=ptable, prefix_lens=prefix, group_offsets=groups, lse=lse, **p.bounds)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for own, shared in (([40, 20, 33, 16, 50], [300, 70]), ([2, 0, 4, 1, 49], [0, 70]), ([17, 20, 5, 16, 2], [129, 1]), ([40, 20, 33, 16, 50], [300, 70])):
        p.lens, p.prefix_lens = torch.tensor(own, dtype=torch.int32), torch.tensor(shared, dtype=torch.int32)
        lens.copy_(p.lens), prefix.copy_(p.prefix_lens), out.fill_(3), lse.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, want_lse, bound, lse_bound = p.want()
        R.close(out.cpu(), want, bound)
        R.close(lse.cpu(), want_lse, lse_bound)
        got = out.clone()
        call()
        assert torch.equal(got, out)                   # the same call gives the same bits
    B.hps_seq_attention_destroy(s)


@pytest.mark.parametrize("new", [1, 20])
def test_tokens_behind_the_last_query(new):
    """Offsets may count more tokens than there are queries for: the others' places in their requests stay what they are."""
    p = (Shared if new == 20 else Packed)(BF, 64, 32, 2, 16, [(40, 2)], [(new, new), (50 + new, 2 * new)], seed=new)
    want, want_lse, bound, lse_bound = p.want()
    T = new + max(1, new // 2)
    p.q = p.q[:T]
    out, lse = p.run()
    assert p.flags == 0
    R.close(out, want[:T], bound[:T])
    R.close(lse, want_lse[:T], lse_bound[:T])


@pytest.mark.parametrize("H,K,requests", [(4, 2, [(5, 1), (40, 2)]), (16, 1, [(60, 9), (9, 9)]), (2, 2, [(33, 1)] * 300), (2, 2, [(700, 1), (2000, 2)])])
def test_scores_of_minus_infinity(H, K, requests):
    """Rows whose scores are all minus infinity get 0, whatever the values and however the keys are cut."""
    for groups, kind in (([], Packed), ([(100, len(requests))], Packed), ([(100, len(requests))], Shared)):
        p = kind(BF, 64, H, K, 16, groups, requests)
        p.q[:] = 1
        for t, n in [(p.block_table[r], int(n)) for r, n in enumerate(p.lens)] + [(p.prefix_table[g], int(n)) for g, n in enumerate(p.prefix_lens)]:
            place = torch.arange(n)
            p.k[t.long()[place // 16], place % 16] = -torch.finfo(BF).max
        out, lse = p.run()
        assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF, HF])
def test_a_step_of_a_server(dtype):
    """Pages for new tokens, queries and keys normed, turned and stored, attention: together, against all of it in 64 bits; then the next step."""
    H, K, D, block, eps = 8, 2, 64, 16, 1e-6
    g = torch.Generator().manual_seed(3)
    users, steps = 3, ((37, 20, 1), (1, 3, 1), (2, 1, 17))
    n_blocks, width = 40, 8
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    free, info, table_of_blocks = torch.randperm(n_blocks, generator=g).int().cuda(), torch.tensor([n_blocks, 0, 0, 0], dtype=torch.int32, device="cuda"), torch.full((users, width), -1, dtype=torch.int32, device="cuda")
    pages = torch.full((n_blocks, K, B.hps_seq_packed_bytes(block, D)), 255, dtype=torch.uint8, device="cuda")
    table = torch.empty(128, D // 2, 2, device="cuda")
    B.hps_seq_rope_table(table)
    qw, kw = 1 + 0.3 * torch.randn(D, generator=g), 1 + 0.3 * torch.randn(D, generator=g)
    past, s = i32(users), B.hps_seq_attention_create(128 * H, D)
    history = [[] for _ in range(users)]               # each user's keys and values as the pages hold them, in 64 bits
    for new in steps:
        T = sum(new)
        offsets, lens, slots, positions, more = i32(users + 1), i32(users), i32(T + 3), i32(T + 3), i32(4)
        B.hps_seq_extend(past, torch.tensor(new, dtype=torch.int32, device="cuda"), block, free, info, table_of_blocks, offsets, lens, slots, positions, more)
        x = torch.randn(T + 3, H + 2 * K, D, generator=g).to(dtype)
        xd = x.cuda()
        q, out, lse = torch.full((T + 3, H, D), 9.0, dtype=dtype, device="cuda"), torch.full((T + 3, H, D), 9.0, dtype=dtype, device="cuda"), torch.full((T + 3, H), 9.0, device="cuda")
        B.hps_seq_append_packed(xd[:, H:H + K], xd[:, H + K:], pages, slots, q=xd[:, :H], q_out=q, positions=positions, table=table, norm=True, q_weight=qw.cuda(), k_weight=kw.cuda(), eps=eps)
        B.hps_seq_attention_packed(s, q, pages, table_of_blocks, lens, offsets, out, lse=lse, max_new=max(new), max_len=width * block)
        torch.cuda.synchronize()
        assert B.hps_seq_attention_flags(s) == 0 and (out[T:] == 9).all() and (q[T:] == 9).all()
        at = positions.cpu()
        keys = P.turned(P.normed(x[:T, H:H + K].double(), kw, eps), at[:T], table.cpu(), False)
        k, v = P.values(*P.quantised(keys, dtype)), P.values(*P.quantised(x[:T, H + K:].double(), dtype))
        want_q, q_bound = P.norm_rope(x[:T, :H], qw, at[:T], table.cpu(), eps, False)
        R.close(q[:T].cpu(), want_q, q_bound)
        t = 0
        for u, n in enumerate(new):
            history[u] += [(k[t + i], v[t + i]) for i in range(n)]
            kk, vv = (torch.stack(y) for y in zip(*history[u]))
            one = torch.zeros(1, len(kk), K, D, dtype=torch.float64), torch.zeros(1, len(kk), K, D, dtype=torch.float64)
            one[0][0], one[1][0] = kk, vv
            want, want_lse, bound, lse_bound = R.attention(q[t:t + n].cpu(), *one, torch.zeros(1, 1, dtype=torch.int32), torch.tensor([len(kk)]), torch.tensor([0, n]), D ** -0.5)
            R.close(out[t:t + n].cpu(), want, bound)
            R.close(lse[t:t + n].cpu(), want_lse, lse_bound)
            t += n
        past, info = lens, more
    B.hps_seq_attention_destroy(s)


@pytest.mark.parametrize("bounds", [{}, dict(max_new=16)])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_many_requests_without_anything_to_attend_to(D, bounds):
    """Tables of width 0 and no history: every row gets 0, whichever kernel the number of rows asks for."""
    n, new, H, K = 512, 16, 32, 8
    q = torch.ones(n * new, H, D, dtype=BF, device="cuda")
    out, lse = torch.full_like(q, 9.0), torch.full((n * new, H), 9.0, device="cuda")
    pages = torch.zeros(4, K, B.hps_seq_packed_bytes(16, D), dtype=torch.uint8, device="cuda")
    offsets = torch.arange(0, n * new + 1, new, dtype=torch.int32, device="cuda")
    s = B.hps_seq_attention_create(n * new * H, D)
    B.hps_seq_attention_packed(s, q, pages, torch.empty(n, 0, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"), offsets, out, lse=lse, **bounds)
    torch.cuda.synchronize()
    flags = B.hps_seq_attention_flags(s)
    B.hps_seq_attention_destroy(s)
    assert flags == 0 and (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [32, 64, 96, 128])
def test_many_rows_do_not_see_what_a_kernel_left(D, dtype):
    """The same bits, whether the kernel in front left zeros or infinities in the LDS of every CU."""
    def leave(x):
        pages, out = torch.full((4, 64, 16, 256), x, dtype=BF, device="cuda"), torch.empty(128, 16, 256, dtype=BF, device="cuda")
        s = B.hps_seq_attention_create(128 * 16, 256)
        B.hps_seq_attention(s, torch.ones_like(out), pages, pages.clone(), torch.arange(4, dtype=torch.int32, device="cuda").repeat(128, 1),
                            torch.full((128,), 256, dtype=torch.int32, device="cuda"), torch.arange(129, dtype=torch.int32, device="cuda"), out, max_new=1)
        torch.cuda.synchronize()
        B.hps_seq_attention_destroy(s)

    p = Shared(dtype, D, 8, 1, 32, [(200, 6)], MANY, seed=D)
    p.q[:] = 0                                         # equal weights, and values that cancel: sums in another order are other sums
    for table, n in zip(p.block_table, p.lens.tolist()):
        for i in range(n):
            at, big = (int(table[i // 32]), i % 32), torch.randn(1, D, generator=torch.Generator().manual_seed(i // 3))
            p.v[at] = (big * (2.0 ** 10, -2.0 ** 10, 2.0 ** -12)[i % 3]).to(dtype)
    leave(0.0)
    want = p.run()
    leave(math.inf)
    got = p.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 256])
def test_hidden_groups_of_every_head_size(D, dtype):
    """Groups of keys and of values behind a query's own place that are no numbers, in each of a head's groups."""
    for kind, H, K, new in ((Packed, 4, 4, 13), (Packed, 4, 2, 13), (Packed, 16, 2, 20), (Shared, 16, 1, 16), (Shared, 32, 2, 24)):      # up to 16 rows, up to 32, more, many
        for group in range(D // 32):
            p = kind(dtype, D, H, K, 16, [(50, 1)], [(40, new)], seed=5)
            p.v[int(p.block_table[0, 2]), 6, 0, 32 * group + 7 * group % 32] = math.nan         # token 38
            p.v[int(p.block_table[0, 1]), 15, K - 1, 32 * group + 31] = math.inf                # token 31
            out, lse = p.run()
            want, want_lse, bound, lse_bound = p.want()
            assert torch.isnan(out[-1]).any() and torch.isfinite(lse).all()
            R.close(out, want, bound)
            R.close(lse, want_lse, lse_bound)
            p.k[int(p.block_table[0, 2]), 5, :, 32 * group + 9] = math.nan                      # token 37: a group of every head
            out, lse = p.run()
            first = 37 - (40 - new)
            assert torch.isnan(out[first:]).all() and torch.isnan(lse[first:]).all()
            R.close(out[:first], want[:first], bound[:first])
            R.close(lse[:first], want_lse[:first], lse_bound[:first])


@pytest.mark.parametrize("D", [32, 96, 128, 256])
@pytest.mark.parametrize("kind,H,K,new", [(Packed, 2, 2, 1), (Packed, 16, 1, 9), (Shared, 16, 1, 16)])
def test_scales_beyond_the_type_of_every_head_size(kind, H, K, new, D):
    """Scale bytes above the type's last one, and 0, in each of a head's groups, of values and of keys."""
    for dtype, last in ((BF, 252), (HF, 140)):
        for group in range(D // 32):
            p = kind(dtype, D, H, K, 16, [(40, 1)], [(new, new)], seed=7)
            tiles = p.tiles()
            _, _, ks, vs = P.places(16, D)
            b = int(p.prefix_table[0, 1])
            tiles[b, 0, vs[3, group]], tiles[b, 0, ks[5, group]] = 0, 0
            p.tiles = lambda: tiles  # noqa: B023
            p.check()
            for byte in (last + 1, 255):
                tiles[b, 0, vs[3, group]] = byte
                out, lse = p.run()
                want, _, bound, _ = p.want()
                spoilt = torch.zeros(D, dtype=torch.bool)
                spoilt[32 * group:32 * group + 32] = True
                assert torch.isnan(out[:, :H // K, spoilt]).all() and torch.isfinite(out[:, :, ~spoilt]).all() and torch.isfinite(lse).all()
                R.close(out, want, bound)
            tiles[b, 0, vs[3, group]], tiles[b, 0, ks[5, group]] = 0, last + 1
            out, lse = p.run()
            assert torch.isnan(out[:, :H // K]).all() and torch.isnan(lse[:, :H // K]).all()
            assert torch.isfinite(out[:, H // K:]).all() and torch.isfinite(lse[:, H // K:]).all()
