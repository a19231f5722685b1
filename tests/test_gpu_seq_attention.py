"""Attention behind shared histories (hps_seq_attention) against the definition in 64 bits."""
import math

import pytest
import torch

import seq_reference as R
from paper_2210_08804_amd import binding as B

pytestmark = pytest.mark.gpu


class Problem:
    """Requests in groups, their pages scattered over a pool whose other places hold `junk`."""

    def __init__(self, dtype, D, H, K, block, groups, requests, seed=0, junk=math.nan, layout="places first", spare=3, tail=0, scale=None, loose=0):
        """groups: [(history length, requests)]; requests: [(own length, new tokens)], in the groups' order, more of them are in no group."""
        g = self.g = torch.Generator().manual_seed(seed)
        self.D, self.H, self.K, self.block, self.dtype = D, H, K, block, dtype
        lens, new = [r[0] for r in requests], [r[1] for r in requests]
        blocks = lambda n: -(-n // block)  # noqa: E731
        need = sum(blocks(p) for p, _ in groups) + sum(blocks(n) for n in lens)
        self.n_blocks = need + spare
        order = torch.randperm(self.n_blocks, generator=g).int()
        table = lambda ns, width: torch.full((len(ns), width), -1, dtype=torch.int32)  # noqa: E731
        self.prefix_lens, self.lens = torch.tensor([p for p, _ in groups], dtype=torch.int32), torch.tensor(lens, dtype=torch.int32)
        self.prefix_table = table(groups, max([blocks(p) for p, _ in groups], default=0) + loose)
        self.block_table = table(lens, max([blocks(n) for n in lens], default=0) + loose)
        T = sum(new) + tail
        self.q = (torch.randn(T, H, D, generator=g) * 1.5).to(dtype)
        self.k, self.v = (torch.full((self.n_blocks, block, K, D), junk, dtype=dtype) for _ in range(2))
        at = 0
        for t, ns in ((self.prefix_table, self.prefix_lens.tolist()), (self.block_table, lens)):
            for i, n in enumerate(ns):
                t[i, :blocks(n)] = order[at:at + blocks(n)]
                at += blocks(n)
                place = torch.arange(n)
                b = t[i, :].long()[place // block]
                self.k[b, place % block] = torch.randn(n, K, D, generator=g).to(dtype)
                self.v[b, place % block] = torch.randn(n, K, D, generator=g).to(dtype)
        self.offsets = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).int()
        self.group_offsets = torch.tensor([0] + [n for _, n in groups], dtype=torch.int32).cumsum(0).int()
        self.scale, self.layout = scale, layout
        self.bounds = dict(max_new=max(new, default=0), max_len=max(lens, default=0), max_prefix=max([p for p, _ in groups], default=0))

    def pages(self):
        if self.layout == "places first":
            return self.k.cuda(), self.v.cuda()
        if self.layout == "heads first":
            return [x.transpose(1, 2).contiguous().cuda().transpose(1, 2) for x in (self.k, self.v)]
        both = torch.stack((self.k, self.v), 1).cuda()
        return both[:, 0], both[:, 1]

    def want(self):
        return R.attention(self.q, self.k, self.v, self.block_table, self.lens, self.offsets, self.scale or self.D ** -0.5,
                           *((self.prefix_table, self.prefix_lens, self.group_offsets) if len(self.prefix_lens) else ()))

    def run(self, bounds=True, strided=False, lse=True, session=None, stream=None):
        T = self.q.shape[0]
        k, v = self.pages()
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
        B.hps_seq_attention(s, q, k, v, self.block_table.cuda(), self.lens.cuda(), self.offsets.cuda(), out, lse=l, scale=self.scale, stream=stream, **kw)
        torch.cuda.synchronize()
        self.flags = B.hps_seq_attention_flags(s, clear=True)
        if session is None:
            B.hps_seq_attention_destroy(s)
        return out.cpu(), l.cpu() if lse else None

    def check(self, **kw):
        out, lse = self.run(**kw)
        assert self.flags == 0
        want, want_lse, bound, lse_bound = self.want()
        n = int(self.offsets[-1])
        R.close(out[:n], want[:n], bound[:n])
        assert (out[n:] == 9).all()                    # rows of tokens behind the last request's
        if lse is not None:
            R.close(lse[:n], want_lse[:n], lse_bound[:n])
            assert (lse[n:] == 9).all()


BF, HF = torch.bfloat16, torch.float16
MIXED = [(5, 1), (1, 1), (17, 3), (33, 1), (64, 2), (2, 2)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("D", [8, 32, 40, 64, 72, 96, 104, 128, 136, 200, 256])
def test_head_dims(D, dtype):
    Problem(dtype, D, 4, 2, 16, [(77, 4), (130, 2)], MIXED, seed=D).check()
    Problem(dtype, D, 8, 1, 32, [(200, 6)], [(9, 7), (40, 11), (1, 1), (130, 3), (64, 20), (3, 3)], seed=D + 1).check()      # many rows: work-groups share the keys


@pytest.mark.parametrize("H,K", [(1, 1), (5, 5), (8, 2), (12, 3), (16, 1), (32, 8), (40, 1), (33, 11)])
def test_heads(H, K):
    Problem(BF, 64, H, K, 16, [(100, 3), (33, 3)], MIXED, seed=H).check()


@pytest.mark.parametrize("block", [1, 2, 8, 16, 32, 64, 128, 1024])
def test_block_sizes(block):
    for dtype, D in ((BF, 128), (HF, 64)):
        Problem(dtype, D, 4, 2, block, [(150, 6)], MIXED, seed=block).check()
        Problem(dtype, D, 16, 2, block, [(300, 6)], [(100, 9), (20, 20), (65, 7), (1, 1), (300, 2), (64, 5)], seed=block).check()


@pytest.mark.parametrize("n", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000])
def test_lengths(n):
    """Histories and own tokens that end at, in front of and behind the steps of the kernels."""
    for new in (1, 9):
        own = max(n, new)
        Problem(BF, 64, 4, 4, 16, [(n, 2)], [(own, new), (new, new)], seed=n).check()
        Problem(BF, 128, 16, 2, 16, [(n, 2)], [(own, new), (new, new)], seed=n + 1).check()
        Problem(HF, 64, 4, 1, 64, [], [(own, new), (new, 1)], seed=n + 2).check()


@pytest.mark.parametrize("rows", [1, 4, 31, 32, 33, 64, 127, 128, 129, 300])
def test_rows(rows):
    Problem(BF, 64, 2, 2, 16, [(270, rows)], [(3, 1)] * rows, seed=rows).check()
    Problem(BF, 64, 2, 1, 16, [(90, 1)], [(rows + 5, rows)], seed=rows).check()


@pytest.mark.parametrize("layout", ["heads first", "keys beside values"])
def test_layouts_and_strides(layout):
    Problem(BF, 96, 6, 3, 16, [(140, 6)], MIXED, layout=layout).check(strided=True)
    Problem(HF, 128, 12, 3, 32, [(140, 6)], [(60, 9)] * 6, layout=layout).check(strided=True)


def test_long_prompts_without_a_history():
    Problem(BF, 128, 4, 1, 16, [], [(513, 513), (700, 300), (40, 40)]).check()
    Problem(HF, 64, 2, 2, 64, [], [(1, 1), (1500, 257)]).check()


def test_long_stretches_are_cut_and_joined():
    Problem(BF, 64, 4, 2, 16, [(9001, 2)], [(5, 1), (1, 1)]).check()
    Problem(BF, 64, 4, 2, 16, [], [(9001, 1), (7777, 2)]).check()
    Problem(HF, 128, 8, 1, 64, [(6000, 3)], [(2500, 8), (3000, 2), (64, 1)]).check()


def test_many_groups():
    groups = [(n, 1 + i % 4) for i, n in enumerate((0, 3, 500, 64, 65, 1, 200, 31, 90, 100, 7))]
    n = sum(g[1] for g in groups)
    Problem(BF, 64, 8, 2, 16, groups, [(1 + i * 7 % 50, 1 + i % 2) for i in range(n)]).check()
    Problem(BF, 64, 8, 2, 16, groups, [(60 + i * 7 % 50, 1 + i * 5 % 40) for i in range(n)]).check()


@pytest.mark.parametrize("new", [1, 30])
def test_rows_that_attend_to_nothing(new):
    """No history and no own tokens; new tokens that are not all in the length; requests without new tokens; requests of no group; tokens of no request."""
    p = Problem(BF, 64, 4, 2, 16, [(0, 2), (40, 2)], [(0, 0), (new, new), (50, 0), (new, new), (4 + new, new), (7 + new, new)], tail=3)
    p.check()
    p = Problem(BF, 64, 4, 2, 16, [(0, 1), (40, 1)], [(new, new), (new, new), (new, new)], tail=2)
    p.lens = torch.tensor([0, new // 2, 0], dtype=torch.int32)
    p.check()
    p.group_offsets = torch.tensor([1, 1, 2], dtype=torch.int32)
    p.check()
    p.check(bounds=False)
    p.check(lse=False)
    p = Problem(BF, 64, 4, 2, 16, [], [(0, 0), (0, 0)], tail=3)
    p.check()


def test_what_is_hidden_has_no_part():
    """Keys and values behind a query's own place that are infinite or no numbers (the pool's unused places are NaN in every test)."""
    for H, K in ((4, 4), (16, 2)):                     # few rows, many rows
        for odd in (math.inf, -math.inf, math.nan):
            p = Problem(BF, 64, H, K, 16, [(50, 1)], [(40, 20)], seed=5)
            for i, d in ((39, 3), (38, 60), (35, 17), (22, 17)):
                b = int(p.block_table[0, i // 16])
                p.v[b, i % 16, 0, d] = odd
            p.v[int(p.block_table[0, 1]), 14, K - 1, 5] = -odd       # token 30: two kinds in one column make NaN where both are seen
            p.check()
            p.k[int(p.block_table[0, 2]), 4] = math.nan              # token 36
            out, lse = p.run()
            want, want_lse, bound, lse_bound = p.want()
            assert torch.isfinite(out[:2]).all() and torch.isnan(out[16:]).all() and torch.isnan(lse[16:]).all()
            R.close(out[:16], want[:16], bound[:16])


def test_extreme_scores():
    """Scores that grow along the keys, fall, and are far apart: the running reference and what is joined."""
    for H, K, new in ((2, 2, 1), (8, 1, 8)):
        for sign in (1, -1):
            p = Problem(BF, 64, H, K, 16, [(700, 1)], [(new + 40, new)], seed=2, scale=1.0)
            p.q[:] = 1
            for t, n in ((p.prefix_table[0], 700), (p.block_table[0], new + 40)):
                for i in range(n):
                    p.k[int(t[i // 16]), i % 16] = sign * (i - 300) / 64
            p.check()
    p = Problem(BF, 64, 4, 2, 16, [(100, 2)], [(5, 1), (9, 2)])
    for t, n in ((p.prefix_table[0], 100), (p.block_table[0], 5), (p.block_table[1], 9)):
        for i in range(n):
            p.k[int(t[i // 16]), i % 16] = -torch.finfo(BF).max
    p.q[:] = 1                                         # every score is minus infinity: as if there were nothing
    out, lse = p.run()
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("H,K,new", [(2, 2, 1), (16, 1, 9)])
def test_large_values_behind_growing_scores(H, K, new):
    """The sums are formed against a reference that may lie behind the largest score: they have room for values of 2^80."""
    p = Problem(BF, 64, H, K, 16, [(3000, 1)], [(new + 40, new)], seed=4, scale=1.0)
    p.q[:] = 1
    for i in range(3000):                              # 0.05 a key: the weights pass every line at which the reference moves
        p.k[int(p.prefix_table[0, i // 16]), i % 16] = i / 1280
    p.v *= 2.0 ** 80
    p.check()
    p.v *= 2.0 ** -160                                 # and small ones are not lost
    p.check()


@pytest.mark.parametrize("H,K,new", [(2, 2, 1), (4, 4, 20), (16, 1, 20)])
def test_odd_queries_spoil_their_own_rows_only(H, K, new):
    """Queries that are no numbers, or infinite: every score of theirs is NaN or infinite, their neighbours' are as ever."""
    for odd in (math.nan, math.inf):
        p = Problem(BF, 64, H, K, 16, [(700, 2)], [(new + 40, new), (new, new)], seed=6)
        p.q[0, 1], p.q[new, 0, 7] = odd, odd
        if new > 1:
            p.q[new - 1, H - 1, 63] = odd
        for offsets in ([0, 2], [0, 0]):               # with and without the history
            p.group_offsets = torch.tensor(offsets, dtype=torch.int32)
            out, lse = p.run()
            want, want_lse, bound, lse_bound = p.want()
            # where all scores are minus infinity the result is just 0, and its bound, of infinite scores, no number
            R.close(out, want, torch.where(torch.isnan(bound), 0.0, bound))
            R.close(lse, want_lse, torch.where(torch.isnan(lse_bound), 0.0, lse_bound))


def test_histories_behind_four_gibibytes():
    """Blocks whose keys and values are more than 2^32 bytes from the first one."""
    K, D, block = 8, 128, 64
    n_blocks = (5 << 30) // (K * D * 2 * block)
    p = Problem(BF, D, 16, K, block, [(500, 2)], [(5, 1), (70, 2)], spare=0)
    pool = torch.zeros(2, n_blocks, block, K, D, dtype=BF, device="cuda")
    shift = n_blocks - p.n_blocks
    pool[0, shift:], pool[1, shift:] = p.k.cuda(), p.v.cuda()
    out, s = torch.empty(3, 16, D, dtype=BF, device="cuda"), B.hps_seq_attention_create(48, D)
    up = lambda t: torch.where(t < 0, t, t + shift).cuda()  # noqa: E731
    B.hps_seq_attention(s, p.q.cuda(), pool[0], pool[1], up(p.block_table), p.lens.cuda(), p.offsets.cuda(), out, prefix_table=up(p.prefix_table),
                        prefix_lens=p.prefix_lens.cuda(), group_offsets=p.group_offsets.cuda(), **p.bounds)
    torch.cuda.synchronize()
    assert B.hps_seq_attention_flags(s) == 0
    B.hps_seq_attention_destroy(s)
    want, _, bound, _ = p.want()
    R.close(out.cpu(), want, bound)


def test_flags():
    p = Problem(BF, 64, 4, 2, 16, [(100, 2)], [(5, 1), (40, 2)], loose=1)
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
        p = Problem(BF, 64, 4, 2, 16, [(100, 2)], [(5, 1), (40, 2)])
        p.prefix_table[0, 3], p.block_table[1, 1] = junk, junk
        out, lse = p.run()
        assert p.flags == B.HPS_SEQ_FLAG_BLOCK
        want, want_lse, bound, lse_bound = p.want()
        R.close(out, want, bound)
        R.close(lse, want_lse, lse_bound)


def test_refusals():
    p = Problem(BF, 64, 4, 2, 16, [(100, 2)], [(5, 1), (40, 2)])
    s = B.hps_seq_attention_create(12, 64)
    k, v = p.pages()
    args = [p.q.cuda(), k, v, p.block_table.cuda(), p.lens.cuda(), p.offsets.cuda(), torch.empty(3, 4, 64, dtype=BF, device="cuda")]
    kw = dict(prefix_table=p.prefix_table.cuda(), prefix_lens=p.prefix_lens.cuda(), group_offsets=p.group_offsets.cuda())

    def refuse(error, at=None, value=None, **more):
        a = list(args)
        if at is not None:
            a[at] = value
        with pytest.raises(error):
            B.hps_seq_attention(s, *a, **{**kw, **more})

    refuse(TypeError, 0, args[0].cpu())
    refuse(TypeError, 0, args[0].half())
    refuse(ValueError, 0, args[0][:, :, :32])
    refuse(ValueError, 0, args[0].transpose(1, 2))
    refuse(TypeError, 1, k.half())
    refuse(ValueError, 1, k.transpose(1, 2))
    refuse(ValueError, 3, args[3][0])
    refuse(TypeError, 4, args[4].long())
    refuse(ValueError, 5, args[5][:2])
    refuse(ValueError, 6, args[6][:2])
    refuse(ValueError, prefix_table=None)
    refuse(ValueError, group_offsets=kw["group_offsets"][:1])
    refuse(ValueError, lse=torch.empty(3, 3, device="cuda"))
    refuse(TypeError, lse=torch.empty(3, 4, device="cuda", dtype=BF))
    for scale in (0.0, -1.0, math.inf, math.nan):
        refuse(B.HpsError, scale=scale)
    refuse(B.HpsError, max_len=1 << 30)
    odd = torch.empty(3 * 4 * 64 + 1, dtype=BF, device="cuda")[1:].view(3, 4, 64)
    refuse(B.HpsError, 0, odd)                         # rows that do not start on 16 bytes
    refuse(B.HpsError, 6, odd)
    with pytest.raises(B.HpsError, match="max_rows"):
        B.hps_seq_attention(s, torch.zeros(4, 4, 64, dtype=BF, device="cuda"), *args[1:6], torch.zeros(4, 4, 64, dtype=BF, device="cuda"), **kw)
    wide = torch.zeros(1, 1, 128, dtype=BF, device="cuda")
    with pytest.raises(B.HpsError, match="max_head_dim"):
        B.hps_seq_attention(s, wide, wide[None], wide[None], args[3], args[4], args[5], wide)
    x = torch.zeros(3, 3, 64, dtype=BF, device="cuda")
    with pytest.raises(B.HpsError, match="multiple of kv_heads"):
        B.hps_seq_attention(s, x, k, v, *args[3:6], x.clone(), **kw)
    f = torch.zeros(1, 1, 64, device="cuda")
    with pytest.raises(B.HpsError, match="dtype"):
        B.hps_seq_attention(s, f, f[None], f[None], args[3], args[4], args[5], f)
    n, none = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, 4, 64, dtype=BF, device="cuda")
    B.hps_seq_attention(s, none, k, v, n.view(0, 1), n, torch.zeros(1, dtype=torch.int32, device="cuda"), none)       # nothing to do
    torch.cuda.synchronize()
    assert B.hps_seq_attention_flags(s) == 0
    B.hps_seq_attention_destroy(s)


def test_one_session_on_another_stream_and_after_other_sizes():
    """What a session's scratch memory holds from one call has no part in the next."""
    s, st = B.hps_seq_attention_create(4096, 128), torch.cuda.Stream()
    for seed, (groups, requests) in enumerate([([(3000, 3)], [(9, 1)] * 3), ([(5, 2)], [(900, 2), (3, 1)]), ([], [(40, 40)]), ([(64, 40)], [(2, 2)] * 40), ([(0, 1), (7, 1)], [(1, 1)] * 3)]):
        for D in (64, 128):
            Problem(BF, D, 4, 2, 16, groups, requests, seed=seed).check(session=s, stream=st)
    B.hps_seq_attention_destroy(s)


def test_graph_replays_on_new_lengths():
    p = Problem(BF, 64, 8, 2, 16, [(300, 3), (70, 2)], [(40, 2), (20, 1), (33, 4), (16, 1), (50, 2)])
    k, v = p.pages()
    T = p.q.shape[0]
    s, out, lse = B.hps_seq_attention_create(T * 8, 64), torch.zeros(T, 8, 64, dtype=BF, device="cuda"), torch.zeros(T, 8, device="cuda")
    q, lens, prefix, table, offsets, ptable, groups = (x.cuda() for x in (p.q, p.lens, p.prefix_lens, p.block_table, p.offsets, p.prefix_table, p.group_offsets))

    def call():
        B.hps_seq_attention(s, q, k, v, table, lens, offsets, out, prefix_table=ptable, prefix_lens=prefix, group_offsets=groups, lse=lse, **p.bounds)

    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        call()
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


@pytest.mark.parametrize("new", [1, 30])
@pytest.mark.parametrize("prefix", [0, 90, 5000])
def test_rows_in_front_of_the_first_request_are_left_alone(new, prefix):
    """A batch in two calls over the same queries and outputs: the second one's offsets begin where the first one's end.  In between the
    session serves another one."""
    p = Problem(BF, 64, 4, 2, 16, [(prefix, 2), (prefix // 2, 3)], [(new, new), (40 + new, 1), (new, new), (70, 2), (3, 1)], tail=2, seed=new)
    k, v = p.pages()
    T, first = p.q.shape[0], 2
    q, table, lens, offsets, ptable, plens = (x.cuda() for x in (p.q, p.block_table, p.lens, p.offsets, p.prefix_table, p.prefix_lens))
    out, lse = torch.full((T, 4, 64), 9.0, dtype=BF, device="cuda"), torch.full((T, 4), 9.0, device="cuda")
    s = B.hps_seq_attention_create(T * 4, 64)
    for r, g, n in ((slice(0, first), slice(0, 1), 2), (slice(first, None), slice(1, None), 3)):
        B.hps_seq_attention(s, q, k, v, table[r], lens[r], offsets[r.start:][:n + 1], out, prefix_table=ptable[g], prefix_lens=plens[g],
                            group_offsets=torch.tensor([0, n], dtype=torch.int32, device="cuda"), lse=lse, **p.bounds)
        B.hps_seq_attention(s, -2 * q, k, v, table, lens, offsets, torch.empty_like(q), prefix_table=ptable, prefix_lens=plens, group_offsets=p.group_offsets.cuda(), **p.bounds)
    torch.cuda.synchronize()
    assert B.hps_seq_attention_flags(s) == 0
    B.hps_seq_attention_destroy(s)
    want, want_lse, bound, lse_bound = p.want()
    n = int(p.offsets[-1])
    R.close(out[:n].cpu(), want[:n], bound[:n])
    R.close(lse[:n].cpu(), want_lse[:n], lse_bound[:n])
    assert (out[n:] == 9).all() and (lse[n:] == 9).all()


@pytest.mark.parametrize("new", [1, 20])
def test_tokens_behind_the_last_query(new):
    """Offsets may count more tokens than there are queries for: the others' places in their requests stay what they are."""
    p = Problem(BF, 64, 4, 2, 16, [(40, 2)], [(new, new), (50 + new, 2 * new)], seed=new)
    want, want_lse, bound, lse_bound = p.want()
    T = new + max(1, new // 2)
    p.q = p.q[:T]
    out, lse = p.run()
    assert p.flags == 0
    R.close(out, want[:T], bound[:T])
    R.close(lse, want_lse[:T], lse_bound[:T])


@pytest.mark.parametrize("H,K,requests", [(4, 2, [(5, 1), (40, 2)]), (16, 1, [(60, 9), (9, 9)]), (2, 2, [(33, 1)] * 300), (2, 2, [(700, 1), (2000, 2)])])
def test_scores_of_minus_infinity_and_infinite_values(H, K, requests):
    """Rows whose scores are all minus infinity get 0, whatever the values and however the keys are cut."""
    for groups in ([], [(100, len(requests))]):
        p = Problem(BF, 64, H, K, 16, groups, requests)
        p.q[:] = 1
        for t, n in [(p.block_table[r], int(n)) for r, n in enumerate(p.lens)] + [(p.prefix_table[g], int(n)) for g, n in enumerate(p.prefix_lens)]:
            place = torch.arange(n)
            p.k[t.long()[place // 16], place % 16] = -torch.finfo(BF).max
            p.v[t.long()[place // 16], place % 16] = math.inf
        out, lse = p.run()
        assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("H,K,new", [(1, 1, 1), (16, 1, 3)])
@pytest.mark.parametrize("shared", [True, False])
def test_small_weights_beside_large_ones(H, K, new, shared, dtype):
    """A key of weight 1 and 31 of weight 2^-26, over and over: small weights are not lost where they are rounded for the product."""
    n = 15000
    p = Problem(dtype, 64, H, K, 16, [(n, 1)] if shared else [], [(new if shared else n + new, new)], seed=8, scale=1.0)
    p.q[:], p.k[:], p.v[:] = 1, -18 / 64, p.v.nan_to_num().abs() * 1024
    first = p.prefix_table[0, :n // 16:2] if shared else p.block_table[0, :n // 16:2]
    p.k[first.long(), 0], p.v[first.long(), 0] = 0, 0
    out, lse = p.run()
    want, want_lse, _, lse_bound = p.want()
    # every weight is rounded relative to itself, and f16's to steps of 2^-32 of the largest (2^-24 where that is 2^8 at least); the result to its
    # type; scores and sums as ever
    e = 18 * 72 * 2.0 ** -24 + 2.0 ** -21
    steps = (n + new) * 2.0 ** -33 * float(p.v.abs().max()) / len(first) if dtype is HF else 0
    bound = 2.02 * R.ROUND[dtype] * want + want * (2 * e + (n + 64) * 2.0 ** -24) + steps + R.TINY[dtype]
    assert 4 * float(bound.max()) < float(want.min())
    R.close(out, want, bound)
    R.close(lse, want_lse, lse_bound)


def test_lengths_are_checked_where_no_history_is_attended():
    """A bound of 0 leaves the histories out of the launch, and tells where there are any all the same."""
    p = Problem(BF, 64, 4, 2, 16, [(100, 2), (3, 1)], [(5, 1), (40, 2), (1, 1)])
    good = dict(max_new=2, max_len=40, max_prefix=100, max_group=3)
    for bad in (dict(max_prefix=0), dict(max_group=0), dict(max_prefix=0, max_group=0)):
        p.bounds = {**good, **bad}
        p.run()
        assert p.flags == B.HPS_SEQ_FLAG_LENGTH, bad
    p.group_offsets = torch.tensor([0, 0, 0], dtype=torch.int32)             # histories of nobody: no new tokens to a group
    p.bounds = {**good, "max_group": 0}
    p.check()
    p = Problem(BF, 64, 4, 2, 16, [(0, 2), (0, 1)], [(5, 1), (40, 2), (1, 1)], loose=1)
    p.check()                                          # histories of no tokens, bounded by 0: nothing to tell
    groups = 1500                                      # more groups than work-groups
    p = Problem(BF, 64, 1, 1, 16, [(0, 0)] * groups + [(0, 1)], [(5, 1)], loose=1)
    p.check()
    p.prefix_lens[groups] = 1
    p.run()
    assert p.flags == B.HPS_SEQ_FLAG_LENGTH


def test_more_work_groups_than_one_launch_takes():
    """Many requests of a token each with the bounds that the shapes give: 2^24 tiles, as many as a launch has no room for."""
    n, H, K, D, L, block = 8192, 32, 8, 64, 3, 4
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g).to(BF)  # noqa: E731
    q, k, v = normal(n, H, D), normal(n, block, K, D), normal(n, block, K, D)
    table = torch.randperm(n, device="cuda", generator=g).int().view(n, 1)
    lens, offsets = torch.full((n,), L, dtype=torch.int32, device="cuda"), torch.arange(n + 1, dtype=torch.int32, device="cuda")
    out, s = torch.full_like(q, 9), B.hps_seq_attention_create(n * H, D)
    B.hps_seq_attention(s, q, k, v, table, lens, offsets, out)
    torch.cuda.synchronize()
    assert B.hps_seq_attention_flags(s) == 0
    B.hps_seq_attention_destroy(s)
    kk, vv = (x[table[:, 0].long(), :L].double().permute(0, 2, 1, 3)[:, :, None] for x in (k, v))          # [n, K, 1, L, D]
    qq = q.double().view(n, K, H // K, 1, D)
    p = ((qq * kk).sum(-1) * D ** -0.5).softmax(-1)[..., None]
    want, mass = ((p * x).sum(-2).view(n, H, D) for x in (vv, vv.abs()))
    # scores of 64 products of values up to 6 in 32 bits, weights and results rounded to the type
    e = 64 * 36 * D ** -0.5 * (D + 8) * 2.0 ** -24 + 2.0 ** -21
    R.close(out.cpu(), want.cpu(), (R.ROUND[BF] * 1.01 * (want.abs() + mass) + mass * (2 * e + (L + 64) * 2.0 ** -24) + 1e-30).cpu())


def test_more_rows_than_one_join_takes():
    """2^29 rows, of which one request has 65,536: the others are left alone."""
    T, H, D, block = 8193, 65536, 8, 2
    torch.cuda.empty_cache()
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn(3, block, H, D, device="cuda", generator=g).half() for _ in range(2))
    q, out = torch.empty(T, H, D, dtype=HF, device="cuda"), torch.empty(T, H, D, dtype=HF, device="cuda").fill_(9)
    q[:1] = torch.randn(1, H, D, device="cuda", generator=g)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    s = B.hps_seq_attention_create(T * H, D)
    B.hps_seq_attention(s, q, k, v, i32(0).view(1, 1), i32(1), i32(0, 1), out, prefix_table=i32(2, 1).view(1, 2), prefix_lens=i32(3), group_offsets=i32(0, 1), max_new=1, max_group=1)
    torch.cuda.synchronize()
    assert B.hps_seq_attention_flags(s) == 0
    B.hps_seq_attention_destroy(s)
    assert all(bool((x == 9).all()) for x in out[1:].split(512))
    kk, vv = (torch.stack((x[2, 0], x[2, 1], x[1, 0], x[0, 0]), 1).double() for x in (k, v))        # [H, 4, D]
    p = ((q[0].double()[:, None] * kk).sum(-1) * D ** -0.5).softmax(-1)[..., None]
    want, mass = (p * vv).sum(1), (p * vv.abs()).sum(1)
    e = 8 * 36 * D ** -0.5 * (D + 8) * 2.0 ** -24 + 2.0 ** -21
    R.close(out[0].cpu(), want.cpu(), (R.ROUND[HF] * 1.01 * (want.abs() + mass) + mass * (2 * e + 68 * 2.0 ** -24) + 4 * R.TINY[HF] * vv.abs().amax(1) + R.TINY[HF]).cpu())


def test_many_parts_of_many_rows():
    """Over 512 parts, of more rows than a work-group each: what the join keeps of them in LDS."""
    T, D, block, n = 8200, 8, 1024, 1 << 20
    p = Problem(HF, D, 1, 1, block, [(n, 1)], [(n, 1)], tail=T - 1)
    p.bounds["max_group"] = 1
    s = B.hps_seq_attention_create(2_000_000, D)       # a session for larger calls: room for parts
    p.check(session=s)
    B.hps_seq_attention_destroy(s)
