"""Block tables and slots, rotary positions and the writing of pages (hps_seq.h) against their definitions."""
import math

import numpy as np
import pytest
import torch

import seq_reference as R
from paper_2210_08804_amd import binding as B

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def i32(*shape, fill=-77):
    return torch.full(shape, fill, dtype=torch.int32, device="cuda")


# ---- extend and release

def run_extend(past, new, block, free, n_free, table, max_tokens, start=None):
    n = len(past)
    t = dev(table)
    out = i32(n + 1), i32(n), i32(max_tokens), i32(max_tokens), i32(4)
    B.hps_seq_extend(dev(past), dev(new), block, dev(free), dev(np.asarray([n_free], dtype=np.int32)), t, *out, start=None if start is None else dev(start))
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (t, *out)]


def check_extend(past, new, block, n_blocks, n_free, width, max_tokens, start=None, seed=0, free=None):
    rng = np.random.RandomState(seed)
    past, new = np.asarray(past, dtype=np.int32), np.asarray(new, dtype=np.int32)
    if free is None:
        free = rng.permutation(n_blocks).astype(np.int32)
    table = rng.randint(0, max(n_blocks, 1), (len(past), width)).astype(np.int32)
    want = R.extend(past, new, start, free, n_free, n_blocks, block, table, max_tokens)
    got = run_extend(past, new, block, free, n_free, table, max_tokens, start)
    for name, g, w in zip(("table", "token_offsets", "total_lens", "slots", "positions", "info"), got, want):
        assert np.array_equal(g, w), f"{name}: {g[g != w][:5]} where {w[g != w][:5]}"


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 1000, 4095, 4096, 4097, 9001])
@pytest.mark.parametrize("block", [1, 16, 64])
def test_extend(n, block):
    rng = np.random.RandomState(n + block)
    past, new = rng.randint(0, 150, n), rng.randint(0, 40, n) * (rng.rand(n) < 0.6)
    start = rng.randint(0, 1000, n).astype(np.int32)
    width = -(-200 // block)
    need = int((-(-(past + new) // block) - -(-past // block)).sum())
    check_extend(past, new, block, need + 10, need + 7, width, int(new.sum()) + 5, start, seed=n)


def test_extend_long_requests():
    """One request's blocks and tokens by many work-groups; odd numbers of tokens, runs of requests without any."""
    check_extend([0, 5, 17, 0], [70001, 0, 33333, 1], 16, 8000, 7999, 5000, 110000)
    new = np.zeros(5000, dtype=np.int32)
    new[[0, 1, 4094, 4096, 4999]] = [3, 20001, 7, 9, 4099]
    check_extend(np.full(5000, 3), new, 32, 6000, 6000, 1000, 24130)


def test_extend_corners():
    check_extend([], [], 16, 4, 4, 3, 9)                                    # no request
    check_extend([3, 0], [0, 0], 16, 4, 4, 3, 0)                            # no token
    check_extend([16, 15, 17], [1, 1, 1], 16, 9, 9, 4, 3)                   # at the ends of blocks
    check_extend([-5, 4], [7, -3], 4, 9, 9, 4, 9)                           # negative lengths count as 0
    check_extend([0, 0, 9], [20, 20, 3], 4, 12, 7, 8, 50)                   # the free list ends inside a request
    check_extend([0, 3, 100], [50, 2, 5], 4, 40, 40, 5, 60)                 # more than tables hold
    check_extend([1, 2, 3], [10, 10, 10], 8, 10, 10, 4, 17)                 # more tokens than slots
    check_extend([1, 2], [5, 5], 2, 10, 99, 8, 17)                          # a length of the free list that is none
    check_extend([1, 2], [5, 5], 2, 10, -3, 8, 17)
    check_extend([1, 2], [5, 5], 2, 10, 10, 8, 17, free=np.full(10, 77, dtype=np.int32))      # a free list of no blocks
    check_extend([0] * 3, [2 ** 31 - 1] * 3, 1024, 4, 4, 2, 100)            # sums that end at 2^31 - 1
    check_extend([0] * 5000, [2 ** 31 - 1] * 5000, 1024, 4, 4, 2, 100)


def test_extend_after_extend_and_release():
    """Steps of a server: lengths, free list and tables handed from call to call."""
    rng = np.random.RandomState(3)
    n, block, n_blocks, width = 300, 16, 3000, 20
    free, table = rng.permutation(n_blocks).astype(np.int32), np.full((n, width), -1, dtype=np.int32)
    lens, n_free = np.zeros(n, dtype=np.int32), n_blocks
    d_free, d_table, d_lens, other, info, before = dev(free), dev(table), dev(lens), i32(n), i32(4), dev(np.asarray([n_free, 0, 0, 0], dtype=np.int32))
    for step in range(6):
        new = rng.randint(0, 30, n).astype(np.int32)
        new = np.minimum(new, width * block - lens)
        most = int(new.sum())
        slots, positions, offsets = i32(most), i32(most), i32(n + 1)
        B.hps_seq_extend(d_lens, dev(new), block, d_free, before, d_table, offsets, other, slots, positions, info)
        want = R.extend(lens, new, None, free, n_free, n_blocks, block, table, most)
        d_lens, other, before, info = other, d_lens, info, before
        table, lens, n_free = want[0], want[2], int(want[5][0])
        assert np.array_equal(slots.cpu().numpy(), want[3]) and np.array_equal(before.cpu().numpy(), want[5])
        held = table[table >= 0]
        assert len(np.unique(held)) == len(held) == n_blocks - n_free       # no block in two places
        done = (rng.rand(n) < 0.3).astype(np.int32)
        B.hps_seq_release(d_lens, dev(done), block, d_table, d_free, before, before)
        lens, table, free, counts = R.release(lens, done, block, table, free, n_free, n_blocks)
        n_free = int(counts[0])
        assert np.array_equal(before.cpu().numpy()[:3], counts)
        for g, w in ((d_lens, lens), (d_table, table), (d_free[:n_free], free[:n_free])):
            assert np.array_equal(g.cpu().numpy(), w)


@pytest.mark.parametrize("n", [0, 1, 4096, 4500])
def test_release(n):
    rng = np.random.RandomState(n)
    block, n_blocks, width = 8, 9000, 3
    table = rng.randint(-2, n_blocks + 2, (n, width)).astype(np.int32)      # some are no blocks, some are given back twice
    lens, done = rng.randint(-3, 40, n).astype(np.int32), (rng.rand(n) < 0.8).astype(np.int32)
    free = np.arange(n_blocks, dtype=np.int32)
    d = [dev(x) for x in (lens, table, free)]
    info, n_free = i32(4), dev(np.asarray([100], dtype=np.int32))
    B.hps_seq_release(d[0], dev(done), block, d[1], d[2], n_free, info)
    want = R.release(lens, done, block, table, free, 100, n_blocks)
    for g, w in zip((*d, info[:3]), want):
        assert np.array_equal(g.cpu().numpy(), w)


# ---- rotary positions

@pytest.mark.parametrize("rot,kw", [(64, {}), (128, dict(scale=1, factor=4.0)), (96, dict(scale=2, factor=8.0, original=512, low=1.0, high=32.0, base=500000.0)), (2, {})])
def test_rope_table(rot, kw):
    for n in (1, 1000, 70001):
        table = torch.empty(n, rot // 2, 2, device="cuda")
        B.hps_seq_rope_table(table, magnitude=1.25, **kw)
        a = np.arange(n)[:, None] * R.angles(rot, **kw)
        want = 1.25 * np.stack((np.cos(a), np.sin(a)), -1)
        # one rounding to 32 bits; angles of up to 7e4 in 64 bits (2^-52 relative, and as much again for the power)
        assert np.abs(table.cpu().numpy() - want).max() <= 1.25 * 2.0 ** -24 + 4 * 7e4 * 2.0 ** -50


def cos_sin(n, rot):
    a = torch.arange(n, dtype=torch.float64)[:, None] * torch.from_numpy(R.angles(rot))
    return torch.stack((a.cos(), a.sin()), -1).float()


ROPE_SHAPES = [                                        # tokens, q heads, k heads, dim, rot
    (1, 1, 1, 64, 64), (3, 8, 2, 128, 128), (7, 32, 8, 128, 64), (5, 12, 12, 96, 96), (5, 12, 3, 96, 48), (4, 3, 1, 80, 80), (9, 5, 5, 64, 24),
    (3, 2, 1, 10, 6), (3, 2, 2, 7, 4), (2, 1, 1, 2, 2), (2, 3, 3, 512, 512), (300, 16, 0, 64, 64), (2, 300, 7, 256, 128), (3, 4, 4, 72, 8), (5, 2, 2, 40, 16),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", ROPE_SHAPES)
def test_rope_and_its_gradient(shape, interleaved, dtype):
    T, H, K, D, rot = shape
    g = torch.Generator().manual_seed(T * 1000 + D + rot)
    x = torch.randn(T, H + K, D, generator=g).to(dtype)
    positions = torch.randint(0, 500, (T,), generator=g).int()
    table = cos_sin(500, rot)
    for inverse in (False, True):
        want, _ = R.rope(x, positions, table, interleaved, inverse)
        dx = x.cuda()
        q, k = dx[:, :H], dx[:, H:]                    # strided: the heads of one projection
        q_out, k_out = torch.empty(T, H, D, dtype=dtype, device="cuda"), torch.empty(T, K, D, dtype=dtype, device="cuda")
        B.hps_seq_rope(q, q_out, positions.cuda(), table.cuda(), k=k if K else None, k_out=k_out if K else None, interleaved=interleaved, inverse=inverse)
        got = torch.cat((q_out, k_out), 1).cpu()
        R.close(got, want, R.rope_bound(x, want, dtype))
        # in place, and from odd addresses: the same bits
        B.hps_seq_rope(q, q, positions.cuda(), table.cuda(), k=k if K else None, k_out=k if K else None, interleaved=interleaved, inverse=inverse)
        assert torch.equal(dx.cpu(), got)
        buf = torch.empty(T * (H + K) * D + 1, dtype=dtype, device="cuda")
        odd = buf[1:].view(T, H + K, D)
        odd.copy_(x)
        B.hps_seq_rope(odd, odd, positions.cuda(), table.cuda(), interleaved=interleaved, inverse=inverse)
        assert torch.equal(odd.cpu(), got)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_gradient_against_differences(interleaved):
    """d/dx of sum(w * rope(x)) by central differences of the operator itself, which is linear: exact but for rounding."""
    g = torch.Generator().manual_seed(4)
    T, H, D, rot = 2, 2, 16, 12
    x, w = torch.randn(T, H, D, generator=g).cuda(), torch.randn(T, H, D, generator=g).cuda()
    positions, table = torch.tensor([3, 77], dtype=torch.int32, device="cuda"), cos_sin(100, rot).cuda()
    grad = torch.empty_like(w)
    B.hps_seq_rope(w, grad, positions, table, interleaved=interleaved, inverse=True)
    y = torch.empty_like(x)
    for i in range(x.numel()):
        sums = []
        for step in (1.0, -1.0):
            z = x.clone()
            z.view(-1)[i] += step
            B.hps_seq_rope(z, y, positions, table, interleaved=interleaved)
            sums.append((y.double() * w.double()).sum().item())
        # values of up to 5, rounded to 2^-24 of that, in two sums of 3 terms that differ, weighed by up to 4
        assert abs((sums[0] - sums[1]) / 2 - grad.view(-1)[i].item()) < 1e-5


def test_rope_positions_outside_the_table():
    x = torch.ones(4, 2, 32, device="cuda")
    out = torch.full((4, 2, 32), 7.0, device="cuda")
    B.hps_seq_rope(x, out, torch.tensor([-1, 9, 10, 2 ** 31 - 1], dtype=torch.int32, device="cuda"), cos_sin(10, 16).cuda())
    assert (out[0] == 7).all() and torch.isfinite(out[1]).all()
    assert torch.isnan(out[2:, :, :16]).all() and (out[2:, :, 16:] == 1).all()


def layouts(n_blocks, block, heads, dim, dtype, fill):
    """Pages as [blocks, places, heads, dim] in several orders of memory."""
    new = lambda *s: torch.full(s, fill, dtype=dtype, device="cuda")  # noqa: E731
    k, v = new(n_blocks, block, heads, dim), new(n_blocks, block, heads, dim)
    yield "places first", k, v
    k, v = new(n_blocks, heads, block, dim), new(n_blocks, heads, block, dim)
    yield "heads first", k.transpose(1, 2), v.transpose(1, 2)
    both = new(n_blocks, 2, block, heads, dim)
    yield "keys beside values", both[:, 0], both[:, 1]
    wide = new(2, n_blocks, block, heads, dim + 8)
    yield "padded", wide[0][..., :dim], wide[1][..., :dim]


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,H,K,D,rot,block", [(1, 4, 4, 64, 64, 16), (37, 8, 2, 128, 64, 32), (100, 0, 3, 96, 96, 1), (65, 5, 5, 20, 10, 64)])
def test_append(T, H, K, D, rot, block, dtype):
    g = torch.Generator().manual_seed(T + D)
    n_blocks = -(-T // block) + 3
    row = torch.randn(T, H + 2 * K, D, generator=g).to(dtype)
    positions, table = torch.randint(0, 300, (T,), generator=g).int(), cos_sin(300, rot)
    slots = torch.randperm(n_blocks * block, generator=g)[:T].int()
    if T > 30:
        slots[3], slots[5], positions[7] = -1, n_blocks * block, -1
    for interleaved in (False, True):
        want, live = R.rope(row, positions, table, interleaved, False)
        for name, kp, vp in layouts(n_blocks, block, K, D, dtype, 3.0):
            d = row.cuda()
            q_out = torch.full((T, H, D), 5.0, dtype=dtype, device="cuda")
            B.hps_seq_append(d[:, H:H + K], d[:, H + K:], kp, vp, slots.cuda(), q=d[:, :H] if H else None, q_out=q_out if H else None, positions=positions.cuda(),
                             table=table.cuda(), interleaved=interleaved)
            bound = R.rope_bound(row, want, dtype)
            R.close(q_out.cpu()[live], want[:, :H][live], bound[:, :H][live])
            assert (q_out.cpu()[~live] == 5).all()
            stored = live & (slots >= 0) & (slots < n_blocks * block)
            k, v = kp.reshape(-1, K, D).cpu(), vp.reshape(-1, K, D).cpu()
            at = slots[stored].long()
            R.close(k[at], want[:, H:H + K][stored], bound[:, H:H + K][stored])
            assert torch.equal(v[at], row[:, H + K:][stored])
            rest = torch.ones(n_blocks * block, dtype=torch.bool)
            rest[at] = False
            assert (k[rest] == 3).all() and (v[rest] == 3).all(), name
    # without turning
    kp, vp = torch.zeros(n_blocks, block, K, D, dtype=dtype, device="cuda"), torch.zeros(n_blocks, block, K, D, dtype=dtype, device="cuda")
    d = row.cuda()
    B.hps_seq_append(d[:, H:H + K], d[:, H + K:], kp, vp, slots.cuda())
    ok = (slots >= 0) & (slots < n_blocks * block)
    assert torch.equal(kp.view(-1, K, D).cpu()[slots[ok].long()], row[:, H:H + K][ok]) and torch.equal(vp.view(-1, K, D).cpu()[slots[ok].long()], row[:, H + K:][ok])


def test_append_behind_four_gibibytes():
    """Slots whose places are more than 2^32 bytes from the first one."""
    K, D, block = 8, 128, 16
    n_blocks = (5 << 30) // (K * D * 2 * block)
    pages = torch.zeros(2, n_blocks, block, K, D, dtype=torch.bfloat16, device="cuda")
    k = torch.randn(2, K, D, device="cuda").bfloat16()
    slots = torch.tensor([n_blocks * block - 1, (9 << 29) // (K * D * 2)], dtype=torch.int32, device="cuda")
    B.hps_seq_append(k, -k, pages[0], pages[1], slots)
    for i, s in enumerate(slots.tolist()):
        assert torch.equal(pages[0].view(-1, K, D)[s], k[i]) and torch.equal(pages[1].view(-1, K, D)[s], -k[i])
    assert int(torch.count_nonzero(pages[0].view(-1, K * D).any(1))) == 2


def test_streams_and_no_tokens():
    x = torch.randn(0, 4, 64, device="cuda")
    B.hps_seq_rope(x, torch.empty_like(x), i32(0), cos_sin(8, 64).cuda())
    st = torch.cuda.Stream()
    x = torch.randn(64, 4, 64, device="cuda")
    out, positions, table = torch.empty_like(x), i32(64, fill=3), cos_sin(8, 64).cuda()
    torch.cuda.synchronize()
    B.hps_seq_rope(x, out, positions, table, stream=st)
    st.synchronize()
    want, _ = R.rope(x.cpu(), positions.cpu(), table.cpu(), False, False)
    R.close(out.cpu(), want, R.rope_bound(x.cpu(), want, torch.float32))


def test_a_graph_of_a_step_is_replayed_on_new_lengths():
    """extend and append captured once; lengths change between the replays, eager work and synchronisation lie between."""
    n, block, n_blocks, width, K, D, most = 50, 16, 600, 12, 2, 64, 400
    free = torch.randperm(n_blocks).int().cuda()
    past, new, n_free = i32(n, fill=0), i32(n, fill=1), i32(1, fill=n_blocks)
    table, offsets, lens, slots, positions, info = i32(n, width, fill=-1), i32(n + 1), i32(n), i32(most), i32(most), i32(4)
    kv = torch.randn(most, 2 * K, D, device="cuda").half()
    kp, vp = torch.zeros(n_blocks, block, K, D, device="cuda").half(), torch.zeros(n_blocks, block, K, D, device="cuda").half()
    rope_table = cos_sin(256, 64).cuda()

    def step():
        B.hps_seq_extend(past, new, block, free, n_free, table, offsets, lens, slots, positions, info)
        B.hps_seq_append(kv[:, :K], kv[:, K:], kp, vp, slots, positions=positions, table=rope_table)

    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    rng = np.random.RandomState(1)
    for _ in range(4):
        p, a = rng.randint(0, 100, n).astype(np.int32), rng.randint(0, 9, n).astype(np.int32)
        past.copy_(torch.from_numpy(p)), new.copy_(torch.from_numpy(a)), table.fill_(5), kp.zero_(), vp.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = R.extend(p, a, None, free.cpu().numpy(), n_blocks, n_blocks, block, np.full((n, width), 5, dtype=np.int32), most)
        for g, w in zip((table, offsets, lens, slots, positions, info), want):
            assert np.array_equal(g.cpu().numpy(), w)
        # kept blocks are all block 5 here, so only fresh ones have slots of their own
        got = vp.view(-1, K, D).cpu()
        seen = {}
        for t, s in enumerate(want[3]):
            seen.setdefault(int(s), []).append(t)
        for s, ts in seen.items():
            if s >= 0 and len(ts) == 1:
                assert torch.equal(got[s], kv[ts[0], K:].cpu())


@pytest.mark.parametrize("pages", [False, True])
def test_more_tokens_than_one_launch_takes(pages):
    """2^24 tokens of 256 threads each: 2^32 threads.  All but a few tokens are passed over."""
    T, H, D = (1 << 24) + 5, 256 if not pages else 252, 2
    torch.cuda.empty_cache()
    at = torch.tensor([0, 77, (1 << 23) - 1, 1 << 23, (1 << 23) + 1, (1 << 24) - 1, 1 << 24, T - 1])
    g = torch.Generator().manual_seed(3)
    x, positions, table = torch.randn(len(at), H, D, generator=g).half(), torch.randint(0, 50, (len(at),), generator=g).int(), cos_sin(50, D)
    rows, every = torch.empty(T, H, D, dtype=torch.float16, device="cuda"), i32(T, fill=-1)
    rows[at.cuda()], every[at.cuda()] = x.cuda(), positions.cuda()
    want, _ = R.rope(x, positions, table, False, False)
    if pages:
        kv = torch.randn(T, 2, 1, D, device="cuda").half()
        kp, vp = torch.zeros(1, 16, 1, D, device="cuda").half(), torch.zeros(1, 16, 1, D, device="cuda").half()
        slots = i32(T, fill=-1)
        slots[at.cuda()] = torch.arange(len(at), dtype=torch.int32, device="cuda") + 3
        B.hps_seq_append(kv[:, 0], kv[:, 1], kp, vp, slots, q=rows, q_out=rows, positions=every, table=table.cuda())
        k = kv[at.cuda(), 0].cpu()
        want_k, _ = R.rope(k, positions, table, False, False)
        R.close(kp[0, 3:3 + len(at)].cpu(), want_k, R.rope_bound(k, want_k, torch.float16))
        assert torch.equal(vp[0, 3:3 + len(at)], kv[at.cuda(), 1])
    else:
        B.hps_seq_rope(rows, rows, every, table.cuda())
    R.close(rows[at.cuda()].cpu(), want, R.rope_bound(x, want, torch.float16))


def test_a_request_that_outgrows_its_table_spoils_no_other():
    """Steps of a request whose table becomes full, and is too short then, between two others: extend, append, attention."""
    block, width, H, K, D, dtype = 4, 3, 4, 2, 64, torch.bfloat16
    g = torch.Generator().manual_seed(9)
    pages = [torch.zeros(20, block, K, D, dtype=dtype, device="cuda") for _ in range(2)]
    free, info, lens = torch.randperm(20, generator=g).int().cuda(), i32(4, fill=20), i32(3, fill=0)
    table, s = i32(3, width, fill=-1), B.hps_seq_attention_create(64, D)
    seen = [[] for _ in range(3)]
    for new, fits in (([2, 7, 1], True), ([3, 5, 4], True), ([1, 3, 2], False)):     # the second one has 7, 12, 15 of 12
        T = sum(new)
        offsets, other, slots, positions, after = i32(4), i32(3), i32(T), i32(T), i32(4)
        B.hps_seq_extend(lens, i32(3).copy_(torch.tensor(new)), block, free, info[:1], table, offsets, other, slots, positions, after)
        lens, info = other, after
        x = torch.randn(T, H + 2 * K, D, generator=g).to(dtype)
        d, at = x.cuda(), [0, *np.cumsum(new)]
        out = torch.full((T, H, D), 9.0, dtype=dtype, device="cuda")
        B.hps_seq_append(d[:, H:H + K], d[:, H + K:], *pages, slots)
        B.hps_seq_attention(s, d[:, :H].contiguous(), *pages, table, lens, offsets, out)
        assert int(info[3]) == (0 if fits else 3) and B.hps_seq_attention_flags(s) == 0
        for r in range(3):
            seen[r].append(x[at[r]:at[r + 1], H:])
            if r == 1 and not fits:
                continue
            kv = torch.cat(seen[r])
            n = kv.shape[0]
            want, _, bound, _ = R.attention(x[at[r]:at[r + 1], :H], kv[None, :, :K], kv[None, :, K:], torch.zeros(1, 1, dtype=torch.int32), [n], [0, new[r]], D ** -0.5)
            R.close(out[at[r]:at[r + 1]].cpu(), want, bound)
    B.hps_seq_attention_destroy(s)
