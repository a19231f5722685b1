"""Norms of heads with their rotation, and the gradients (hps_seq_norm_rope, hps_seq_norm_rope_grad), against the definition in 64 bits."""
import math

import pytest
import torch

import packed_reference as P
import seq_reference as R
from paper_2210_08804_amd import binding as B

pytestmark = pytest.mark.gpu
F32, HF, BF = torch.float32, torch.float16, torch.bfloat16


def table_of(positions, rot, seed=3):
    angle = torch.rand(positions, rot // 2, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * 6.3
    return torch.stack((angle.cos(), angle.sin()), -1).float()


class Heads:
    """Queries, keys and gradients in rows of one array, `lead` values from its start."""

    def __init__(self, dtype, T, H, K, D, rot=None, seed=0, size=1.5, lead=0, positions=50, weights=True):
        g = torch.Generator().manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        width = (H + K + 1) * D + lead
        self.row = (normal(T, width) * size).to(dtype)
        self.back = normal(T, width).to(dtype)
        cut = lambda r: (r[:, lead:lead + H * D].view(T, H, D) if T and H else r.new_zeros(T, H, D),  # noqa: E731
                         r[:, lead + H * D:lead + (H + K) * D].view(T, K, D) if T and K else r.new_zeros(T, K, D))
        self.cut, self.dtype, self.T, self.H, self.K, self.D = cut, dtype, T, H, K, D
        self.table = table_of(positions, rot) if rot else None
        self.positions = torch.randint(0, positions, (T,), generator=g).int()
        self.qw, self.kw = (1 + 0.3 * normal(D), 1 + 0.3 * normal(D)) if weights else (None, None)

    def kw_of(self, eps, interleaved):
        cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
        return dict(q_weight=cuda(self.qw), k_weight=cuda(self.kw), positions=self.positions.cuda() if self.table is not None else None, table=cuda(self.table), eps=eps,
                    interleaved=interleaved)

    def check(self, eps=1e-6, interleaved=False, in_place=False):
        q, k = self.cut(self.row.cuda())
        if in_place:
            q_out, k_out = q, k
        else:
            q_out, k_out = torch.full_like(q, 9.0), torch.full((self.K, self.T, self.D), 9.0, dtype=self.dtype, device="cuda").transpose(0, 1)
        B.hps_seq_norm_rope(q, q_out, k=k if self.K else None, k_out=k_out if self.K else None, **self.kw_of(eps, interleaved))
        torch.cuda.synchronize()
        keep = P.live(self.positions, self.table, self.T)
        for x, w, got in zip(self.cut(self.row), (self.qw, self.kw), (q_out, k_out)):
            want, bound = P.norm_rope(x, w, self.positions, self.table, eps, interleaved)
            R.close(got.cpu()[keep], want[keep], bound[keep])
            assert torch.equal(got.cpu()[~keep], x[~keep] if in_place else torch.full_like(x[~keep], 9.0))

    def grads(self, eps=1e-6, interleaved=False, alias=None, stream=None, wanted=True):
        """(dq, dk, dwq, dwk) of the device."""
        q, k = self.cut(self.row.cuda())
        bq, bk = self.cut(self.back.cuda())
        dq, dk = (q, k) if alias == "x" else (bq, bk) if alias == "back" else (torch.full_like(q, 9.0), torch.full_like(k, 9.0))
        wq, wk = (torch.full((self.D,), 9.0, device="cuda") for _ in range(2))
        parts = torch.full((B.HPS_SEQ_NORM_PARTS * 2 * self.D,), math.nan, device="cuda")
        torch.cuda.synchronize()
        B.hps_seq_norm_rope_grad(q, bq, dq, q_weight_grad=wq if wanted else None, k=k if self.K else None, k_out_grad=bk if self.K else None, k_grad=dk if self.K else None,
                                 k_weight_grad=wk if wanted else None, parts=parts if wanted else None, stream=stream, **self.kw_of(eps, interleaved))
        torch.cuda.synchronize()
        return dq.cpu(), dk.cpu(), wq.cpu(), wk.cpu()

    def check_grads(self, eps=1e-6, interleaved=False, **kw):
        got = self.grads(eps, interleaved, **kw)
        keep = P.live(self.positions, self.table, self.T)
        left = [torch.full_like(x, 9.0) for x in got[:2]] if kw.get("alias") is None else self.cut(self.row if kw["alias"] == "x" else self.back)
        for i, (x, back, w) in enumerate(zip(self.cut(self.row), self.cut(self.back), (self.qw, self.kw))):
            dx, bound, dw, w_bound = P.norm_rope_grad(x, w, back, self.positions, self.table, eps, interleaved)
            R.close(got[i][keep], dx[keep], bound[keep])
            assert torch.equal(got[i][~keep], left[i][~keep])
            if kw.get("wanted", True):
                R.close(got[2 + i], dw, w_bound)
            else:
                assert (got[2 + i] == 9).all()


@pytest.mark.parametrize("dtype", [F32, HF, BF])
@pytest.mark.parametrize("D,rot", [(1, 0), (2, 2), (5, 4), (8, 8), (16, 8), (24, 24), (32, 16), (40, 8), (64, 64), (96, 96), (96, 48), (100, 50), (128, 128), (128, 64), (129, 128), (256, 256), (511, 2),
                                   (512, 512)])
def test_head_dims(D, rot, dtype):
    for interleaved in (False, True):
        h = Heads(dtype, 7, 4, 2, D, rot, seed=D)
        h.check(interleaved=interleaved)
        h.check_grads(interleaved=interleaved)


@pytest.mark.parametrize("T,H,K", [(T, *heads) for T in (0, 1, 2, 3, 31) for heads in ((1, 0), (5, 5), (8, 2), (33, 1), (48, 8))] + [(1025, 33, 1), (5003, 8, 2), (5003, 1, 0)])
def test_tokens_and_heads(T, H, K):
    h = Heads(BF, T, H, K, 64, 64, seed=T + H)
    h.check()
    h.check_grads()


def test_many_tokens():
    """More tokens than work-groups, of which each goes through several."""
    h = Heads(F32, 20011, 2, 1, 32, 32, seed=4)
    h.check()
    h.check_grads()


@pytest.mark.parametrize("dtype", [F32, HF, BF])
@pytest.mark.parametrize("lead", [1, 4, 8])
def test_rows_that_start_anywhere(lead, dtype):
    """Rows that are not in whole 16-byte vectors."""
    h = Heads(dtype, 9, 3, 2, 64, 32, seed=lead, lead=lead)
    for interleaved in (False, True):
        h.check(interleaved=interleaved)
        h.check_grads(interleaved=interleaved)


def test_without_table_and_without_weights():
    for dtype in (F32, BF):
        for h in (Heads(dtype, 9, 3, 2, 96, None, seed=1), Heads(dtype, 9, 3, 2, 96, 96, seed=2, weights=False), Heads(dtype, 9, 3, 0, 96, None, seed=3, weights=False)):
            h.check()
            h.check_grads()
            h.check_grads(wanted=False)


def test_outputs_that_are_inputs():
    for lead in (0, 1):
        h = Heads(BF, 33, 5, 2, 128, 64, seed=7, lead=lead)
        h.check(in_place=True)
        h.check_grads(alias="x")
        h.check_grads(alias="back")


def test_positions_that_are_none():
    """Negative ones are passed over: their rows stay, and have no part in the weights' gradients.  Ones behind the table turn to NaN."""
    h = Heads(F32, 40, 3, 2, 64, 32, seed=8)
    h.positions[::3] = -1
    h.positions[1] = -2 ** 31
    h.check()
    h.check_grads()
    h.positions[:] = -1
    h.check_grads()                                    # gradients of the weights are 0
    h.positions[:] = 5
    h.positions[7], h.positions[8] = 50, 2 ** 31 - 1
    h.check()
    got = h.grads()
    for x in got[:2]:
        assert torch.isnan(x[7:9]).all() and torch.isfinite(x[:7]).all() and torch.isfinite(x[9:]).all()
    for x in got[2:]:                                  # of the values that are turned
        assert torch.isnan(x[:32]).all() and torch.isfinite(x[32:]).all()


@pytest.mark.parametrize("dtype", [F32, HF, BF])
def test_sizes_of_values(dtype):
    """Heads of zeros, tiny and large ones; a head that is not finite leaves the others alone."""
    big = 60000.0 if dtype is HF else 2.0 ** 58
    h = Heads(dtype, 8, 2, 1, 64, 64, seed=9)
    h.row[0] = 0
    h.row[1] *= 1e-4 if dtype is HF else 1e-15
    h.row[2] = (torch.sign(h.row[2].float()) * big).to(dtype)
    h.check(eps=1e-6)
    h.check(eps=1e-3)
    h.row[0, 5] = 1                                    # one value among zeros
    h.check(eps=0.0)
    h.check_grads(eps=1e-6)
    for odd in (math.inf, -math.inf, math.nan):
        x = Heads(dtype, 8, 2, 1, 64, None, seed=10)
        x.row[3, 2] = odd
        q, _ = x.cut(x.row.cuda())
        out = torch.empty_like(q)
        B.hps_seq_norm_rope(q, out)
        torch.cuda.synchronize()
        assert torch.isnan(out[3, 0, 2]) and torch.isfinite(out[3, 1]).all() and torch.isfinite(out[:3]).all() and torch.isfinite(out[4:]).all()


def test_twice_the_same():
    """The weights' gradients are summed in an order that is always the same."""
    h = Heads(BF, 3001, 8, 2, 128, 128, seed=11)
    a, b = h.grads(), h.grads()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_stream_of_its_own():
    h = Heads(BF, 300, 8, 2, 128, 128, seed=12)
    want = h.grads()
    s = torch.cuda.Stream()
    got = h.grads(stream=s)
    assert all(torch.equal(x, y) for x, y in zip(want, got))


def test_captured_and_replayed():
    """Forward and backward in one graph, replayed on new inputs, with the eager calls between."""
    h = Heads(BF, 130, 4, 2, 64, 64, seed=13)
    kw = h.kw_of(1e-6, False)
    (q, k), (bq, bk) = h.cut(h.row.cuda()), h.cut(h.back.cuda())
    bufs = lambda: [torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(q), torch.zeros_like(k), torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")]  # noqa: E731
    parts = [torch.empty(B.HPS_SEQ_NORM_PARTS * 2 * 64, device="cuda") for _ in range(2)]

    def step(o, p):
        B.hps_seq_norm_rope(q, o[0], k=k, k_out=o[1], **kw)
        B.hps_seq_norm_rope_grad(q, bq, o[2], q_weight_grad=o[4], k=k, k_out_grad=bk, k_grad=o[3], k_weight_grad=o[5], parts=p, **kw)

    eager, graphed = bufs(), bufs()
    step(eager, parts[0])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(graphed, parts[1])
    for i in range(4):
        q.mul_(1 + 0.25 * i)
        bk.add_(0.125)
        step(eager, parts[0])
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(eager, graphed))


def test_gradients_by_differences():
    """The loss sum(y * b) along a direction, by central differences of the kernel's own forward pass in 32 bits."""
    T, H, D = 6, 2, 64
    h = Heads(F32, T, H, 0, D, 32, seed=14)
    kw = h.kw_of(1e-6, False)
    q, b = h.cut(h.row.cuda())[0].contiguous(), h.cut(h.back.cuda())[0].contiguous()
    dq, dw, parts = torch.empty_like(q), torch.empty(D, device="cuda"), torch.empty(B.HPS_SEQ_NORM_PARTS * 2 * D, device="cuda")
    B.hps_seq_norm_rope_grad(q, b, dq, q_weight_grad=dw, parts=parts, **kw)
    g = torch.Generator().manual_seed(15)
    u, uw = torch.randn(T, H, D, generator=g).cuda(), torch.randn(D, generator=g).cuda()
    step = 2.0 ** -6

    def loss(sign, what):
        out = torch.empty_like(q)
        more = dict(kw, q_weight=kw["q_weight"] + sign * step * uw) if what == "w" else kw
        B.hps_seq_norm_rope(q + sign * step * u if what == "x" else q, out, **more)
        return float((out.double() * b.double()).sum())

    for what, along in (("x", float((dq.double() * u.double()).sum())), ("w", float((dw.double() * uw.double()).sum()))):
        slope = (loss(1, what) - loss(-1, what)) / (2 * step)
        # third derivatives along a unit-size direction times step^2 / 6 (values and their derivatives are of size 1; 768 of them), and 32 bits' roundings over the step
        assert abs(slope - along) <= T * H * D * (step * step + 64 * 2.0 ** -24 / step)


@pytest.mark.parametrize("size", [1e-15, 1e-18, 1e-19, 3e-20, 1e-20])
@pytest.mark.parametrize("dim", [64, 63])
def test_small_heads(size, dim):
    """Mean squares on both sides of 2^-126, eps 0.  Below it a square, a sum of dim squares and their mean are each off by 2^-150 at most: the mean by 2^-149 in all, where it is
    size^2 at least, and the root by half of that."""
    g = torch.Generator().manual_seed(5)
    x, dy = size * (1 + torch.rand(3, 2, dim, generator=g) / 2), torch.randn(3, 2, dim, generator=g)
    y, dx = torch.empty_like(x).cuda(), torch.empty_like(x).cuda()
    B.hps_seq_norm_rope(x.cuda(), y, eps=0.0)
    B.hps_seq_norm_rope_grad(x.cuda(), dy.cuda(), dx, eps=0.0)
    xd, d = x.double(), dy.double()
    r = xd.square().mean(-1, keepdim=True).rsqrt()
    n = xd * r
    off = dim * 2.0 ** -24 + 2.0 ** -149 / size ** 2
    assert ((y.cpu().double() - n).abs() <= off * n).all()
    # r, n and the mean of d n (n <= 1.5) are each off by `off` at most: (1 + 2 * 1.5 * 1.5) * off, and the sum's own dim * 2^-24
    expected = r * (d - n * (d * n).mean(-1, keepdim=True))
    assert ((dx.cpu().double() - expected).abs() <= r * d.abs().amax(-1, keepdim=True) * 8 * off).all()


@pytest.mark.parametrize("eps", [1e-6, 1e-38, 1e-41, 1e-60])
def test_heads_of_zeros_stay_zeros(eps):
    x, y = torch.zeros(2, 3, 64, device="cuda"), torch.ones(2, 3, 64, device="cuda")
    B.hps_seq_norm_rope(x, y, eps=eps)
    assert (y == 0).all()


SIZES = [(F32, s) for s in (1e-42, 1e-38, 1e-30, 1e-24, 1e-22, 1e19, 1e20, 1e30, 1e38)] + [(BF, s) for s in (1e-38, 1e-30, 1e-22, 1e20, 1e38)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,size", SIZES)
def test_heads_of_any_size(dtype, size, interleaved):
    """Heads whose squares 32 bits do not hold, beside ordinary ones; gradients of them too."""
    for D, rot, eps in ((64, 64, 0.0), (64, None, 0.0), (63, 32, 0.0), (128, 64, min(size * size / 4, 1e-6)), (64, 32, min(size * size * 1e-6, 1e30))):
        h = Heads(dtype, 5, 3, 2, D, rot, seed=16)
        odd, (q, k) = h.row.clone(), h.cut(h.row)
        for x in h.cut(odd):
            x.copy_((x.double().clamp(-2, 2) * size).to(dtype))
        h.row[1], h.row[4] = odd[1], odd[4]
        h.cut(h.row)[0][2, 1] = h.cut(odd)[0][2, 1]    # one of a token's heads
        h.check(eps=eps, interleaved=interleaved)
        if size < 1:
            h.back = (h.back.double() * max(size, 1e-20) ** 0.5).to(dtype)
        h.check_grads(eps=eps, interleaved=interleaved)


def test_gradients_whose_products_are_large_or_small():
    """Values and gradients whose products' sum 32 bits do not hold, where they hold the heads' gradients."""
    h = Heads(F32, 3, 2, 1, 64, 64, seed=17)
    h.row[1] *= 1e18
    h.back[1] *= 1e22
    h.row[2] *= 1e-12
    h.back[2] *= 1e-32
    h.check_grads(eps=0.0)
