"""The example that runs the cache and the sequence operators together, against the same model in 64 bits."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def turned(x, positions, dim):
    angle = positions.double()[:, None] * (10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim))
    a, b = x[..., :dim // 2], x[..., dim // 2:]
    cos, sin = angle.cos()[:, None], angle.sin()[:, None]
    return torch.cat((a * cos - b * sin, a * sin + b * cos), -1)


def test_scores_of_candidates():
    import history_scoring as E
    torch.manual_seed(2)
    items, events, candidates = 2000, [37, 1, 150], [4, 9, 2]
    history, asked = torch.randint(0, items, (sum(events),)), torch.randint(0, items + 50, (sum(candidates),))       # some are not cached
    rows = E.Rows(items, 128, 256)
    s = E.Scorer(n_blocks=64, max_events=200, max_candidates=32)
    before = s.free.sort().values.clone(), int(s.info[0])
    try:
        kept = s.take_in(rows(history.cuda()), E.i32(events))
        held = int(s.info[0])
        for _ in range(3):                             # candidates' pages come back every time
            h, c = rows(history.cuda()), rows(asked.cuda())
            scores = s.score(kept, c, E.i32(candidates))
            torch.cuda.synchronize()
            assert int(s.info[0]) == held and held == before[1] - sum(-(-e // 16) for e in events)
        E.B.hps_seq_release(kept[1], torch.ones_like(kept[1]), 16, kept[0], s.free, s.info, E.empty(4))
        assert torch.equal(s.free.sort().values, before[0])
        assert (c[asked.cuda() >= items] == 0).all() and (c[asked.cuda() < items] != 0).any(1).float().mean() > 0.9
        # the model in 64 bits, with the roundings of its stages to 16 bits: projections, turned queries and keys, the output
        f = lambda x: x.to(torch.bfloat16).double()  # noqa: E731
        w, back, H, K, D = s.qkv.double().cpu(), s.back.double().cpu(), s.q_heads, s.kv_heads, s.head_dim
        hx, cx = (f(f(x.cpu()) @ w).view(-1, H + 2 * K, D) for x in (h, c))
        first_event, first = 0, 0
        for u, (e, n) in enumerate(zip(events, candidates)):
            x, y = hx[first_event:first_event + e], cx[first:first + n]
            k = f(turned(x[:, H:H + K], torch.arange(e), D)).repeat_interleave(H // K, 1)
            v = x[:, H + K:].repeat_interleave(H // K, 1)
            at = torch.full((n,), e)
            q, own_k, own_v = f(turned(y[:, :H], at, D)), f(turned(y[:, H:H + K], at, D)).repeat_interleave(H // K, 1), y[:, H + K:].repeat_interleave(H // K, 1)
            a = torch.cat(((q.transpose(0, 1) @ k.permute(1, 2, 0).contiguous()).transpose(0, 1), (q * own_k).sum(-1, keepdim=True)), -1) * D ** -0.5
            p = a.softmax(-1)
            out = (p[..., :e].transpose(0, 1) @ v.transpose(0, 1).contiguous()).transpose(0, 1) + p[..., e:] * own_v
            r = c[first:first + n].double().cpu()
            z = out.reshape(n, -1)
            want = ((z @ back) * r).sum(1)
            # each stage is rounded to 8 bits, twice at most where a product in 32 bits falls beside a step of that rounding: 2^-7 of what its
            # terms add up to, for projections (into scores and values), weights, output, its projection
            score_off = 2.0 ** -6 * (q.abs().transpose(0, 1) @ k.abs().permute(1, 2, 0).contiguous()).amax() * D ** -0.5
            bound = (2.0 ** -5 + 2 * score_off) * ((z.abs() + p.amax() * v.abs().amax()) @ back.abs() * r.abs()).sum(1)
            got = scores[first:first + n].double().cpu()
            assert ((got - want).abs() <= bound + 1e-6).all()
            assert torch.corrcoef(torch.stack((got, want)))[0, 1] > 0.99 or n < 3
            first_event, first = first_event + e, first + n
    finally:
        s.close()
        rows.close()


def test_the_command_runs(capsys):
    import history_scoring as E
    E.main(3, 5, 100)
    assert "flags 0" in capsys.readouterr().out
