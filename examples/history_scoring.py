"""Candidates scored against users' histories: the embedding cache and the sequence operators together.

A user's history is a list of item ids.  Its items' rows are looked up once (distinct keys, query, expansion), projected to
keys and values, turned by their positions and written to pages: the shared part of the user's group.  Every candidate of a
user is a request of that group: its row gives a query, a key and a value, its key and value go to a page of its own, and one
call attends every candidate to its user's whole history and to itself.  The score of a candidate is the product of its
attention's output, projected, with its row.  Finished candidates give their pages back.

    python examples/history_scoring.py [users] [candidates per user] [events per user]
"""
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2210_08804_amd import binding as B  # noqa: E402
from paper_2210_08804_amd import inputs  # noqa: E402


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32, device="cuda")


def empty(*shape):
    return torch.empty(*shape, dtype=torch.int32, device="cuda")


class Rows:
    """Rows of item ids, from an embedding cache with room for four times as many (few sets get more than they hold)."""

    def __init__(self, items, dim, max_keys):
        self.dim, self.handle, self.dedup = dim, B.hps_cache_create(4 * items, 8, dim), B.hps_dedup_create(max_keys)
        keys = torch.arange(items, dtype=torch.int64)
        rows = torch.from_numpy(inputs.backing_rows(keys.numpy(), dim))
        rows = torch.nan_to_num(rows, nan=0.0, posinf=1.0, neginf=-1.0).clamp(-1, 1).cuda()      # the generator's rows are any bit patterns
        B.hps_cache_insert(self.handle, keys.cuda(), rows, items)
        self.miss = empty(max_keys), torch.empty(max_keys, dtype=torch.int64, device="cuda"), empty(1)
        self.distinct, self.inverse, self.n_distinct = torch.empty(max_keys, dtype=torch.int64, device="cuda"), empty(max_keys), empty(1)

    def __call__(self, keys):
        """Distinct keys, their query, expansion to positions.  An item that is not cached has a row of zeros."""
        n = keys.numel()
        rows, out = torch.zeros(n, self.dim, device="cuda"), torch.empty(n, self.dim, device="cuda")
        B.hps_dedup(self.dedup, keys, n, self.distinct, self.inverse, self.n_distinct)
        B.hps_cache_query_dn(self.handle, self.distinct, n, self.n_distinct, rows, *self.miss)
        B.hps_expand_rows(rows, self.inverse, n, self.dim, out)
        return out

    def close(self):
        torch.cuda.synchronize()
        B.hps_dedup_destroy(self.dedup)
        B.hps_cache_destroy(self.handle)


class Scorer:
    """One attention layer over histories in pages."""

    def __init__(self, dim=128, q_heads=8, kv_heads=2, head_dim=64, block=16, n_blocks=4096, max_events=4096, max_candidates=1024, dtype=torch.bfloat16, seed=0):
        g = torch.Generator().manual_seed(seed)
        weight = lambda *s: (torch.randn(*s, generator=g) / s[0] ** 0.5).to(dtype).cuda()  # noqa: E731
        self.q_heads, self.kv_heads, self.head_dim, self.block, self.dtype = q_heads, kv_heads, head_dim, block, dtype
        self.qkv, self.back = weight(dim, (q_heads + 2 * kv_heads) * head_dim), weight(q_heads * head_dim, dim)
        self.k_pages, self.v_pages = (torch.zeros(n_blocks, block, kv_heads, head_dim, dtype=dtype, device="cuda") for _ in range(2))
        self.free, self.info = torch.arange(n_blocks, dtype=torch.int32, device="cuda"), i32([n_blocks, 0, 0, 0])
        self.table = torch.empty(max_events + 1, head_dim // 2, 2, device="cuda")
        B.hps_seq_rope_table(self.table)
        self.session = B.hps_seq_attention_create(max_candidates * q_heads, head_dim)

    def close(self):
        torch.cuda.synchronize()
        B.hps_seq_attention_destroy(self.session)

    def project(self, rows):
        return (rows.to(self.dtype) @ self.qkv).view(rows.shape[0], self.q_heads + 2 * self.kv_heads, self.head_dim)

    def extend(self, past, new, block_table, max_tokens, start=None):
        """Pages for new tokens: (offsets, lens, slots, positions)."""
        n = past.numel()
        out, info = (empty(n + 1), empty(n), empty(max_tokens), empty(max_tokens)), empty(4)
        B.hps_seq_extend(past, new, self.block, self.free, self.info, block_table, *out, info, start=start)
        self.info = info
        return out

    def append(self, x, slots, positions, with_queries):
        H, K = self.q_heads, self.kv_heads
        q = x[:, :H] if with_queries else None
        q_out = torch.empty(x.shape[0], H, self.head_dim, dtype=self.dtype, device="cuda") if with_queries else None
        B.hps_seq_append(x[:, H:H + K], x[:, H + K:], self.k_pages, self.v_pages, slots, q=q, q_out=q_out, positions=positions, table=self.table)
        return q_out

    def take_in(self, rows, events):
        """Histories of `events` [users] rows each, one behind the other in `rows`: (table, lengths), what the candidates share."""
        users = events.numel()
        table = torch.full((users, -(-int(events.max()) // self.block)), -1, dtype=torch.int32, device="cuda")
        _, lens, slots, positions = self.extend(torch.zeros_like(events), events, table, rows.shape[0])
        self.append(self.project(rows), slots, positions, False)
        return table, lens

    def score(self, history, rows, candidates):
        """rows: of the users' candidates, `candidates` [users] of each; returns their scores."""
        prefix_table, prefix_lens = history
        n = rows.shape[0]
        groups = torch.cat((i32([0]), candidates.cumsum(0, dtype=torch.int32)))
        start = torch.repeat_interleave(prefix_lens, candidates, output_size=n)
        table = torch.full((n, 1), -1, dtype=torch.int32, device="cuda")
        offsets, lens, slots, positions = self.extend(torch.zeros_like(start), torch.ones_like(start), table, n, start=start)
        x = self.project(rows)
        q = self.append(x, slots, positions, True)
        out = torch.empty_like(q)
        B.hps_seq_attention(self.session, q, self.k_pages, self.v_pages, table, lens, offsets, out, prefix_table=prefix_table, prefix_lens=prefix_lens,
                            group_offsets=groups, max_new=1, max_len=1)
        scores = ((out.view(n, -1) @ self.back).float() * rows).sum(1)
        self.release(table, lens)
        return scores

    def release(self, table, lens):
        info = empty(4)
        B.hps_seq_release(lens, torch.ones_like(lens), self.block, table, self.free, self.info, info)
        self.info = info


def main(users=26, candidates=40, events=1000):
    items = 1 << 16
    g = torch.Generator().manual_seed(1)
    lens = torch.randint(max(1, events // 4), events + 1, (users,), generator=g).int()
    history = torch.randint(0, items, (int(lens.sum()),), generator=g).cuda()
    asked = torch.randint(0, items, (users * candidates,), generator=g).cuda()
    rows = Rows(items, 128, max(history.numel(), asked.numel()))
    scorer = Scorer(n_blocks=2 * (history.numel() // 16 + users * (candidates + 1)), max_events=events, max_candidates=users * candidates)
    kept = scorer.take_in(rows(history), lens.cuda())
    per_user = i32([candidates] * users)
    for _ in range(3):
        scores = scorer.score(kept, rows(asked), per_user)
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(20):
        scores = scorer.score(kept, rows(asked), per_user)
    torch.cuda.synchronize()
    took = (time.perf_counter() - began) / 20
    best = scores.view(users, candidates).argmax(1)
    flags = B.hps_seq_attention_flags(scorer.session)
    print(f"{users} users, {int(lens.sum())} events, {candidates} candidates each: {took * 1e6:.0f} us a pass, flags {flags}, "
          f"{int(scorer.info[0])} blocks free, best of the first user: candidate {int(best[0])}")
    scorer.close()
    rows.close()


if __name__ == "__main__":
    main(*(int(x) for x in sys.argv[1:4]))
