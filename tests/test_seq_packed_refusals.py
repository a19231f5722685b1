"""What the entry points of head norms and packed pages refuse, before anything reaches a GPU; the argument structures' layout."""
import math
import os
import subprocess

import pytest
import torch

import packed_reference as P
from paper_2210_08804_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x1000                                             # an aligned address that nobody follows


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def refused(lib, status):
    assert status == B.HPS_ERR_INVALID_ARG
    assert len(lib.hps_seq_last_error()) > 0


def test_structures_have_the_size_that_the_binding_packs(tmp_path):
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text('#include <stdio.h>\n#include "hps_seq.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %u", sizeof(hps_seq_norm_args_t), sizeof(hps_seq_packed_t), '
                   "sizeof(hps_seq_append_packed_args_t), sizeof(hps_seq_attention_packed_args_t), sizeof(hps_seq_heads_t), HPS_SEQ_NORM_PARTS); return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    sizes = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert sizes == [B._SEQ_NORM.size, B._SEQ_PACKED.size, B._SEQ_APPEND_PACKED.size, B._SEQ_ATTENTION_PACKED.size, B._SEQ_HEADS.size, B.HPS_SEQ_NORM_PARTS]


def norm(**bad):
    d = dict(q=A, k=A, q_out=A, k_out=A, qw=A, kw=A, positions=A, table=A, eps=1e-6, n=3, qh=2, kh=1, dim=64, rot=64, max_pos=9, dtype=0, inter=0)
    d.update(bad)
    return B._SEQ_NORM.pack(d["q"], 64, 64, d["k"], 64, 64, d["q_out"], 64, 64, d["k_out"], 64, 64, *list(d.values())[4:])


NORM_BAD = [dict(q=0), dict(q_out=A + 2), dict(k=0), dict(k_out=0), dict(qw=A + 2), dict(kw=A + 1), dict(positions=0), dict(table=A + 4), dict(eps=-1e-6), dict(eps=math.inf), dict(eps=1e39),
            dict(eps=math.nan), dict(n=1 << 31), dict(qh=65536), dict(dim=0), dict(dim=513), dict(rot=0), dict(rot=63), dict(rot=66), dict(max_pos=0), dict(max_pos=(1 << 31) + 1), dict(dtype=3),
            dict(dtype=-1)]


@pytest.mark.parametrize("bad", NORM_BAD)
def test_norm_rope(lib, bad):
    refused(lib, lib.hps_seq_norm_rope(norm(**bad), None))


def heads(p=A):
    return B._SEQ_HEADS.pack(p, 64, 64)


@pytest.mark.parametrize("bad", NORM_BAD)
def test_norm_rope_grad(lib, bad):
    refused(lib, lib.hps_seq_norm_rope_grad(norm(**bad), heads(), heads(), A, A, A, None))


def test_norm_rope_grad_outputs(lib):
    for q, k, qw, kw, parts in ((None, heads(), A, A, A), (heads(), None, A, A, A), (heads(0), heads(), A, A, A), (heads(), heads(A + 2), A, A, A), (heads(), heads(), A + 2, A, A),
                                (heads(), heads(), A, A + 1, A), (heads(), heads(), A, A, None), (heads(), heads(), A, None, None), (heads(), heads(), A, A, A + 2)):
        refused(lib, lib.hps_seq_norm_rope_grad(norm(), q, k, qw, kw, parts, None))


def test_nothing_to_do(lib):
    assert lib.hps_seq_norm_rope(norm(n=0, positions=0), None) == B.HPS_OK
    assert lib.hps_seq_norm_rope(norm(qh=0, kh=0, q=0, table=0, rot=7), None) == B.HPS_OK
    assert lib.hps_seq_norm_rope_grad(norm(n=0), None, None, None, None, None, None) == B.HPS_OK
    assert lib.hps_seq_append_packed(append(n=0, slots=0), None) == B.HPS_OK
    assert lib.hps_seq_read_packed(pages(), None, 0, 1, 64, heads(), heads(), 0, None) == B.HPS_OK
    assert lib.hps_seq_read_packed(pages(blocks=0, data=0), A, 5, 1, 64, heads(), heads(), 0, None) == B.HPS_OK
    assert lib.hps_seq_read_packed(pages(), A, 5, 1, 64, heads(0), heads(0), 0, None) == B.HPS_OK


def test_packed_bytes():
    for block in (16, 32, 1024):
        for dim in (32, 64, 96, 128, 256):
            (kb, _), (vb, _), ks, vs = P.places(block, dim)
            every = torch.cat([x.flatten() for x in (kb[:, ::2], ks, vs)] + [vb[:, ::2].flatten()]).sort().values
            assert torch.equal(every, torch.arange(B.hps_seq_packed_bytes(block, dim)))          # every byte of a tile is one thing
    for block, dim in ((8, 64), (24, 64), (2048, 64), (0, 64), (16, 0), (16, 16), (16, 48), (16, 160), (16, 512)):
        assert B.hps_seq_packed_bytes(block, dim) == 0


def append(**bad):
    d = dict(q=A, q_out=A, k=A, v=A, data=A, bs=4352, hs=1088, blocks=4, block=16, slots=A, positions=A, table=A, qw=A, kw=A, eps=1e-6, n=3, qh=2, kh=1, dim=64, rot=64, max_pos=9, dtype=2, inter=0, norm=1)
    d.update(bad)
    return B._SEQ_APPEND_PACKED.pack(d["q"], 64, 64, d["q_out"], 64, 64, d["k"], 64, 64, d["v"], 64, 64, *list(d.values())[4:])


@pytest.mark.parametrize("bad", [dict(q=0), dict(q_out=0), dict(k=A + 1), dict(k=0), dict(v=0), dict(data=0), dict(data=A + 8), dict(bs=-16), dict(bs=8), dict(hs=1087), dict(hs=-1088),
                                 dict(blocks=1 << 27), dict(block=0), dict(block=8), dict(block=48), dict(block=2048), dict(slots=0), dict(slots=A + 2), dict(positions=0), dict(qw=A + 1), dict(kw=A + 2),
                                 dict(eps=-1.0), dict(eps=math.nan), dict(n=1 << 31), dict(qh=65536), dict(kh=0), dict(dim=0), dict(dim=48), dict(dim=160), dict(dim=512), dict(rot=7), dict(rot=66),
                                 dict(max_pos=0), dict(dtype=5)])
def test_append_packed(lib, bad):
    refused(lib, lib.hps_seq_append_packed(append(**bad), None))


def pages(**bad):
    return B._SEQ_PACKED.pack(*{**dict(data=A, bs=4352, hs=1088, blocks=4, block=16), **bad}.values())


def test_read_packed(lib):
    good = [pages(), A, 5, 1, 64, heads(), heads(), 0]
    for at, value in ((0, None), (0, pages(data=0)), (0, pages(hs=8)), (0, pages(block=8)), (0, pages(blocks=1 << 27)), (1, None), (1, A + 2), (2, 1 << 31), (3, 0), (3, 65537), (4, 48), (5, None),
                      (5, heads(A + 2)), (6, None), (6, heads(A + 1)), (7, 3), (7, -1)):
        bad = list(good)
        bad[at] = value
        refused(lib, lib.hps_seq_read_packed(*bad, None))


def test_null_arguments(lib):
    for call in (lib.hps_seq_norm_rope, lib.hps_seq_append_packed):
        refused(lib, call(None, None))
    refused(lib, lib.hps_seq_norm_rope_grad(None, heads(), heads(), None, None, None, None))
    refused(lib, lib.hps_seq_attention_packed(None, None, None))


def test_the_binding_refuses_what_it_cannot_describe():
    """Tensors on the host never reach the library; outputs that are missing are named."""
    i, x = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, 64)
    tiles = torch.zeros(1, 2, 16 * 68, dtype=torch.uint8)
    for call in (lambda: B.hps_seq_norm_rope(x, x), lambda: B.hps_seq_norm_rope_grad(x, x, x), lambda: B.hps_seq_append_packed(x, x, tiles, i),
                 lambda: B.hps_seq_read_packed(tiles, i, x, x), lambda: B.hps_seq_attention_packed(None, x, tiles, i.view(4, 1), i, torch.zeros(5, dtype=torch.int32), x)):
        with pytest.raises(TypeError, match="device tensor"):
            call()
    with pytest.raises(ValueError, match="k_out: needed with k"):
        B.hps_seq_norm_rope(x, x, k=x)
    with pytest.raises(ValueError, match="positions: needed with a table"):
        B.hps_seq_norm_rope(x, x, table=torch.zeros(9, 32, 2))
    with pytest.raises(ValueError, match="q_out: needed with q"):
        B.hps_seq_append_packed(x, x, tiles, i, q=x)
    with pytest.raises(ValueError, match="one is needed"):
        B.hps_seq_read_packed(tiles, i)


def test_the_definition_of_gradients_agrees_with_differences():
    """The reference's gradients of norms and rotations, against central differences of its forward pass in 64 bits."""
    g = torch.Generator().manual_seed(1)
    T, H, D, rot = 3, 2, 12, 8
    x, back, w = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((T, H, D), (T, H, D), (D,)))
    angle = torch.rand(5, rot // 2, generator=g, dtype=torch.float64)
    table, positions = torch.stack((angle.cos(), angle.sin()), -1), torch.tensor([4, 0, 2])
    for interleaved in (False, True):
        dx, _, dw, _ = P.norm_rope_grad(x.float(), w.float(), back.float(), positions, table, 1e-3, interleaved)
        xd, wd, bd = x.float().double(), w.float().double(), back.float().double()
        loss = lambda x, w: float((P.turned(P.normed(x, w, 1e-3), positions, table, interleaved) * bd).sum())  # noqa: E731, B023
        h = 1e-5
        for t, grad in ((xd, dx), (wd, dw)):
            for j in range(0, t.numel(), 5):
                step = torch.zeros_like(t).view(-1)
                step[j] = h
                step = step.view(t.shape)
                slope = (loss(xd + step, wd) - loss(xd - step, wd)) / (2 * h) if t is xd else (loss(xd, wd + step) - loss(xd, wd - step)) / (2 * h)
                assert abs(slope - float(grad.reshape(-1)[j])) < 1e-7       # third derivatives of size 10 times h^2, roundings of 1e-15 over h
