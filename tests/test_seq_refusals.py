"""What the entry points of hps_seq.h refuse, before anything reaches a GPU; the argument structures' layout."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2210_08804_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x1000                                             # an aligned address that nobody follows


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def test_structures_have_the_size_that_the_binding_packs(tmp_path):
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text('#include <stdio.h>\n#include "hps_seq.h"\nint main(void) { printf("%zu %zu %zu %zu", sizeof(hps_seq_extend_args_t), sizeof(hps_seq_rope_args_t), '
                   "sizeof(hps_seq_append_args_t), sizeof(hps_seq_attention_args_t)); return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    sizes = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert sizes == [B._SEQ_EXTEND.size, B._SEQ_ROPE.size, B._SEQ_APPEND.size, B._SEQ_ATTENTION.size]


def refused(lib, status):
    assert status == B.HPS_ERR_INVALID_ARG
    assert len(lib.hps_seq_last_error()) > 0


EXTEND = dict(past=P, new=P, start=0, free=P, n_free=P, table=P, offsets=P, lens=P + 64, slots=P, positions=P, info=P + 128, n=4, block=16, blocks=8, width=4, most=9)


@pytest.mark.parametrize("bad", [dict(block=0), dict(block=24), dict(block=2048), dict(past=0), dict(new=P + 2), dict(free=0), dict(n_free=0), dict(table=0), dict(offsets=P + 1),
                                 dict(lens=P), dict(slots=0), dict(positions=0), dict(info=P), dict(info=0), dict(start=P + 3), dict(n=(1 << 24) + 1), dict(blocks=1 << 27),
                                 dict(width=1 << 27), dict(most=1 << 31)])
def test_extend(lib, bad):
    refused(lib, lib.hps_seq_extend(B._SEQ_EXTEND.pack(*{**EXTEND, **bad}.values()), None))


def test_null_arguments(lib):
    for call in (lib.hps_seq_extend, lib.hps_seq_rope, lib.hps_seq_append):
        refused(lib, call(None, None))
    refused(lib, lib.hps_seq_attention(None, None, None))
    refused(lib, lib.hps_seq_attention_create(16, 64, None))
    f = C.c_uint32()
    refused(lib, lib.hps_seq_attention_flags(None, C.byref(f), 0))
    assert lib.hps_seq_attention_destroy(None) == B.HPS_OK
    h = C.c_void_p()
    for rows, dim in ((0, 64), (1 << 31, 64), (16, 0), (16, 257)):
        refused(lib, lib.hps_seq_attention_create(rows, dim, C.byref(h)))
        assert h.value is None


def test_release(lib):
    good = [P, P, 4, 16, P, 4, P, 8, P, P]
    for at, value in ((0, None), (1, P + 2), (2, (1 << 24) + 1), (3, 0), (3, 48), (4, None), (5, 1 << 28), (6, None), (7, 1 << 28), (8, None), (9, None)):
        bad = list(good)
        bad[at] = value
        refused(lib, lib.hps_seq_release(*bad, None))


def test_rope_table(lib):
    good = [P, 16, 64, 10000.0, B.HPS_SEQ_SCALE_PARTS, 4.0, 512.0, 1.0, 32.0, 1.0]
    nan, inf = float("nan"), float("inf")
    for at, values in ((0, (None, P + 4)), (1, ((1 << 31) + 1,)), (2, (0, 63, 514)), (3, (0.0, -1.0, nan, inf)), (4, (-1, 3)), (5, (0.0, nan)), (6, (0.0, inf)), (7, (32.0, nan)),
                       (8, (1.0, inf)), (9, (nan,))):
        for value in values:
            bad = list(good)
            bad[at] = value
            refused(lib, lib.hps_seq_rope_table(*bad, None))


HEADS = dict(data=P, token=64, head=64)


def rope(**bad):
    d = dict(q=P, k=P, q_out=P, k_out=P, positions=P, table=P, n=3, qh=2, kh=1, dim=64, rot=64, max_pos=9, dtype=0, inter=0, inverse=0)
    d.update(bad)
    return B._SEQ_ROPE.pack(d["q"], 64, 64, d["k"], 64, 64, d["q_out"], 64, 64, d["k_out"], 64, 64, *list(d.values())[4:])


@pytest.mark.parametrize("bad", [dict(q=0), dict(q_out=P + 2), dict(k=0), dict(k_out=0), dict(positions=0), dict(table=0), dict(table=P + 4), dict(n=1 << 31), dict(qh=65536), dict(dim=0),
                                 dict(dim=513), dict(rot=0), dict(rot=63), dict(rot=66), dict(max_pos=0), dict(max_pos=(1 << 31) + 1), dict(dtype=3), dict(dtype=-1)])
def test_rope(lib, bad):
    refused(lib, lib.hps_seq_rope(rope(**bad), None))


def test_nothing_to_do(lib):
    assert lib.hps_seq_rope(rope(n=0, positions=0), None) == B.HPS_OK
    assert lib.hps_seq_rope(rope(qh=0, kh=0, q=0), None) == B.HPS_OK
    assert lib.hps_seq_append(append(n=0, slots=0), None) == B.HPS_OK
    assert lib.hps_seq_rope_table(None, 0, 64, 10000.0, 0, 1.0, 1.0, 1.0, 2.0, 1.0, None) == B.HPS_OK


def append(**bad):
    d = dict(q=P, q_out=P, k=P, v=P, pk=P, pv=P, blocks=4, block=16, slots=P, positions=P, table=P, n=3, qh=2, kh=1, dim=64, rot=64, max_pos=9, dtype=2, inter=0)
    d.update(bad)
    return B._SEQ_APPEND.pack(d["q"], 64, 64, d["q_out"], 64, 64, d["k"], 64, 64, d["v"], 64, 64, d["pk"], d["pv"], 1024, 64, 64, *list(d.values())[6:])


@pytest.mark.parametrize("bad", [dict(q=0), dict(q_out=0), dict(k=P + 1), dict(v=0), dict(pk=0), dict(pv=P + 1), dict(blocks=1 << 27), dict(block=0), dict(block=12), dict(block=2048), dict(slots=0),
                                 dict(slots=P + 2), dict(positions=0), dict(n=1 << 31), dict(qh=65536), dict(kh=0), dict(dim=0), dict(dim=516), dict(rot=7), dict(max_pos=0), dict(dtype=5)])
def test_append(lib, bad):
    refused(lib, lib.hps_seq_append(append(**bad), None))


def test_the_binding_refuses_what_it_cannot_describe():
    """Tensors on the host never reach the library."""
    i = torch.zeros(4, dtype=torch.int32)
    x = torch.zeros(4, 2, 64)
    with pytest.raises(TypeError, match="device tensor"):
        B.hps_seq_extend(i, i, 16, i, i, i.view(4, 1), torch.zeros(5, dtype=torch.int32), i, i, i, i)
    with pytest.raises(TypeError, match="device tensor"):
        B.hps_seq_rope(x, x, i, torch.zeros(9, 32, 2))
    with pytest.raises(TypeError, match="device tensor"):
        B.hps_seq_append(x, x, x.view(1, 4, 2, 64), x.view(1, 4, 2, 64), i)
    with pytest.raises(TypeError, match="device tensor"):
        B.hps_seq_attention(None, x, x.view(1, 4, 2, 64), x.view(1, 4, 2, 64), i.view(4, 1), i, torch.zeros(5, dtype=torch.int32), x)
    with pytest.raises(ValueError, match="requests, width"):
        B.hps_seq_extend(i, i, 16, i, i, i, torch.zeros(5, dtype=torch.int32), i, i, i, i)


def test_outputs_that_are_missing_are_named():
    x, i = torch.zeros(4, 2, 64), torch.zeros(4, dtype=torch.int32)
    pages = x.view(1, 4, 2, 64)
    with pytest.raises(ValueError, match="k_out: needed with k"):
        B.hps_seq_rope(x, x, i, None, k=x)
    with pytest.raises(ValueError, match="q_out: needed with q"):
        B.hps_seq_append(x, x, pages, pages, i, q=x)
