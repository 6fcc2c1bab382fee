"""The calls on pages refuse every output that shares memory with an input or with another output, on the host, before anything is
launched (no GPU here)."""
import ctypes as C

import pytest

from paper_2506_19651_b200 import binding as pb
from paper_2506_19651_b200 import build as pbuild

SEQS, MAX_PAGES, NUM_PAGES, ROWS = 5, 7, 11, 24
RELEASE = dict(finished=SEQS, lens=SEQS, page_table=SEQS * MAX_PAGES, free_list=NUM_PAGES, free_count=1, lens_out=SEQS, free_count_out=1)
RELEASE_OUT = ("free_list", "lens_out", "free_count_out")
ASSIGN = dict(lens=SEQS, new_lens=SEQS, page_table=SEQS * MAX_PAGES, free_list=NUM_PAGES, free_count=1, lens_out=SEQS, free_count_out=1,
              row_start=SEQS + 1, slots=ROWS, positions=ROWS)
ASSIGN_OUT = ("page_table", "lens_out", "free_count_out", "row_start", "slots", "positions")


def _call(names, addresses, rows=ROWS):
    lib, g = pb.lib(), pb.make_pages(NUM_PAGES, 16, SEQS, MAX_PAGES)
    args = [C.c_void_p(addresses[n]) for n in names]
    return lib.pevlm_pages_release(C.byref(g), *args, None) if names is RELEASE else lib.pevlm_pages_assign(C.byref(g), *args, rows, None)


@pytest.mark.parametrize("names,outputs", [(RELEASE, RELEASE_OUT), (ASSIGN, ASSIGN_OUT)], ids=["release", "assign"])
def test_every_pair(names, outputs):
    pbuild.build()
    apart = {n: 4096 * (i + 1) for i, n in enumerate(names)}
    for out in outputs:
        for other in names:
            if other == out:
                continue
            step = 4 if not {out, other} & {"slots", "positions"} else 16  # these two have to be aligned
            size, others = 4 * names[out], 4 * names[other]
            # the same place; the output's first entries on the other's last ones, and the other way round
            for offset in (0, (others - 1) // step * step, -((size - 1) // step * step)):
                moved = dict(apart)
                moved[out] = apart[other] + offset
                assert _call(names, moved) == pb.PEVLM_EINVAL, (out, other, offset)


@pytest.mark.gpu
def test_side_by_side_is_served():
    """All arrays of a step as neighbouring parts of one buffer; arrays of no rows may stand anywhere."""
    import torch
    pbuild.build()
    g = pb.make_pages(NUM_PAGES, 16, SEQS, MAX_PAGES)
    buf = torch.zeros(1024, dtype=torch.int32, device="cuda")
    at, part = 0, {}
    for name, n in (("slots", ROWS), ("positions", ROWS), ("lens", SEQS), ("mid", SEQS), ("new_lens", SEQS), ("finished", SEQS), ("page_table", SEQS * MAX_PAGES),
                    ("free_list", NUM_PAGES), ("free_count", 1), ("count_mid", 1), ("row_start", SEQS + 1)):
        part[name] = buf[at:at + n]
        at += n
    part["free_list"].copy_(torch.arange(NUM_PAGES, device="cuda"))
    part["free_count"].fill_(NUM_PAGES)
    part["new_lens"].copy_(torch.tensor([3, 0, 17, 1, 2], device="cuda"))
    p = part
    pb.pevlm_pages_release(g, p["finished"], p["lens"], p["page_table"], p["free_list"], p["free_count"], p["mid"], p["count_mid"])
    pb.pevlm_pages_assign(g, p["mid"], p["new_lens"], p["page_table"], p["free_list"], p["count_mid"], p["lens"], p["free_count"], p["row_start"], p["slots"],
                          p["positions"], ROWS)
    assert p["lens"].tolist() == [3, 0, 17, 1, 2] and p["row_start"].tolist() == [0, 3, 3, 20, 21, 23]
    pages = [10, 9, 8, 7, 6]  # from the top of the list
    assert p["slots"].tolist() == [160, 161, 162] + [144 + i for i in range(16)] + [128, 112, 96, 97, -1] and int(p["free_count"]) == NUM_PAGES - len(pages)
    assert bool((buf[at:] == 0).all())
    p["new_lens"].zero_()
    assert p["page_table"].data_ptr() % 16 == 0
    pb.pevlm_pages_assign(g, p["lens"], p["new_lens"], p["page_table"], p["free_list"], p["free_count"], p["mid"], p["count_mid"], p["row_start"],
                          p["page_table"], p["page_table"], 0)
    assert p["lens"].tolist() == [3, 0, 17, 1, 2]


def test_rows_that_a_step_cannot_bring():
    pbuild.build()
    lib, g = pb.lib(), pb.make_pages(NUM_PAGES, 16, SEQS, MAX_PAGES)
    args = [C.c_void_p(4096 * (i + 1)) for i in range(10)]
    for room, n in ((ROWS, -1), (ROWS, ROWS + 1), (0, 1), (-1, -1)):
        assert lib.pevlm_pages_assign_rows(C.byref(g), *args, room, n, None, None) == pb.PEVLM_EINVAL
    args[5] = args[0]
    assert lib.pevlm_pages_assign_rows(C.byref(g), *args, ROWS, ROWS, None, None) == pb.PEVLM_EINVAL


def test_key_lens_apart_from_everything():
    pbuild.build()
    lib, g = pb.lib(), pb.make_pages(NUM_PAGES, 16, SEQS, MAX_PAGES)
    args = [C.c_void_p(4096 * (i + 1)) for i in range(10)]
    for i, (name, n) in enumerate(ASSIGN.items()):
        for offset in (0, 4 * n - 4, 4 - 4 * SEQS):
            assert lib.pevlm_pages_assign_rows(C.byref(g), *args, ROWS, ROWS, C.c_void_p(4096 * (i + 1) + offset), None) == pb.PEVLM_EINVAL, name
    assert lib.pevlm_pages_assign_rows(C.byref(g), *args, ROWS, ROWS, C.c_void_p(2), None) == pb.PEVLM_EALIGN
