"""Sequences that a step turns away: what they hold, and nothing else, stays theirs."""
import numpy as np
import pytest

import packed_reference as R

pytestmark = pytest.mark.gpu


def _i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _rows(n, heads=(4, 2, 2), seed=0):
    import torch
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return [torch.randn((n, h, 64), generator=gen, device="cuda").to(torch.bfloat16) for h in heads]


CASES = [  # pages, page_len, sequences, max_pages, longest held, most new, capacity, rows that come
    (64, 16, 7, 20, 60, 5, 64, 9), (3000, 16, 300, 40, 100, 200, 70000, 13001), (900, 128, 1024, 3, 128, 100, 60000, 0), (4000, 64, 1025, 9, 300, 1, 2048, 300),
    (9000, 32, 2500, 12, 90, 64, 100001, 100001), (30, 16, 40, 8, 16, 33, 2000, 1999)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_rows_that_do_not_come(case):
    """pevlm_pages_assign_rows against the sequential allocator with that many rows; slots and positions up to the capacity."""
    import torch
    from paper_2506_19651_b200 import binding as pb
    pages, P, seqs, most, longest, new_most, room, n = case
    rng = np.random.default_rng(pages + n)
    lens = np.minimum(rng.integers(0, longest + 1, seqs), most * P)
    while (-(-lens // P)).sum() > pages:
        lens //= 2
    held = -(-lens // P)
    order = rng.permutation(pages)
    table = np.full((seqs, most), -1, np.int32)
    for r in range(seqs):
        table[r, :held[r]] = order[held[:r].sum():held[:r + 1].sum()]
    count = pages - int(held.sum())
    free = np.concatenate([order[pages - count:], np.full(pages - count, -7)]).astype(np.int32)
    new = rng.integers(0, new_most + 1, seqs) * (rng.random(seqs) < 0.9)
    ref = R.Allocator(pages, P, seqs, most)
    w_lens, w_table, w_count, w_start, w_slots, w_positions = ref.assign(lens, new, table, free, count, n)
    _, _, _, _, _, all_positions = ref.assign(lens, new, table, free, count, room)
    d_table, out, count_out = _i32(table), _i32(np.zeros(seqs)), _i32([-1])
    start, slots, positions = _i32(np.full(seqs + 1, -99)), _i32(np.full(room + 8, -99)), _i32(np.full(room + 8, -99))
    pb.pevlm_pages_assign_rows(pb.make_pages(pages, P, seqs, most), _i32(lens), _i32(new), d_table, _i32(free), _i32([count]), out, count_out, start, slots,
                               positions, room, n)
    assert np.array_equal(out.cpu().numpy(), w_lens) and int(count_out) == w_count and np.array_equal(start.cpu().numpy(), w_start)
    assert np.array_equal(slots.cpu().numpy()[:n], w_slots) and bool((slots[n:room] == -1).all()) and bool((slots[room:] == -99).all())
    assert np.array_equal(positions.cpu().numpy()[:room], all_positions) and bool((positions[room:] == -99).all())
    for r in range(seqs):  # entries within the lengths
        assert np.array_equal(d_table.cpu().numpy()[r, :-(-w_lens[r] // P)], w_table[r, :-(-w_lens[r] // P)])


@pytest.mark.parametrize("way", ["step", "extend with rows", "extend"])
def test_a_sequence_whose_rows_are_not_all_there_holds_none_of_them(way):
    """Two of the five new rows of the second sequence do not come.  Its pages held another sequence's tokens before."""
    import torch
    from paper_2506_19651_b200.layer import PackedCache
    make = lambda: PackedCache(2, 64, 4, 16, 64, 4, 2, 64, 1e4)
    c = make()
    q, k, v = _rows(64, seed=1)
    c.step(q, k, v, _i32([0, 64]))                              # all pages
    c.step(*_rows(0), _i32([0, 0]), _i32([0, 1]))               # given back
    q, k, v = _rows(20, seed=2)
    c.step(q, k, v, _i32([10, 10]))
    q, k, v = _rows(4, seed=3)
    new = _i32([1, 5])
    if way == "step":
        c.step(q, k, v, new)
    else:
        c.extend(new, rows=4) if way == "extend with rows" else c.extend(new)
        c.store(k, v)
    assert c.lens.tolist() == [11, 10] and int(c.free_count) == 2
    assert c.slots.tolist()[1:] == [-1] * 63 and c.positions.tolist()[:6] == [10, 10, 11, 12, 13, 14] and c.row_start.tolist() == [0, 1, 6]
    # it goes on as if that step had never been
    q, k, v = _rows(5, seed=4)
    o, lse = c.step(q, k, v, _i32([0, 5]))
    twin = make()
    q0, k0, v0 = _rows(20, seed=2)
    twin.step(q0, k0, v0, _i32([10, 10]))
    want, want_lse = twin.step(q, k, v, _i32([0, 5]))
    assert c.lens.tolist() == [11, 15] and torch.equal(o, want) and torch.equal(lse, want_lse)


def test_all_rows_that_come_are_held():
    """store() of all rows of a step (padding among them) leaves what extend() granted."""
    import torch
    from paper_2506_19651_b200.layer import PackedCache
    c = PackedCache(2, 64, 8, 16, 64, 4, 2, 64, 1e4)
    for rows in (None, 9):
        before = c.lens.tolist()
        c.extend(_i32([3, 5]), rows=rows)
        c.store(*_rows(9, (2, 2)))
        assert c.lens.tolist() == [before[0] + 3, before[1] + 5] and c.slots.tolist()[8:] == [-1] * 56
    assert int(c.free_count) == 6
    with pytest.raises(ValueError, match="rows for a step of 4"):
        c.extend(_i32([0, 0]), rows=4)
        c.store(*_rows(5, (2, 2)))
    with pytest.raises(ValueError, match="at most 64 fit"):
        c.extend(_i32([0, 0]), rows=65)


@pytest.mark.parametrize("why", ["the free list", "the table", "the room for rows", "rows that do not come"])
def test_rows_that_were_turned_away_say_so(why):
    """Output 0 and LSE -inf for all of them, and the right numbers for the others."""
    import torch
    from paper_2506_19651_b200.layer import PackedCache
    make = lambda pages: PackedCache(3, 48, pages, 16, 40, 4, 2, 64, 1e4)
    c, twin = make(4 if why == "the free list" else 9), make(9)  # 9, 20 and 3 tokens hold four
    first = _rows(32, seed=5)
    for x in (c, twin):
        x.step(*first, _i32([9, 20, 3]))
    new = {"the free list": [7, 20, 1], "the table": [7, 29, 1], "the room for rows": [7, 2, 32], "rows that do not come": [7, 2, 9]}[why]
    turned = {"the free list": 1, "the table": 1}.get(why, 2)
    n = {"the room for rows": 40, "rows that do not come": 15}.get(why, sum(new))
    q, k, v = _rows(n, seed=6)
    o, lse = c.step(q, k, v, _i32(new))
    start = np.concatenate([[0], np.cumsum(new)])
    rows = torch.zeros(n, dtype=torch.bool, device="cuda")
    rows[start[turned]:start[turned + 1]] = True
    assert bool((o[rows] == 0).all()) and bool((lse[:, rows] == -float("inf")).all()) and int(rows.sum()) > 0
    assert c.lens.tolist() == [x + (0 if r == turned else y) for r, (x, y) in enumerate(zip([9, 20, 3], new))]
    served = [0 if r == turned else x for r, x in enumerate(new)]
    want, want_lse = twin.step(*(x[~rows].contiguous() for x in (q, k, v)), _i32(served))
    # the same rows, shared out among the warps otherwise: two results, each off by the tolerances of test_gpu_packed_attn at most, with |v| <= 8,
    # sum |q k| * scale <= 16 and |lse| <= 7: 2 (2^-8 |o| + (2^-11 + 2^-22 + 2^-13) 8) and 2 (64 * 2^-24 * 16 + 2^-20 * 8)
    assert bool(o[~rows].double().sub(want.double()).abs().max() <= 2.0 ** -7 * want.double().abs().max() + 16 * (2.0 ** -11 + 2.0 ** -22 + 2.0 ** -13))
    assert bool((lse[:, ~rows] - want_lse).abs().max() <= 2.0 ** -13 + 2.0 ** -16)
    assert bool(torch.isfinite(lse[:, ~rows]).all())


def test_key_lengths():
    """lens_out, 0 for the sequences that are turned away; one without new rows never is."""
    from paper_2506_19651_b200 import binding as pb
    g, seqs = pb.make_pages(6, 16, 7, 3), 7
    lens, new = _i32([5, 16, 40, 0, 33, 48, 20]), _i32([3, 20, 9, 0, 1, 0, 2])
    for n, want in ((64, [8, 36, 0, 0, 34, 48, 22]), (23, [8, 36, 0, 0, 0, 48, 0])):
        out, key = _i32([-9] * seqs), _i32([-9] * seqs)
        pb.pevlm_pages_assign_rows(g, lens, new, _i32(np.zeros((seqs, 3))), _i32(range(6)), _i32([6]), out, _i32([0]), _i32([0] * 8), _i32([0] * 64), _i32([0] * 64),
                                   64, n, key)
        assert key.tolist() == want
        assert out.tolist() == [w or x for w, x in zip(want, lens.tolist())]


@pytest.mark.parametrize("new", [[3, 5, 0], [0, 5, 9], [-2, 8, 1], [2 ** 31 - 1, 4, 2 ** 31 - 1]])
def test_new_lengths_may_be_gone_by_the_time_the_rows_come(new):
    """extend() has read them: a store() of fewer rows goes by what it kept."""
    from paper_2506_19651_b200.layer import PackedCache
    make = lambda: PackedCache(3, 64, 12, 16, 40, 4, 2, 64, 1e4)
    c, twin = make(), make()
    first, rows = _rows(12, (2, 2), 7), _rows(8, (2, 2), 8)
    for x in (c, twin):
        x.extend(_i32([4, 4, 4]), rows=12)
        x.store(*first)
    lens = _i32(new)
    c.extend(lens)
    lens.zero_()
    c.store(*rows)
    twin.extend(_i32(new), rows=8)
    twin.store(*rows)
    for name in ("lens", "free_count", "slots", "positions"):
        assert getattr(c, name).tolist() == getattr(twin, name).tolist(), name
    # of the sequences that have rows in the step (starts past 2^31 are cut off, so that those behind have no rows at all in one of them)
    has = [start < 8 for start in c.row_start.tolist()[:3]]
    for name in ("row_start", "_key_lens"):
        assert [x for x, h in zip(getattr(c, name).tolist(), has) if h] == [x for x, h in zip(getattr(twin, name).tolist(), has) if h], name
