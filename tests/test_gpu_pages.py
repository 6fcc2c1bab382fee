"""Page tables, slots and positions against a sequential allocator: every number equal."""
import numpy as np
import pytest

from packed_reference import Allocator

pytestmark = pytest.mark.gpu


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _state(rng, pages, P, seqs, most, lens):
    held = -(-lens // P)
    order = rng.permutation(pages)
    table = np.full((seqs, most), -1, np.int32)
    at = 0
    for r in range(seqs):
        table[r, :held[r]] = order[at:at + held[r]]
        at += held[r]
    free = np.full(pages, -7, np.int32)
    free[:pages - at] = order[at:]
    return table, free, pages - at


CASES = [  # pages, page_len, sequences, max_pages, longest held, most new, capacity for rows (None = exactly the new ones)
    (1, 16, 1, 1, 0, 1, None), (4, 16, 1, 4, 15, 40, None), (64, 16, 7, 20, 60, 5, 64), (3000, 16, 300, 40, 100, 200, 70000),
    (900, 128, 1024, 3, 128, 100, None), (4000, 64, 1025, 9, 300, 1, 2048), (9000, 32, 2500, 12, 90, 64, 100001),
    (30, 16, 40, 8, 16, 33, None), (50, 32, 9, 2, 64, 64, None), (500, 16, 30, 40, 200, 300, 1000), (20000, 16, 3, 7000, 0, 100000, 300003),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_release_then_assign(case):
    import torch
    from paper_2506_19651_b200 import binding as pb
    pages, P, seqs, most, longest, new_most, room = case
    rng = np.random.default_rng(hash(case[:6]) % 1000)
    lens = np.minimum(rng.integers(0, longest + 1, seqs), most * P)
    while (-(-lens // P)).sum() > pages:
        lens //= 2
    table, free, count = _state(rng, pages, P, seqs, most, lens)
    finished = (rng.random(seqs) < 0.2) * rng.integers(1, 5, seqs)
    new = rng.integers(0, new_most + 1, seqs) * (rng.random(seqs) < 0.9)
    max_rows = int(new.sum()) if room is None else room
    g = pb.make_pages(pages, P, seqs, most)
    ref = Allocator(pages, P, seqs, most)
    want_lens, want_free, want_count = ref.release(finished, lens, table, free, count)
    d_table, d_free = _dev(table), _dev(free)
    lens_a, lens_b, count_a, count_b = _dev(lens), _dev(np.zeros(seqs)), _dev([count]), _dev([-1])
    pb.pevlm_pages_release(g, _dev(finished), lens_a, d_table, d_free, count_a, lens_b, count_b)
    assert np.array_equal(lens_b.cpu().numpy(), want_lens) and int(count_b) == want_count
    assert np.array_equal(d_free.cpu().numpy(), want_free) and np.array_equal(d_table.cpu().numpy(), table)
    guard = 64
    slots, positions = (torch.full((max_rows + guard,), -99, dtype=torch.int32, device="cuda") for _ in range(2))
    start = torch.full((seqs + 1 + guard,), -99, dtype=torch.int32, device="cuda")
    pb.pevlm_pages_assign(g, lens_b, _dev(new), d_table, d_free, count_b, lens_a, count_a, start, slots, positions, max_rows)
    w_lens, w_table, w_count, w_start, w_slots, w_positions = ref.assign(want_lens, new, table, want_free, want_count, max_rows)
    assert np.array_equal(start.cpu().numpy()[:seqs + 1], w_start)
    assert np.array_equal(lens_a.cpu().numpy(), w_lens) and int(count_a) == w_count
    assert np.array_equal(d_table.cpu().numpy(), w_table)
    assert np.array_equal(slots.cpu().numpy()[:max_rows], w_slots)
    assert np.array_equal(positions.cpu().numpy()[:max_rows], w_positions)
    assert np.array_equal(d_free.cpu().numpy(), want_free)
    for t, n in ((slots, max_rows), (positions, max_rows), (start, seqs + 1)):
        assert bool((t[n:] == -99).all())


def test_numbers_out_of_range_stay_in_bounds():
    """Negative new lengths count as 0, lengths past the table and counts past the list as the nearest in range, and a list that holds no page hands out none."""
    import torch
    from paper_2506_19651_b200 import binding as pb
    g = pb.make_pages(8, 16, 4, 2)
    lens, out = _dev([-5, 1000, 31, 0]), _dev([0] * 4)
    table = _dev([[0, 1], [2, 3], [4, 5], [6, 7]])
    free, count, count_out = _dev([-1, 99, 5, 6, 7, 0, 1, 2]), _dev([1000]), _dev([0])
    start, slots, positions = _dev([0] * 5), _dev([0] * 8), _dev([0] * 8)
    pb.pevlm_pages_assign(g, lens, _dev([-3, 1, 1, 2]), table, free, count, out, count_out, start, slots, positions, 8)
    assert out.tolist() == [0, 32, 32, 2] and start.tolist() == [0, 0, 1, 2, 4]
    assert slots.tolist() == [-1, 5 * 16 + 15, 2 * 16, 2 * 16 + 1, -1, -1, -1, -1]
    assert positions.tolist() == [32, 31, 0, 1, 0, 0, 0, 0] and int(count_out) == 7
    pb.pevlm_pages_assign(g, _dev([0] * 4), _dev([0, 0, 0, 3]), table, free, _dev([2]), out, count_out, start, slots, positions, 8)
    assert slots.tolist()[:3] == [-1, -1, -1] and int(count_out) == 1   # page 99 is none
    pb.pevlm_pages_release(g, _dev([1, 1, 1, 1]), _dev([32, 32, 32, 32]), table, free, _dev([5]), out, count_out)
    assert int(count_out) == 8 and out.tolist() == [0] * 4


def test_replayed_step_and_another_stream():
    """A step captured with release then assign between two sets of buffers runs on at each replay, on the stream it is replayed on."""
    import torch
    from paper_2506_19651_b200 import binding as pb
    P, seqs, most = 16, 5, 8
    pages = seqs * most
    g = pb.make_pages(pages, P, seqs, most)
    ref = Allocator(pages, P, seqs, most)
    lens = np.array([3, 0, 16, 31, 7])
    table, free, count = _state(np.random.default_rng(3), pages, P, seqs, most, lens)
    d_lens, mid, d_count, count_mid = _dev(lens), _dev([0] * 5), _dev([count]), _dev([0])
    d_table, d_free, fin, new = _dev(table), _dev(free), _dev([0] * 5), _dev([1, 2, 1, 3, 17])
    start, slots, positions = _dev([0] * 6), _dev([0] * 32), _dev([0] * 32)

    def step():
        pb.pevlm_pages_release(g, fin, d_lens, d_table, d_free, d_count, mid, count_mid)
        pb.pevlm_pages_assign(g, mid, new, d_table, d_free, count_mid, d_lens, d_count, start, slots, positions, 32)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    for finished in ([0] * 5, [0, 0, 1, 0, 1], [1, 0, 0, 0, 0]):
        fin.copy_(_dev(finished))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        lens, free, count = ref.release(np.array(finished), lens, table, free, count)
        lens, table, count, w_start, w_slots, w_positions = ref.assign(lens, new.cpu().numpy(), table, free, count, 32)
        assert np.array_equal(slots.cpu().numpy(), w_slots) and np.array_equal(positions.cpu().numpy(), w_positions)
        assert np.array_equal(d_lens.cpu().numpy(), lens) and int(d_count) == count and np.array_equal(start.cpu().numpy(), w_start)
        assert np.array_equal(d_table.cpu().numpy(), table) and np.array_equal(d_free.cpu().numpy()[:count], free[:count])
