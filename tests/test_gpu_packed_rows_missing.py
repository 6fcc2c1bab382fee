"""Attention over the packed cache of fewer rows than row_start speaks of: a sequence whose rows are not all there sees no key (where
its rows stand could only be guessed), the others are served as ever."""
import pytest

from test_gpu_packed_attn import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [0, 1, 5, 68, 70, 75])
@pytest.mark.parametrize("rows", [[2, 3, 70], [2, 66, 7], [1, 4, 70]])
@pytest.mark.parametrize("window,sink", [(0, 0), (40, 5)])
def test_rows_that_are_not_all_there(rows, n, window, sink):
    import torch
    c = Case([300, 90, 200], rows, 4, 2, 64, 16, window=window, sink=sink, seed=11)
    full, lse_full = c.run()
    c.check(full, lse_full)
    pb, total = c.pb, sum(rows)
    o, lse = torch.full((total, 4, 64), -7.0, dtype=torch.bfloat16, device="cuda"), torch.full((4, max(n, 1)), -7.0, device="cuda")
    for most in {min(n, 1), min(n, 5), n}:
        ws = torch.empty(pb.pevlm_packed_workspace_bytes(c.shape, c.pages, n, most), dtype=torch.uint8, device="cuda")
        o.fill_(-7.0)
        pb.pevlm_packed_attn(c.shape, c.pages, window, c.q, c.cache, c.table, c.d_lens, c.start, n, most, o, lse, ws)
        assert bool((o[n:] == -7).all())
        row = 0
        for r in rows:
            here = slice(row, min(row + r, n))
            if row + r <= n:  # two results, each off by the tolerances of test_gpu_packed_attn at most: |v| <= 8, sum |q k| * scale <= 16, |lse| <= 9
                assert bool((o[here].double() - full[here].double()).abs().max() <= 2.0 ** -7 * full[here].double().abs().max() + 16 * (2.0 ** -11 + 2.0 ** -22 + 2.0 ** -13))
                assert bool((lse[:, here] - lse_full[:, here]).abs().max() <= 2 * (2.0 ** -14 + 2.0 ** -20 * 10))
            elif row < n:
                assert bool((o[here] == 0).all()) and bool((lse[:, here] == -float("inf")).all())
            row += r
