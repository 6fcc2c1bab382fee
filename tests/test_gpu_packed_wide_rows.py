"""Rows of Q whose elements differ by many powers of two, against keys that are 0 where the large ones stand: the scores come from the small elements alone.

What fp16 holds of a row after the power of two is exact down to 2^-31 of its largest element, so the tolerances are those of test_gpu_packed_attn, whose S = sum |q k|
holds no part of the large elements."""
import numpy as np
import pytest

import packed_reference as R
from test_gpu_packed_attn import Case, _bf16, _values

pytestmark = pytest.mark.gpu


class WideCase(Case):
    """Keys whose first group of 16 elements is 0; rows of Q with `large` in that group and, in the others, numbers around `small`.  `wide` chooses the rows (of a
    sequence's rows), the others are as in Case."""

    def __init__(self, *args, large, small, k_scale=64.0, wide=lambda i: True, **kw):
        super().__init__(*args, k_scale=1.0, **kw)
        rng = np.random.default_rng(17)
        n, Hkv, d, P = len(self.lens), self.Hkv, self.d, self.P
        import torch
        table = self.table.cpu().numpy().astype(np.int64)
        for r in range(n):
            L = int(self.lens[r])
            k = rng.standard_normal((L, Hkv, d)) * k_scale
            k[..., :16] = 0
            k = _bf16(k)
            t = np.arange(L)
            slots = torch.from_numpy((table[r, t // P] * P + t % P).astype(np.int32)).cuda()
            v = _bf16(self.v[r])   # values of the cache: they stay what they are
            self.pb.pevlm_packed_store(self.shape, self.pages, k, v, slots, L, self.cache)
            self.k[r], self.v[r] = R.dequantise(*R.quantise(_values(k))), R.dequantise(*R.quantise(_values(v)))
        q = self.q_values.copy()
        row = 0
        for rows in self.rows:
            for i in range(rows):
                if wide(i):
                    x = rng.standard_normal((self.Hq, d)) * small
                    x[:, :16] = 0
                    x[np.arange(self.Hq), rng.integers(0, 16, self.Hq)] = large
                    q[row + i] = x
            row += rows
        width = self.q.shape[1]
        flat = np.zeros((max(self.n_rows, 1), width))
        flat[:self.used, :self.Hq * d] = q.reshape(self.used, -1)
        self.q = _bf16(flat)
        self.q_values = _values(self.q)[:self.used, :self.Hq * d].reshape(self.used, self.Hq, d)


FORMS = {"one token": ([400], [1], 7, 1, 128), "16 rows": ([300, 90], [4, 3], 14, 2, 128), "heads of 64": ([260, 100], [1, 2], 8, 2, 64),
         "a question": ([700, 200], [64, 60], 7, 1, 128), "a question, heads of 64": ([500], [130], 4, 2, 64)}


@pytest.mark.parametrize("ratio", [2.0 ** -10, 2.0 ** -16, 2.0 ** -20, 2.0 ** -24])
@pytest.mark.parametrize("form", FORMS)
def test_small_elements_beside_a_large_one(form, ratio):
    """Down to seven powers of two below the ratio (numbers that normal variates leave aside in all but 1 of 128 cases) the rows are exact."""
    lens, rows, Hq, Hkv, d = FORMS[form]
    large = 2.0 ** -8 / ratio
    c = WideCase(lens, rows, Hq, Hkv, d, 16, large=large, small=2.0 ** -8, seed=3)
    c.check(*c.run())


@pytest.mark.parametrize("form", ["16 rows", "a question"])
def test_large_keys_beside_a_large_element(form):
    """1024 beside elements of 2^-10 * 129/128 whose keys are 2688: a score of 26.19, of which 0.2 would be lost if fp16 did not hold the small ones."""
    lens, rows, Hq, Hkv, d = FORMS[form]
    c = WideCase(lens, rows, Hq, Hkv, d, 16, large=1024.0, small=0.0, k_scale=0.0, seed=3)
    import torch
    q = _values(c.q)
    q = q[:, :Hq * d].reshape(-1, Hq, d)
    q[..., 16:] = 2.0 ** -10 * 129 / 128
    c.q = _bf16(q.reshape(len(q), -1))
    c.q_values = _values(c.q)[:c.used].reshape(c.used, Hq, d)
    table = c.table.cpu().numpy().astype(np.int64)
    for r, L in enumerate(c.lens):
        k = np.zeros((L, Hkv, d))
        k[1::2, :, 16:] = 2688
        t = np.arange(L)
        slots = torch.from_numpy((table[r, t // 16] * 16 + t % 16).astype(np.int32)).cuda()
        c.pb.pevlm_packed_store(c.shape, c.pages, _bf16(k), _bf16(c.v[r]), slots, L, c.cache)
        c.k[r] = k
    c.check(*c.run())


@pytest.mark.parametrize("where", ["first", "last", "second half", "every third"])
def test_wide_rows_beside_others(where):
    """In a pair of row tiles some rows are wide and some are not."""
    wide = {"first": lambda i: i == 0, "last": lambda i: i == 89, "second half": lambda i: i >= 45, "every third": lambda i: i % 3 == 0}[where]
    c = WideCase([500], [90], 4, 1, 128, 32, large=2.0 ** 12, small=2.0 ** -8, wide=wide, k_scale=8.0, seed=4)
    c.check(*c.run())


@pytest.mark.parametrize("rows", [2, 70])
@pytest.mark.parametrize("large,small,scale", [(2.0 ** 127, 2.0 ** 107, 2.0 ** -107), (1.9921875 * 2.0 ** 127, 2.0 ** 104, 2.0 ** -104), (2.0 ** -100, 2.0 ** -120, 2.0 ** 110),
                                               (2.0 ** -126, 2.0 ** -128, 2.0 ** 120), (0.0, 2.0 ** -130, 2.0 ** 120)])
def test_at_the_ends_of_bf16(rows, large, small, scale):
    """The largest and the smallest numbers there are; elements around 2^-130 are multiples of 2^-133."""
    c = WideCase([300], [rows], 4, 2, 64, 16, large=large, small=small, k_scale=1.0, scale=scale, seed=5)
    c.check(*c.run())


@pytest.mark.parametrize("rows", [1, 80])
def test_what_is_too_small_is_off_by_no_more_than_is_said(rows):
    """Elements 2^-36 times the largest: a score is off by 2^-39 max|q| * sum |k| * scale at most, which stands beside the derived tolerances here."""
    c = WideCase([300], [rows], 4, 2, 128, 16, large=2.0 ** 28, small=2.0 ** -8, k_scale=64.0, seed=6)
    o, lse = c.run()
    more = 2.0 ** -39 * 2.0 ** 28 * np.abs(c.k[0]).sum(-1).max() * c.scale
    q, k = c.q_values.reshape(rows, 2, 2, 128), c.k[0]
    s = np.einsum("nhgd,khd->nhgk", q, k) * c.scale
    pos = 300 - rows + np.arange(rows)
    s = np.where((np.arange(300) <= pos[:, None])[:, None, None], s, -np.inf)
    z = np.logaddexp.reduce(s, -1).reshape(rows, 4).T
    big = (np.einsum("nhgd,khd->nhgk", np.abs(q), np.abs(k)) * c.scale).max()
    assert more < 0.5
    assert (np.abs(lse.double().cpu().numpy() - z) <= more + 64 * 2.0 ** -24 * big + 2.0 ** -20 * (1 + np.abs(z))).all()
