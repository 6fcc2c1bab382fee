"""Scores so large that fp32 keeps no more than whole numbers of them, or not even those: the derived tolerance of test_gpu_packed_attn (twice 64 * 2^-24 of the sum of the
products' magnitudes) allows any weights then, but outputs stay means of the values and numbers throughout."""
import numpy as np
import pytest

from test_gpu_packed_attn import Case, _values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [2.0 ** 10, 2.0 ** 18, 2.0 ** 20, 2.0 ** 21, 2.0 ** 22, 2.0 ** 23])
@pytest.mark.parametrize("lens,rows,Hq,Hkv,d", [([700, 90], [1, 2], 7, 1, 128), ([300], [4], 8, 2, 64), ([900, 300], [64, 60], 7, 1, 128), ([1000], [130], 4, 2, 64)])
def test_numbers_all_the_same(lens, rows, Hq, Hkv, d, scale):
    import torch
    for seed in range(3):
        c = Case(lens, rows, Hq, Hkv, d, 16, scale=scale, seed=seed)
        o, lse = c.run()
        assert bool(torch.isfinite(o[:c.used]).all()) and bool(torch.isfinite(lse[:, :c.used]).all())
        most = max(np.abs(v).max() for v in c.v)
        assert float(o[:c.used].abs().max()) <= most * (1 + 2.0 ** -7)
        c.check(o, lse)
