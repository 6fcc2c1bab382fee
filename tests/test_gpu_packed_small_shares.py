"""One key that outweighs the others by far, whose values in turn are far larger than its own: what the many small probabilities add up to.

Tolerance: that of test_gpu_packed_attn, the probabilities' smallest step being 2^-32 of the reference here, and the term for it taken where it belongs: keys * 2^-32
max |v| / l, with l = sum p >= 1 counted from the largest score."""
import numpy as np
import pytest

import packed_reference as R
from test_gpu_packed_attn import Case, _bf16, _values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,Hq,Hkv,d", [(1, 7, 1, 128), (3, 14, 2, 128), (2, 8, 2, 64), (70, 7, 1, 128), (130, 4, 2, 64)])
@pytest.mark.parametrize("gap", [14.0, 17.5, 19.0])
def test_many_small_beside_one(rows, Hq, Hkv, d, gap):
    import torch
    L, first = 3000, 5
    c = Case([L], [rows], Hq, Hkv, d, 16, seed=2)
    rng = np.random.default_rng(3)
    table = c.table.cpu().numpy().astype(np.int64)
    k, v = np.zeros((L, Hkv, d)), rng.uniform(100, 500, (L, Hkv, d))
    k[first, :, 0] = 4.0
    v[first] = rng.standard_normal((Hkv, d))
    t = np.arange(L)
    slots = torch.from_numpy((table[0, t // 16] * 16 + t % 16).astype(np.int32)).cuda()
    kb, vb = _bf16(k), _bf16(v)
    c.pb.pevlm_packed_store(c.shape, c.pages, kb, vb, slots, L, c.cache)
    k, v = R.dequantise(*R.quantise(_values(kb))), R.dequantise(*R.quantise(_values(vb)))
    q = rng.standard_normal((rows, Hq, d))
    q[:, :, 0] = gap / 4.0 / c.scale * rng.uniform(0.95, 1.0, (rows, Hq))
    c.q = _bf16(q.reshape(rows, -1))
    qv = _values(c.q).reshape(rows, Hkv, Hq // Hkv, d)
    o, lse = c.run()
    s = np.einsum("nhgd,khd->nhgk", qv, k) * c.scale
    big = (np.einsum("nhgd,khd->nhgk", np.abs(qv), np.abs(k)) * c.scale).max()
    see = t <= (L - rows + np.arange(rows))[:, None]
    s = np.where(see[:, None, None], s, -np.inf)
    top = s.max(-1, keepdims=True)
    p = np.exp(s - top)
    l = p.sum(-1, keepdims=True)
    want, a = np.einsum("nhgk,khd->nhgd", p, v) / l, np.einsum("nhgk,khd->nhgd", p, np.abs(v)) / l
    score = 64 * 2.0 ** -24 * big
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -22 + 2 * score) * a + L * 2.0 ** -32 * np.abs(v).max() / l
    got = _values(o).reshape(want.shape)
    assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()
    z = (top + np.log(l))[..., 0].reshape(rows, Hq).T
    assert (np.abs(lse.double().cpu().numpy() - z) <= score + 2.0 ** -20 * (1 + np.abs(z))).all()
