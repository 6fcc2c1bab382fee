"""What each single key adds to an output of the attention over the packed cache.

V is 0 but for one key a column of the head, whose value is 2688 (6 times the largest scale: stored exactly): column c of the output is p_j / l * 2688 of its key j, so a
tile, a share of a warp or of a CTA that is lost, taken twice or joined wrongly shows in its own column.  Tolerance: 2^-8 of the output for bf16, 2^-11 + 2^-22 and twice the score's error
(64 * 2^-24 sum |q k| * scale) for the probability, which with one key a column are all relative to the output, and 2^-32 * 2688 / l for the smallest probabilities."""
import numpy as np
import pytest

import packed_reference as R
from test_gpu_packed_attn import Case, _bf16, _values, visible

pytestmark = pytest.mark.gpu


def _expected(q, k, keys, pos, scale, window, sink):
    """q [n, Hkv, G, d], k [L, Hkv, d], keys [Hkv, d]: the share of each column's key, 2688 times, with its tolerance; log-sum-exp with its."""
    s = np.einsum("nhgd,khd->nhgk", q, k) * scale
    score = 64 * 2.0 ** -24 * (np.einsum("nhgd,khd->nhgk", np.abs(q), np.abs(k)) * scale).max()
    see = visible(pos[:, None], np.arange(k.shape[0]), window, sink)
    s = np.where(see[:, None, None], s, -np.inf)
    top = s.max(-1, keepdims=True)
    p = np.exp(s - top)
    l = p.sum(-1, keepdims=True)
    z = (top + np.log(l))[..., 0]
    want = 2688 * np.take_along_axis(p, np.broadcast_to(keys[None, :, None], q.shape), -1) / l
    return want, (2.0 ** -8 + 2.0 ** -11 + 2.0 ** -22 + 2 * score) * want + 2.0 ** -32 * 2688 / l, z, score + 2.0 ** -20 * (1 + np.abs(z))


def _planted(keys, L):
    """V [L, Hkv, d] of those keys."""
    v = np.zeros((L, *keys.shape))
    h, c = np.indices(keys.shape)
    v[keys, h, c] = 2688.0
    return v


FORMS = {  # keys, rows, heads, window and sink
    "a token": (9001, 1, 28, 4, 128, 0, 0), "a token, heads of 64": (12000, 1, 8, 2, 64, 0, 0), "drafted tokens": (5003, 4, 32, 8, 64, 0, 0), "17 rows a head": (4000, 17, 4, 4, 128, 0, 0),
    "a question": (9000, 64, 28, 4, 128, 0, 0), "a question, heads of 64": (7000, 100, 8, 2, 64, 0, 0), "a long question": (3001, 300, 7, 1, 128, 0, 0),
    "a token under a window": (9001, 1, 28, 4, 128, 3000, 64), "a question under a window": (9000, 130, 4, 2, 128, 2500, 200)}


@pytest.mark.parametrize("form", FORMS)
def test_every_tile_of_a_long_cache(form):
    import torch
    L, rows, Hq, Hkv, d, window, sink = FORMS[form]
    c = Case([L], [rows], Hq, Hkv, d, 16, window=window, sink=sink, seed=len(form))
    table = c.table.cpu().numpy().astype(np.int64)
    t = np.arange(L)
    slots = torch.from_numpy((table[0, t // 16] * 16 + t % 16).astype(np.int32)).cuda()
    k = _bf16(c.k[0])
    rng = np.random.default_rng(1)
    # a key of every tile of 16 that some row sees, the tiles' ends among them, and in each head others
    tiles = np.arange(-(-L // 16))
    low = L - rows - window + 1
    if window:
        tiles = tiles[(tiles * 16 < sink) | (tiles * 16 + 15 >= low)]
    rounds = -(-len(tiles) // d)
    q = c.q_values.reshape(rows, Hkv, Hq // Hkv, d)
    pos = L - rows + np.arange(rows)
    for i in range(rounds):
        keys = np.empty((Hkv, d), np.int64)
        for h in range(Hkv):
            mine = np.roll(tiles, -i * d - 7 * h)[:d]
            keys[h] = np.resize(mine, d) * 16 + rng.choice([0, 1, 7, 8, 15], d)
        keys = np.minimum(keys, L - 1)
        keys[:, -1], keys[:, -2] = L - 1, 0
        v = _planted(keys, L)
        c.pb.pevlm_packed_store(c.shape, c.pages, k, _bf16(v), slots, L, c.cache)
        c.k[0] = R.dequantise(*R.quantise(_values(k)))  # (the values of the cache, quantised once more)
        o, lse = c.run()
        want, tol, z, z_tol = _expected(q, c.k[0], keys, pos, c.scale, window, sink)
        got = _values(o).reshape(want.shape)
        over = np.abs(got - want) - tol
        at = np.unravel_index(over.argmax(), over.shape)
        assert over.max() <= 0, (at, got[at], want[at], tol[at])
        assert (np.abs(lse.double().cpu().numpy().T.reshape(z.shape) - z) <= z_tol).all()


def test_keys_of_many_sequences():
    """Sequences of very different lengths, whose units begin and end anywhere in the warps' parts: 40 keys of each, of their own values."""
    import torch
    lens, rows = [(i * 577) % 2500 + 30 for i in range(40)], [1 + i % 2 for i in range(40)]
    Hq, Hkv, d = 8, 2, 128
    c = Case(lens, rows, Hq, Hkv, d, 32, seed=8)
    table = c.table.cpu().numpy().astype(np.int64)
    rng = np.random.default_rng(2)
    all_keys = []
    for r, L in enumerate(lens):
        keys = np.sort(rng.integers(0, L, (Hkv, d)), -1)
        keys[:, -1] = L - 1
        all_keys.append(keys)
        t = np.arange(L)
        slots = torch.from_numpy((table[r, t // 32] * 32 + t % 32).astype(np.int32)).cuda()
        k = _bf16(c.k[r])
        c.pb.pevlm_packed_store(c.shape, c.pages, k, _bf16(_planted(keys, L)), slots, L, c.cache)
        c.k[r] = R.dequantise(*R.quantise(_values(k)))
    o, lse = c.run()
    o, row = _values(o), 0
    for r, (L, n) in enumerate(zip(lens, rows)):
        q = c.q_values[row:row + n].reshape(n, Hkv, Hq // Hkv, d)
        want, tol, z, z_tol = _expected(q, c.k[r], all_keys[r], L - n + np.arange(n), c.scale, 0, 0)
        assert (np.abs(o[row:row + n].reshape(want.shape) - want) <= tol).all(), r
        assert (np.abs(lse.double().cpu().numpy()[:, row:row + n].T.reshape(z.shape) - z) <= z_tol).all()
        row += n


@pytest.mark.parametrize("rows", [1, 50])
def test_keys_of_a_resident_video(rows):
    """A video stored through PackedCache, then a step: every tile of 16 of its keys."""
    import torch
    from paper_2506_19651_b200.layer import PackedCache
    L, Hq, Hkv, d, P = 4000, 14, 2, 128, 64
    cache = PackedCache(3, 8192, 200, P, L, Hq, Hkv, d, 1e6)
    rng = np.random.default_rng(4)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    cache.extend(i32([0, 700, 0]), rows=700)  # another video first
    cache.store(*(_bf16(rng.standard_normal((700, Hkv, d))) for _ in range(2)))
    tiles = np.arange(L // 16)
    keys = np.stack([rng.permutation(tiles)[:d] * 16 + rng.integers(0, 16, d) for _ in range(Hkv)])
    cache.extend(i32([0, 0, L]), rows=L)
    cache.store(_bf16(rng.standard_normal((L, Hkv, d))), _bf16(_planted(keys, L)))
    q, k = _bf16(rng.standard_normal((rows, Hq, d))), _bf16(rng.standard_normal((rows, Hkv, d)))
    o, lse = cache.step(q, k, torch.zeros_like(k), i32([0, 0, rows]))
    total = L + rows
    t = np.arange(total)
    slots = cache.page_table[2].cpu().numpy().astype(np.int64)[t // P] * P + t % P
    kk, vv = cache.load(i32(slots.tolist()))
    assert np.array_equal(_values(vv)[:L], _planted(keys, L)) and bool((vv[L:] == 0).all())
    roped = torch.empty_like(q)
    from paper_2506_19651_b200 import binding as pb
    pb.pevlm_rope_qk(cache.shape, q, k, roped, torch.empty_like(k), L, rows, None)
    want, tol, z, z_tol = _expected(_values(roped).reshape(rows, Hkv, Hq // Hkv, d), _values(kk), keys, L + np.arange(rows), d ** -0.5, 0, 0)
    assert (np.abs(_values(o).reshape(want.shape) - want) <= tol).all()
    assert (np.abs(lse.double().cpu().numpy().T.reshape(z.shape) - z) <= z_tol).all()


@pytest.mark.parametrize("lens,rows,Hq,Hkv,d", [([9001], [1], 28, 4, 128), ([12000, 3, 700, 5000], [1, 1, 2, 1], 8, 2, 64), ([9000], [64], 28, 4, 128), ([5000, 2100], [130, 3], 4, 2, 64)])
def test_random_values_of_a_long_cache(lens, rows, Hq, Hkv, d):
    """As test_gpu_packed_attn, its term for the smallest probabilities divided by the row's sum l, which for long caches is some hundred."""
    c = Case(lens, rows, Hq, Hkv, d, 32, seed=12)
    o, lse = c.run()
    c.check(o, lse)
    o, row = _values(o), 0
    for r, (L, n) in enumerate(zip(lens, rows)):
        q = c.q_values[row:row + n].reshape(n, Hkv, Hq // Hkv, d)
        s = np.einsum("nhgd,khd->nhgk", q, c.k[r]) * c.scale
        score = 64 * 2.0 ** -24 * (np.einsum("nhgd,khd->nhgk", np.abs(q), np.abs(c.k[r])) * c.scale).max()
        see = np.arange(L) <= (L - n + np.arange(n))[:, None]
        s = np.where(see[:, None, None], s, -np.inf)
        p = np.exp(s - s.max(-1, keepdims=True))
        l = p.sum(-1, keepdims=True)
        want, a = np.einsum("nhgk,khd->nhgd", p, c.v[r]) / l, np.einsum("nhgk,khd->nhgd", p, np.abs(c.v[r])) / l
        tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -22 + 2 * score) * a + L * 2.0 ** -32 * np.abs(c.v[r]).max() / l
        assert (np.abs(o[row:row + n].reshape(want.shape) - want) <= tol).all(), r
        row += n
