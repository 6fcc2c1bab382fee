"""Rows to the packed cache and back: every byte and every value equal to the format's description."""
import numpy as np
import pytest

import packed_reference as R
from helpers import GuardedAllocator, bits_to_f64, to_bits

pytestmark = pytest.mark.gpu


def _bf16(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(torch.bfloat16)


def _values(t):
    return bits_to_f64(to_bits(t)).reshape(t.shape)


def _hard_rows(rng, rows, Hkv, d):
    """N(0, 1) and, by rows, everything that rounds at an edge: exact halfway points of codes and scales, groups of zeros, subnormal and
    huge magnitudes, one large value among small ones, negative zeros."""
    x = rng.standard_normal((rows, Hkv, d)).astype(np.float32)
    for r in range(rows):
        k = r % 9
        if k == 1:  # codes halfway between two magnitudes, at a scale that is exact
            s = 2.0 ** rng.integers(-6, 6) * rng.choice([8, 9, 11, 15]) / 8
            x[r] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], (Hkv, d)) * s * rng.choice([-1, 1], (Hkv, d))
            x[r, :, ::16] = 6 * s
        elif k == 2:  # the group's largest is 6 times a number halfway between two scales
            x[r, :, ::16] = 6 * rng.choice([17, 19, 21, 31], (Hkv, d // 16)) / 16 * 2.0 ** rng.integers(-5, 5)
        elif k == 3:
            x[r] = 0.0
            x[r, 0, 3] = -0.0
        elif k == 4:
            x[r] *= 2.0 ** rng.integers(-40, -5)
        elif k == 5:
            x[r] *= 2.0 ** rng.integers(8, 60)
        elif k == 6:
            x[r, :, ::16] *= 300
        elif k == 7:  # at the ends of the scales
            x[r] *= rng.choice([2.0 ** -9, 2.0 ** -10, 448 * 6 / 3, 448.0])
    return x


@pytest.mark.parametrize("rows,Hkv,d,P,fused", [(1, 1, 64, 16, False), (1, 4, 128, 64, True), (37, 2, 128, 16, True), (333, 4, 128, 64, False),
                                                (1000, 8, 64, 32, True), (777, 3, 64, 128, False), (130, 1, 128, 128, True)])
def test_store_then_load(rows, Hkv, d, P, fused):
    import torch
    from paper_2506_19651_b200 import binding as pb
    rng = np.random.default_rng(rows + d)
    s = pb.make_shape(0, 1, 0, 1, Hkv, Hkv, d)
    pages = -(-rows // P) + 2
    g = pb.make_pages(pages, P, 1, pages)
    if fused:
        kv = _bf16(rng.standard_normal((rows, 2 * Hkv + 1, d)))
        kv[:, :Hkv], kv[:, Hkv:2 * Hkv] = _bf16(_hard_rows(rng, rows, Hkv, d)), _bf16(_hard_rows(rng, rows, Hkv, d))
        k, v = kv[:, :Hkv], kv[:, Hkv:2 * Hkv]
    else:
        k, v = _bf16(_hard_rows(rng, rows, Hkv, d)), _bf16(_hard_rows(rng, rows, Hkv, d))
    slots = rng.permutation(pages * P)[:rows].astype(np.int32)
    if rows > 4:
        slots[:5] = -1, 0, 5, pages * P, 9   # padding, and one past the end
        slots[5:rows // 2] = np.arange(5, rows // 2) + 7  # a run in order
        slots[rows // 2:] = rng.permutation(np.arange(rows // 2 + 7, pages * P))[:rows - rows // 2]
    d_slots = torch.from_numpy(slots).cuda()
    guard = GuardedAllocator()
    assert pb.pevlm_packed_cache_bytes(s, g) == pages * Hkv * P // 16 * 18 * d
    cache = guard((pages, Hkv, P // 16, 18 * d), torch.uint8)
    cache.fill_(0xEE)
    pb.pevlm_packed_store(s, g, k, v, d_slots, rows, cache, k.stride(0), v.stride(0))
    ok = (slots >= 0) & (slots < pages * P)
    want = np.full((pages, Hkv, P // 16, 18 * d), 0xEE, np.uint8)
    (kc, ks), (vc, vs) = R.quantise(_values(k)), R.quantise(_values(v))
    # tiles of what was written, with a mask of the bytes that belong to it
    ones = np.ones((16, d), np.int64)
    tiles = {}
    for r in np.nonzero(ok)[0]:
        tiles.setdefault(slots[r] // 16, []).append(r)
    for tile, members in tiles.items():
        page, t = tile * 16 // P, tile * 16 % P // 16
        for h in range(Hkv):
            parts, there = [np.zeros((16, d), np.int64), np.zeros((16, d), np.int64), np.zeros((16, d // 16), np.int64), np.zeros((16, d // 16), np.int64)], np.zeros((16, 1), np.int64)
            for r in members:
                u = slots[r] % 16
                there[u] = 1
                for part, src in zip(parts, (kc, vc, ks, vs)):
                    part[u] = src[r, h]
            mask = R.pack(there * 15 * ones, there * 15 * ones, there * 255 * np.ones((16, d // 16), np.int64), there * 255 * np.ones((16, d // 16), np.int64))
            w = want[page, h, t]
            w[:] = np.where(mask != 0, R.pack(*parts), w)
    got = cache.cpu().numpy()
    codes = np.arange(18 * d) < 16 * d
    for half in (0x0F, 0xF0):  # the sign of a zero is not part of the format
        for a in (got, want):
            a[codes & ((a & half) == (half & 0x88))] &= 0xFF ^ half
    assert np.array_equal(got, want)
    n = rows + 3
    again = np.concatenate([slots, [-5, 2 ** 31 - 1, slots[-1]]]).astype(np.int32)
    k_out, v_out = guard((n, Hkv, d), torch.bfloat16), guard((n, Hkv, d), torch.bfloat16)
    pb.pevlm_packed_load(s, g, cache, torch.from_numpy(again).cuda(), n, k_out, v_out)
    for x, codes, scales in ((k_out, kc, ks), (v_out, vc, vs)):
        y = np.where(ok[:, None, None], R.dequantise(codes, scales), 0.0)
        y = np.concatenate([y, np.zeros((2, Hkv, d)), y[-1:]])
        assert np.array_equal(_values(x), y)
    guard.check()


def test_error_of_a_value_is_half_a_step():
    """Away from saturation a value is off by at most half the distance of its neighbours: 1/4 s below 2 s, 1/2 s below 4 s, s up to 6 s, and
    6 s itself is within 2^-4 of the largest magnitude (the rounding of its scale)."""
    import torch
    from paper_2506_19651_b200 import binding as pb
    rows, Hkv, d = 500, 2, 128
    s, g = pb.make_shape(0, 1, 0, 1, Hkv, Hkv, d), pb.make_pages(8, 64, 1, 8)
    torch.manual_seed(5)
    k = torch.randn((rows, Hkv, d), device="cuda").to(torch.bfloat16)
    v = torch.randn((rows, Hkv, d), device="cuda").to(torch.bfloat16) * 40
    cache = torch.zeros(pb.pevlm_packed_cache_bytes(s, g), dtype=torch.uint8, device="cuda")
    slots = torch.arange(rows, dtype=torch.int32, device="cuda")
    pb.pevlm_packed_store(s, g, k, v, slots, rows, cache)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    pb.pevlm_packed_load(s, g, cache, slots, rows, ko, vo)
    for x, y in ((k, ko), (v, vo)):
        x, y = x.double().unflatten(-1, (-1, 16)), y.double().unflatten(-1, (-1, 16))
        top = x.abs().amax(-1, keepdim=True)
        # the scale is within 2^-4 of top / 6; the widest step, from 4 s to 6 s, is 2 s
        assert bool(((x - y).abs() <= top / 6 * (1 + 2 ** -4) + 1e-30).all())
        assert bool(((x - y).abs() <= torch.where(x.abs() < top / 3 * (1 - 2 ** -4), top / 24 * (1 + 2 ** -4), top / 6 * (1 + 2 ** -4)) + 1e-30).all())


def test_infinities_and_nan_leave_numbers():
    """What is stored is finite whatever comes in, so a masked key can never reach an output."""
    import torch
    from paper_2506_19651_b200 import binding as pb
    s, g = pb.make_shape(0, 1, 0, 1, 1, 1, 64), pb.make_pages(1, 16, 1, 1)
    k = torch.full((16, 1, 64), float("nan"), device="cuda").to(torch.bfloat16)
    k[1::2] = float("inf")
    k[2, 0, 0] = -float("inf")
    cache = torch.zeros(pb.pevlm_packed_cache_bytes(s, g), dtype=torch.uint8, device="cuda")
    slots = torch.arange(16, dtype=torch.int32, device="cuda")
    pb.pevlm_packed_store(s, g, k, k, slots, 16, cache)
    ko, vo = torch.empty_like(k), torch.empty_like(k)
    pb.pevlm_packed_load(s, g, cache, slots, 16, ko, vo)
    assert bool(torch.isfinite(ko).all()) and bool(torch.isfinite(vo).all())


def test_the_same_slot_again_and_again():
    """One slot in every row that is read, and the last bytes of a cache that ends there."""
    import torch
    from paper_2506_19651_b200 import binding as pb
    s, g = pb.make_shape(0, 1, 0, 1, 2, 2, 128), pb.make_pages(3, 16, 1, 3)
    cache = GuardedAllocator()((3, 2, 1, 18 * 128), torch.uint8)
    cache.fill_(0)
    k, v = (torch.randn((48, 2, 128), device="cuda").to(torch.bfloat16) for _ in range(2))
    pb.pevlm_packed_store(s, g, k, v, torch.arange(48, dtype=torch.int32, device="cuda"), 48, cache)
    for slot in (0, 17, 47):
        once, many = ([torch.empty((n, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for n in (1, 5000))
        pb.pevlm_packed_load(s, g, cache, torch.tensor([slot], dtype=torch.int32, device="cuda"), 1, *once)
        pb.pevlm_packed_load(s, g, cache, torch.full((5000,), slot, dtype=torch.int32, device="cuda"), 5000, *many)
        for a, b in zip(once, many):
            assert bool((a == b).all())
        for a, x in zip(once, (k, v)):
            assert np.array_equal(_values(a)[0], R.dequantise(*R.quantise(_values(x[slot:slot + 1])))[0])
