"""The calls on pages and on the packed cache refuse bad arguments on the host, before anything is launched (no GPU here)."""
import ctypes as C

import numpy as np
import pytest

import packed_reference as R
from paper_2506_19651_b200 import binding as pb
from paper_2506_19651_b200 import build as pbuild


@pytest.fixture(scope="module")
def lib():
    pbuild.build()
    return pb.lib()


def at(x):
    return C.c_void_p(x)


BAD_PAGES = [((0, 16, 1, 1), pb.PEVLM_EINVAL), ((4, 16, 0, 1), pb.PEVLM_EINVAL), ((4, 16, 1, 0), pb.PEVLM_EINVAL), ((4, 0, 1, 1), pb.PEVLM_EUNSUPPORTED),
             ((4, 48, 1, 1), pb.PEVLM_EUNSUPPORTED), ((4, 256, 1, 1), pb.PEVLM_EUNSUPPORTED), ((2 ** 27, 16, 1, 1), pb.PEVLM_EINVAL),
             ((4, 128, 1, 2 ** 23 + 1), pb.PEVLM_EINVAL), ((4, 16, 2 ** 20 + 1, 1), pb.PEVLM_EINVAL)]


def test_pages(lib):
    g = pb.make_pages(8, 16, 4, 2)
    p = [at(4096 * (i + 1)) for i in range(12)]
    release = [p[0], p[1], p[2], p[3], p[4], p[5], p[6]]
    assign = [p[0], p[1], p[2], p[3], p[4], p[5], p[6], p[7], p[8], p[9]]
    for fields, code in BAD_PAGES:
        bad = pb.make_pages(*fields)
        assert lib.pevlm_pages_release(C.byref(bad), *release, None) == code, fields
        assert lib.pevlm_pages_assign(C.byref(bad), *assign, 8, None) == code, fields
    assert lib.pevlm_pages_release(None, *release, None) == pb.PEVLM_EINVAL
    for i in range(7):
        a = list(release); a[i] = None
        assert lib.pevlm_pages_release(C.byref(g), *a, None) == pb.PEVLM_EINVAL
        a[i] = at(4098)
        assert lib.pevlm_pages_release(C.byref(g), *a, None) == pb.PEVLM_EALIGN
    for i in range(10):
        a = list(assign); a[i] = None
        assert lib.pevlm_pages_assign(C.byref(g), *a, 8, None) == pb.PEVLM_EINVAL
        a[i] = at(4098)
        assert lib.pevlm_pages_assign(C.byref(g), *a, 8, None) == pb.PEVLM_EALIGN
    for i in (8, 9):  # written 16 bytes at a time
        a = list(assign); a[i] = at(4100)
        assert lib.pevlm_pages_assign(C.byref(g), *a, 8, None) == pb.PEVLM_EALIGN
    # outputs that are inputs
    a = list(release); a[5] = a[1]
    assert lib.pevlm_pages_release(C.byref(g), *a, None) == pb.PEVLM_EINVAL
    a = list(release); a[6] = a[4]
    assert lib.pevlm_pages_release(C.byref(g), *a, None) == pb.PEVLM_EINVAL
    for out, src in ((5, 0), (5, 1), (6, 4)):
        a = list(assign); a[out] = a[src]
        assert lib.pevlm_pages_assign(C.byref(g), *a, 8, None) == pb.PEVLM_EINVAL
    for i, other in ((5, 4096 + 12), (7, 4096 + 12), (5, 8192 - 12), (8, 4096), (9, 8192)):  # four lengths at 4096, four more at 8192: parts of them
        a = list(assign); a[i] = at(other)
        assert lib.pevlm_pages_assign(C.byref(g), *a, 8, None) == pb.PEVLM_EINVAL, i
    a = list(release); a[5] = at(4096 + 8)   # finished
    assert lib.pevlm_pages_release(C.byref(g), *a, None) == pb.PEVLM_EINVAL
    for rows in (-1, 2 ** 30 + 1):
        assert lib.pevlm_pages_assign(C.byref(g), *assign, rows, None) == pb.PEVLM_EINVAL


def test_cache_of_more_than_can_be_counted(lib):
    s, g = pb.make_shape(0, 1, 0, 1, 8, 8, 128), pb.make_pages(2 ** 24, 64, 4, 2)
    assert pb.pevlm_packed_cache_bytes(s, g) == 0
    assert pb.pevlm_packed_cache_bytes(s, pb.make_pages(2 ** 21, 64, 4, 2)) == 2 ** 21 * 8 * 4 * 18 * 128


def test_packed_rows(lib):
    s, g = pb.make_shape(0, 1, 0, 1, 4, 2, 64), pb.make_pages(8, 16, 4, 2)
    assert pb.pevlm_packed_cache_bytes(s, g) == 8 * 2 * 18 * 64
    p = at(4096)
    store = lambda s, g, k=p, v=p, ks=0, vs=0, sl=p, n=4, c=p: lib.pevlm_packed_store(C.byref(s), C.byref(g), k, v, ks, vs, sl, n, c, None)
    load = lambda s, g, c=p, sl=p, n=4, k=p, v=p: lib.pevlm_packed_load(C.byref(s), C.byref(g), c, sl, n, k, v, None)
    for fields, code in BAD_PAGES:
        bad = pb.make_pages(*fields)
        assert store(s, bad) == code and load(s, bad) == code and pb.pevlm_packed_cache_bytes(s, bad) == 0
    for field, val, code in (("head_dim", 96, pb.PEVLM_EUNSUPPORTED), ("num_kv_heads", 3, pb.PEVLM_EINVAL), ("batch", 2, pb.PEVLM_EUNSUPPORTED),
                             ("batch", 0, pb.PEVLM_EINVAL)):
        bad = pb.make_shape(0, 1, 0, 1, 4, 2, 64)
        setattr(bad, field, val)
        assert store(bad, g) == code and load(bad, g) == code, field
    for f in (store, load):
        for name in ("k", "v", "sl", "c"):
            assert f(s, g, **{name: None}) == pb.PEVLM_EINVAL
            assert f(s, g, **{name: at(4098)}) == pb.PEVLM_EALIGN
        assert f(s, g, n=-1) == pb.PEVLM_EINVAL and f(s, g, n=2 ** 30 + 1) == pb.PEVLM_EINVAL
        assert f(s, g, n=0, k=None, v=None, sl=None) == pb.PEVLM_OK
    assert load(s, g, k=at(4096 + 16)) == pb.PEVLM_EALIGN and load(s, g, v=at(4096 + 16)) == pb.PEVLM_EALIGN  # written 32 bytes at a time
    assert store(s, g, k=at(4096 + 16), n=0) == pb.PEVLM_OK
    assert store(s, g, ks=120) == pb.PEVLM_EINVAL and store(s, g, vs=-128) == pb.PEVLM_EINVAL
    assert store(s, g, ks=132) == pb.PEVLM_EALIGN


def test_packed_attn(lib):
    s, g = pb.make_shape(0, 1, 0, 1, 4, 2, 64), pb.make_pages(8, 16, 4, 2)
    p = at(4096)
    size = pb.pevlm_packed_workspace_bytes(s, g, 8, 2)
    assert size > 0
    names = dict(window=0, q=p, qs=0, c=p, tab=p, lens=p, start=p, rows=8, most=2, o=p, lse=p, ws=p, wb=size)

    def attn(s=s, g=g, **kw):
        return lib.pevlm_packed_attn(C.byref(s), C.byref(g), *(dict(names, **kw)[n] for n in names), None)
    for fields, code in BAD_PAGES:
        bad = pb.make_pages(*fields)
        assert attn(g=bad) == code and pb.pevlm_packed_workspace_bytes(s, bad, 8, 2) == 0
    for field, val, code in (("head_dim", 96, pb.PEVLM_EUNSUPPORTED), ("num_kv_heads", 3, pb.PEVLM_EINVAL), ("batch", 2, pb.PEVLM_EUNSUPPORTED),
                             ("softmax_scale", -1.0, pb.PEVLM_EINVAL), ("sink_len", -1, pb.PEVLM_EINVAL)):
        bad = pb.make_shape(0, 1, 0, 1, 4, 2, 64)
        setattr(bad, field, val)
        assert attn(s=bad) == code, field
    for name in ("q", "c", "tab", "lens", "start", "o"):
        assert attn(**{name: None}) == pb.PEVLM_EINVAL, name
        assert attn(**{name: at(4098)}) == pb.PEVLM_EALIGN, name
    assert attn(lse=at(4100)) == pb.PEVLM_EALIGN and attn(o=at(4096 + 16)) == pb.PEVLM_EALIGN
    assert attn(window=-1) == pb.PEVLM_EINVAL
    assert attn(qs=248) == pb.PEVLM_EINVAL and attn(qs=260) == pb.PEVLM_EALIGN
    for rows, most in ((-1, 0), (8, 9), (8, -1), (2 ** 30, 1)):
        assert attn(rows=rows, most=most) == pb.PEVLM_EINVAL
        assert pb.pevlm_packed_workspace_bytes(s, g, rows, most) == 0
    assert attn(ws=None) == pb.PEVLM_EWORKSPACE and attn(wb=size - 1) == pb.PEVLM_EWORKSPACE and attn(ws=at(4096 + 128)) == pb.PEVLM_EALIGN
    assert attn(rows=0, most=0, q=None, o=None) == pb.PEVLM_OK


def test_binding_types():
    s, g = pb.make_shape(0, 1, 0, 1, 4, 2, 64), pb.make_pages(8, 16, 4, 2)
    with pytest.raises(C.ArgumentError):
        pb.pevlm_packed_store(g, s, None, None, None, 0, None)
    with pytest.raises(C.ArgumentError):
        pb.pevlm_pages_release(s, *[None] * 7)


def test_reference_quantiser():
    """The tests' own quantiser: hand values, and never a better choice of code at its scale."""
    x = np.zeros((1, 16)); x[0, :8] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]
    codes, scale = R.quantise(x)
    assert R.SCALES[scale[0, 0]] == 1.0 and codes[0, :8].tolist() == [7, 0, 2, 2, 4, 4, 6, 6]
    rng = np.random.default_rng(1)
    x = rng.standard_normal((64, 16)) * 2.0 ** rng.integers(-6, 7, (64, 1))
    codes, scale = R.quantise(x)
    y = R.dequantise(codes, scale)
    s = R.SCALES[scale][:, :, None]
    best = np.abs(np.abs(x)[:, :, None] - s * R.MAGNITUDES).min(-1)
    assert np.array_equal(np.abs(x - y), best) and (np.sign(y) * np.sign(x) >= 0).all()


def test_reference_allocator():
    a = R.Allocator(6, 16, 3, 3)
    table, free = np.full((3, 3), -1), np.array([0, 1, 2, 3, 4, 5])
    lens, table, count, start, slots, pos = a.assign(np.array([0, 0, 0]), np.array([17, 1, 60]), table, free, 6, 100)
    assert lens.tolist() == [17, 1, 0] and count == 3 and table[0, :2].tolist() == [5, 4] and table[1, 0] == 3
    assert slots[:18].tolist() == list(range(80, 96)) + [64, 48] and (slots[18:] == -1).all() and start.tolist() == [0, 17, 18, 78]
    lens, free, count = a.release([0, 1, 0], lens, table, free, count)
    assert lens.tolist() == [17, 0, 0] and count == 4 and free[3] == 3


def test_window_attn(lib):
    s, p = pb.make_shape(4, 1, 0, 1, 4, 2, 64), at(4096)
    size = pb.pevlm_window_workspace_bytes(s, 100, 50, 4)
    names = dict(window=100, q=p, k=p, v=p, first=50, n=4, rows=54, o=p, lse=p, ws=p, wb=size)
    attn = lambda s=s, **kw: lib.pevlm_window_attn(C.byref(s), *(dict(names, **kw)[n] for n in names), None)
    for field, val, code in (("head_dim", 96, pb.PEVLM_EUNSUPPORTED), ("num_kv_heads", 3, pb.PEVLM_EINVAL), ("batch", 0, pb.PEVLM_EINVAL),
                             ("softmax_scale", -1.0, pb.PEVLM_EINVAL), ("sink_len", -1, pb.PEVLM_EINVAL)):
        bad = pb.make_shape(4, 1, 0, 1, 4, 2, 64)
        setattr(bad, field, val)
        assert attn(s=bad) == code and pb.pevlm_window_workspace_bytes(bad, 100, 50, 4) == 0, field
    for name in ("q", "k", "v", "o"):
        assert attn(**{name: None}) == pb.PEVLM_EINVAL and attn(**{name: at(4098)}) == pb.PEVLM_EALIGN, name
    assert attn(lse=at(4100)) == pb.PEVLM_EALIGN and attn(o=at(4096 + 16)) == pb.PEVLM_EALIGN
    for window, first, n in ((0, 50, 4), (-1, 50, 4), (100, -1, 4), (100, 50, -1), (100, 2 ** 30, 1), (100, 2 ** 62, 2 ** 62)):
        assert attn(window=window, first=first, n=n, rows=2 ** 30) == pb.PEVLM_EINVAL
        assert pb.pevlm_window_workspace_bytes(s, window, first, n) == 0
    assert attn(rows=53) == pb.PEVLM_EINVAL and attn(rows=2 ** 30 + 1) == pb.PEVLM_EINVAL
    assert attn(ws=None) == pb.PEVLM_EWORKSPACE and attn(wb=size - 1) == pb.PEVLM_EWORKSPACE and attn(ws=at(4096 + 128)) == pb.PEVLM_EALIGN
    assert attn(n=0, q=None, k=None, v=None, o=None) == pb.PEVLM_OK
    # one workspace for any cache and window of the same rows
    assert pb.pevlm_window_workspace_bytes(s, 1, 0, 4) == size == pb.pevlm_window_workspace_bytes(s, 2 ** 31 - 1, 10 ** 6, 4)


def test_packed_cache_refuses(monkeypatch):
    import torch
    from paper_2506_19651_b200 import layer
    pbuild.build()
    monkeypatch.setattr(pb, "_native", lambda: pytest.fail("a call was made"))
    with pytest.raises(ValueError, match="no packed cache"):
        layer.PackedCache(2, 100, 4, 24, 8, 4, 2, 64, 1e4, device="cpu")
    with pytest.raises(ValueError, match="step of 0 rows"):
        layer.PackedCache(2, 100, 4, 16, 0, 4, 2, 64, 1e4, device="cpu")
    c = layer.PackedCache(2, 100, 14, 16, 8, 4, 2, 64, 1e4, device="cpu")
    rows = lambda n: [torch.zeros(n, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2)]
    lens = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="at most 8 fit"):
        c.step(*rows(9), lens)
    q, k, v = rows(4)
    with pytest.raises(ValueError, match="the same of each"):
        c.step(q, k[:3], v, lens)
    with pytest.raises(ValueError, match="2 sequences"):
        c.step(q, k, v, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="2 sequences"):
        c.step(q, k, v, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="rows apart"):
        c.store(k, v[:1].expand(4, -1, -1))          # a row for all would be read as four
    with pytest.raises(ValueError, match="rows apart"):
        c.attend(q.transpose(0, 1).contiguous().transpose(0, 1))
    with pytest.raises(ValueError, match="where bf16"):
        c.attend(q.float())
    with pytest.raises(ValueError, match="where bf16"):
        c.store(q, q)
    with pytest.raises(ValueError, match="one after another"):
        c.step(torch.zeros(4, 8, 64, dtype=torch.bfloat16)[:, :4], k, v, lens)
    with pytest.raises(ValueError, match="int32 are read"):
        c.load(torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="2 sequences"):
        c.extend(lens, torch.zeros(1, dtype=torch.int32))
    # a cache, or a tensor beside it, that the current device does not have
    for call in (lambda: c.extend(lens), lambda: c.store(k, v), lambda: c.attend(q), lambda: c.step(q, k, v, lens), lambda: c.load(lens)):
        with pytest.raises(ValueError, match="current device"):
            call()
    class Elsewhere:
        device = torch.device("cuda", 1)
    c.cache = Elsewhere()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: c.extend(lens), lambda: c.store(k, v), lambda: c.attend(q), lambda: c.step(q, k, v, lens), lambda: c.load(lens)):
        with pytest.raises(ValueError, match="on cpu beside"):
            call()
