"""A step over the packed cache that is refused has changed nothing: whatever the calls would refuse is looked at before the first of them."""
import pytest


def _shifted(rows, by):
    """The same rows at an address `by` elements past a multiple of 16 bytes."""
    import torch
    buf = torch.empty(rows.numel() + 16, dtype=rows.dtype, device=rows.device)
    at = buf[by:by + rows.numel()].view(rows.shape)
    at.copy_(rows)
    return at


def _apart(rows, stride):
    import torch
    n, h, d = rows.shape
    buf = torch.empty((n, stride), dtype=rows.dtype, device=rows.device)
    at = buf[:, :h * d].unflatten(1, (h, d))
    at.copy_(rows)
    return at


def _bad_steps(q, k, v):
    yield dict(q=_shifted(q, 3), k=k, v=v)
    yield dict(q=q, k=_shifted(k, 1), v=v)
    yield dict(q=q, k=k, v=_shifted(v, 5))
    yield dict(q=q, k=k, v=_apart(v, 2 * 64 + 4))
    yield dict(q=q, k=k, v=v, most=-1)


def _rows(n, device):
    import torch
    torch.manual_seed(n)
    return [torch.randn((n, h, 64), device=device).to(torch.bfloat16) for h in (4, 2, 2)]


def test_before_any_call(monkeypatch):
    import torch
    from paper_2506_19651_b200 import binding as pb
    from paper_2506_19651_b200 import build, layer
    build.build()
    monkeypatch.setattr(pb, "_native", lambda: pytest.fail("a call was made"))
    monkeypatch.setattr(layer.PackedCache, "_at_hand", lambda self, *tensors: None)
    c = layer.PackedCache(2, 100, 14, 16, 8, 4, 2, 64, 1e4, device="cpu")
    lens = torch.ones(2, dtype=torch.int32)
    for bad in _bad_steps(*_rows(2, "cpu")):
        with pytest.raises(ValueError, match="16 bytes at a time|at most -1 rows"):
            c.step(new_lens=lens, **bad)
    c._room = 8  # as extend() leaves it: store() of fewer rows would make the page call again
    for bad in list(_bad_steps(*_rows(2, "cpu")))[1:4]:
        with pytest.raises(ValueError, match="16 bytes at a time"):
            c.store(bad["k"], bad["v"])


def test_a_cache_whose_steps_would_all_be_refused():
    from paper_2506_19651_b200 import build, layer
    build.build()
    for window in (-1, 2 ** 31, 2 ** 32 + 5):
        with pytest.raises(ValueError, match="window"):
            layer.PackedCache(2, 100, 14, 16, 8, 4, 2, 64, 1e4, window=window, device="cpu")


@pytest.mark.gpu
def test_nothing_changes():
    import torch
    from paper_2506_19651_b200.layer import PackedCache
    c = PackedCache(2, 100, 14, 16, 40, 4, 2, 64, 1e4)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    c.step(*_rows(30, "cuda"), i32([20, 10]))
    state = lambda: [x.clone() for x in (c.lens, c.free_count, c.page_table, c.free_list, c.row_start, c.slots, c.positions, c.cache)]
    before = state()
    for bad in _bad_steps(*_rows(17, "cuda")):
        with pytest.raises(ValueError):
            c.step(new_lens=i32([0, 17]), finished=i32([1, 0]), **bad)
        assert all(torch.equal(a, b) for a, b in zip(before, state()))
    o, lse = c.step(*_rows(17, "cuda"), i32([0, 17]), i32([1, 0]))
    assert c.lens.tolist() == [0, 27] and bool(torch.isfinite(lse).all())


def test_no_slots_before_the_first_step():
    """A store() that no extend() has made room for would put all its rows into the first slot of the first page."""
    from paper_2506_19651_b200 import build, layer
    build.build()
    c = layer.PackedCache(2, 100, 14, 16, 8, 4, 2, 64, 1e4, device="cpu")
    assert c.slots.tolist() == [-1] * 8 and str(c.slots.dtype) == "torch.int32"


@pytest.mark.gpu
def test_nothing_to_store_behind_a_refused_extend():
    """New lengths that are the cache's own: refused by the second page call, and the rows of the step before cannot be stored once more."""
    import torch
    from paper_2506_19651_b200 import binding as pb
    from paper_2506_19651_b200.layer import PackedCache
    c = PackedCache(2, 100, 14, 16, 40, 4, 2, 64, 1e4)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    c.extend(i32([7, 2]))
    with pytest.raises(pb.PevlmError):
        c.extend(c.lens)
    with pytest.raises(ValueError, match="for a step of 0"):
        c.store(*_rows(9, "cuda")[1:])
    assert c.lens.tolist() == [7, 2]
    c.extend(i32([1, 1]))
    c.store(*_rows(2, "cuda")[1:])
    assert c.lens.tolist() == [8, 3] and int(c.free_count) == 12
