"""Attention over the packed cache against 64-bit arithmetic on the values that the cache stands for.

Tolerance of an output, derived: the result is rounded to bf16 (2^-8 of it at most); probabilities are rounded to fp16, 2^-11 of each and 2^-25
of the running reference (which is at most 2^8 below the largest) where that is more; scores come from exact products summed in fp32 (under 64 partial sums of at most S = sum |q k|,
2^-24 of it each, an exponential of its own 2^-22).  With A = sum p |v| / sum p:
    2^-8 |o| + (2^-11 + 2^-22 + 2 * 64 * 2^-24 S scale) A + keys * 2^-25 max |v|
and of the log-sum-exp the score's error and fp32's roundings, 64 * 2^-24 S scale + 2^-20 (1 + |lse|).  S is taken as its largest value."""
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


def visible(pos, j, window, sink):
    see = j <= pos
    if window:
        see = see & ((j > pos - window) | (j < sink))
    return see


class Case:
    """Sequences of the given lengths and row counts over pages in random order, stored through the library; the cache's own values come from
    the 64-bit quantiser.  Bytes that nobody stored are 0xFF: codes of -6 with scales that are NaN."""

    def __init__(self, lens, rows, Hq, Hkv, d, P, window=0, sink=0, seed=0, k_scale=1.0, extra_rows=0, stride=0, holes=(), scale=0.0, q_scale=1.0):
        import torch
        from paper_2506_19651_b200 import binding as pb
        self.pb, self.window, self.sink, self.d, self.Hq, self.Hkv, self.P = pb, window, sink, d, Hq, Hkv, P
        rng = np.random.default_rng(seed)
        self.lens, self.rows = np.array(lens), np.array(rows)
        n = len(lens)
        held = -(-self.lens // P)
        pages, most = int(held.sum()) + 3, max(int(held.max()), 1) + 1
        order = rng.permutation(pages)
        table = rng.integers(-3, 2 ** 31 - 1, (n, most))
        at = 0
        for r in range(n):
            table[r, :held[r]] = order[at:at + held[r]]
            at += held[r]
        self.shape = pb.make_shape(sink, 1, 0, 1, Hq, Hkv, d, scale=scale)
        self.scale = scale or d ** -0.5
        self.pages = pb.make_pages(pages, P, n, most)
        self.cache = torch.full((pages, Hkv, P // 16, 18 * d), 0xFF, dtype=torch.uint8, device="cuda")
        self.k, self.v = [], []
        for r in range(n):
            L = int(self.lens[r])
            k = _bf16(rng.standard_normal((L, Hkv, d)) * k_scale)
            v = _bf16(rng.standard_normal((L, Hkv, d)))
            t = np.arange(L)
            slots = torch.from_numpy((table[r, t // P] * P + t % P).astype(np.int32)).cuda()
            pb.pevlm_packed_store(self.shape, self.pages, k, v, slots, L, self.cache)
            for x, to in ((k, self.k), (v, self.v)):
                to.append(R.dequantise(*R.quantise(_values(x))) if L else np.zeros((0, Hkv, d)))
        for r, page in holes:
            table[r, page] = [-1, pages, 2 ** 31 - 1][page % 3]
        self.holes = holes
        i32 = lambda a: torch.from_numpy(np.asarray(a, dtype=np.int64).astype(np.int32)).cuda()
        self.table, self.d_lens = i32(table), i32(lens)
        start = np.concatenate([[0], np.cumsum(rows)])
        self.start, self.n_rows = i32(start), int(start[-1]) + extra_rows
        self.used = int(start[-1])
        self.stride = stride
        width = stride or Hq * d
        q = rng.standard_normal((max(self.n_rows, 1), width)) * q_scale
        self.q = _bf16(q)
        self.q_values = _values(self.q)[:self.used, :Hq * d].reshape(self.used, Hq, d)

    def run(self, max_rows=None):
        import torch
        pb = self.pb
        guard = GuardedAllocator()
        o, lse = guard((self.n_rows, self.Hq, self.d), torch.bfloat16), guard((self.Hq, self.n_rows), torch.float32)
        o.fill_(-7.0)
        lse.fill_(-7.0)
        most = int(self.rows.max()) if max_rows is None else max_rows
        size = pb.pevlm_packed_workspace_bytes(self.shape, self.pages, self.n_rows, most)
        assert size > 0
        ws = guard((size,), torch.uint8)
        ws.fill_(0xFF)
        pb.pevlm_packed_attn(self.shape, self.pages, self.window, self.q, self.cache, self.table, self.d_lens, self.start, self.n_rows, most,
                             o, lse, ws, self.stride)
        assert pb.pevlm_read_status(ws) == (0, 0)
        guard.check()
        return o, lse

    def check(self, o, lse):
        o_all, lse_all = _values(o), lse.double().cpu().numpy()
        assert (o_all[self.used:] == -7).all() and (lse_all[:, self.used:] == -7).all()
        G, row = self.Hq // self.Hkv, 0
        for r, (L, n) in enumerate(zip(self.lens, self.rows)):
            if n == 0:
                continue
            q = self.q_values[row:row + n].reshape(n, self.Hkv, G, self.d)
            j = np.arange(L)
            pos = L - n + np.arange(n)
            see = visible(pos[:, None], j, self.window, self.sink)
            for hole_r, page in self.holes:
                if hole_r == r:
                    see = see & (j // self.P != page)
            s = np.einsum("nhgd,khd->nhgk", q, self.k[r]) * self.scale
            big = (np.einsum("nhgd,khd->nhgk", np.abs(q), np.abs(self.k[r])) * self.scale).max() if L else 0.0
            s = np.where(see[:, None, None], s, -np.inf)
            top = np.max(s, axis=-1, keepdims=True, initial=-np.inf)
            p = np.exp(s - np.where(np.isinf(top), 0.0, top))
            l = p.sum(-1)
            inv = np.where(l > 0, 1 / np.where(l > 0, l, 1), 0.0)
            want = np.einsum("nhgk,khd->nhgd", p, self.v[r]) * inv[..., None]
            a = np.einsum("nhgk,khd->nhgd", p, np.abs(self.v[r])) * inv[..., None]
            with np.errstate(divide="ignore"):
                z = np.where(l > 0, np.where(np.isinf(top[..., 0]), 0.0, top[..., 0]) + np.log(l), -np.inf)
            score = 64 * 2.0 ** -24 * big
            tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 + 2.0 ** -22 + 2 * score) * a + L * 2.0 ** -25 * (np.abs(self.v[r]).max() if L else 0.0)
            got = o_all[row:row + n].reshape(n, self.Hkv, G, self.d)
            assert np.isfinite(got).all()
            over = np.abs(got - want) - tol
            assert over.max() <= 0, (r, L, n, np.unravel_index(over.argmax(), over.shape), over.max())
            got_z = lse_all[:, row:row + n].T.reshape(n, self.Hkv, G)
            none = np.isinf(z)
            assert np.array_equal(got_z[none], z[none])
            assert (np.abs(got_z[~none] - z[~none]) <= score + 2.0 ** -20 * (1 + np.abs(z[~none]))).all()
            row += n


CASES = {
    "one key": dict(lens=[1], rows=[1], Hq=7, Hkv=1, d=128, P=16),
    "no key": dict(lens=[0], rows=[1], Hq=4, Hkv=2, d=64, P=16),
    "no key among others": dict(lens=[5, 0, 40, 0], rows=[1, 2, 1, 0], Hq=4, Hkv=2, d=128, P=32),
    "page ends": dict(lens=[15, 16, 17, 63, 64, 65, 127, 128, 129], rows=[1] * 9, Hq=8, Hkv=1, d=128, P=64),
    "page ends, heads of 64": dict(lens=[15, 16, 17, 31, 32, 33, 1, 2], rows=[1, 2, 3, 1, 1, 2, 1, 2], Hq=8, Hkv=2, d=64, P=16),
    "more rows than keys": dict(lens=[3, 1], rows=[9, 4], Hq=4, Hkv=4, d=64, P=16),
    "drafted tokens": dict(lens=[300, 77, 1000], rows=[4, 2, 3], Hq=14, Hkv=2, d=128, P=32),
    "17 rows of a group of 3": dict(lens=[200], rows=[17], Hq=3, Hkv=1, d=128, P=16),
    "a question": dict(lens=[700, 90], rows=[64, 33], Hq=28, Hkv=4, d=128, P=64),
    "as many rows as keys": dict(lens=[150, 40], rows=[150, 40], Hq=4, Hkv=2, d=64, P=128),
    "group of 16": dict(lens=[260], rows=[3], Hq=16, Hkv=1, d=128, P=16),
    "group of 1": dict(lens=[260, 31], rows=[1, 1], Hq=5, Hkv=5, d=64, P=16),
    "many short": dict(lens=list(range(0, 120)), rows=[1] * 120, Hq=8, Hkv=2, d=64, P=16),
    "many without rows": dict(lens=[50] * 70, rows=[0] * 33 + [1] + [0] * 35 + [2], Hq=7, Hkv=1, d=128, P=16),
    "long": dict(lens=[9001], rows=[1], Hq=28, Hkv=4, d=128, P=64),
    "long and short": dict(lens=[12000, 3, 700, 5000], rows=[1, 1, 2, 1], Hq=8, Hkv=2, d=64, P=32),
    "window": dict(lens=[500, 40, 16, 1000], rows=[1, 1, 3, 2], Hq=8, Hkv=2, d=64, P=16, window=100, sink=4),
    "window of one": dict(lens=[50, 3], rows=[5, 1], Hq=4, Hkv=1, d=128, P=16, window=1, sink=0),
    "window, sink at tile ends": dict(lens=[400, 400, 33], rows=[2, 1, 1], Hq=7, Hkv=1, d=128, P=64, window=17, sink=32),
    "sink longer than the sequence": dict(lens=[20, 300], rows=[2, 2], Hq=4, Hkv=2, d=64, P=16, window=8, sink=64),
    "window longer than all": dict(lens=[100, 260], rows=[2, 9], Hq=4, Hkv=2, d=128, P=32, window=2 ** 31 - 1, sink=3),
    "question under a window": dict(lens=[600], rows=[130], Hq=14, Hkv=2, d=128, P=32, window=70, sink=5),
    "extra rows": dict(lens=[40, 70], rows=[1, 2], Hq=4, Hkv=2, d=64, P=16, extra_rows=5),
    "strided rows": dict(lens=[90, 70], rows=[1, 2], Hq=4, Hkv=2, d=64, P=16, stride=4 * 64 + 4 * 64),
    "pages that are not there": dict(lens=[100, 64, 300], rows=[1, 2, 1], Hq=4, Hkv=2, d=64, P=16, holes=[(0, 2), (1, 0), (1, 1), (1, 2), (1, 3), (2, 18)]),
    "large keys": dict(lens=[400], rows=[2], Hq=7, Hkv=1, d=128, P=16, k_scale=8.0),
    "small queries": dict(lens=[400], rows=[2], Hq=7, Hkv=1, d=128, P=16, q_scale=2.0 ** -100, k_scale=30.0),
    "large queries": dict(lens=[100], rows=[2], Hq=7, Hkv=1, d=64, P=16, q_scale=2.0 ** 40, scale=2.0 ** -43),
    "40 rows": dict(lens=[129], rows=[40], Hq=2, Hkv=2, d=128, P=16),
    "question, heads of 64": dict(lens=[1000, 127, 128, 129], rows=[50, 127, 128, 40], Hq=8, Hkv=2, d=64, P=16),
    "question of a long cache": dict(lens=[9000], rows=[64], Hq=28, Hkv=4, d=128, P=64),
    "questions of 300 and 1": dict(lens=[2500, 700, 1, 0, 300], rows=[300, 1, 1, 2, 300], Hq=7, Hkv=1, d=128, P=32),
    "more question than cache": dict(lens=[100, 0, 30], rows=[400, 70, 50], Hq=4, Hkv=2, d=64, P=16),
    "chunk of a prefill under a window": dict(lens=[3000, 900], rows=[700, 900], Hq=4, Hkv=1, d=128, P=64, window=150, sink=70),
    "window, heads of 64, sink of two tiles": dict(lens=[1500], rows=[333], Hq=6, Hkv=2, d=64, P=32, window=260, sink=200),
    "short window": dict(lens=[700], rows=[200], Hq=2, Hkv=1, d=64, P=16, window=3, sink=1),
    "question, pages that are not there": dict(lens=[1100, 300], rows=[64, 40], Hq=4, Hkv=2, d=128, P=16, holes=[(0, 0), (0, 7), (0, 20), (0, 21), (0, 68), (1, 18)]),
    "whole tiles that are not there": dict(lens=[900], rows=[90], Hq=4, Hkv=2, d=64, P=128, holes=[(0, 0), (0, 3), (0, 7)]),
    "many questions": dict(lens=[(i * 53) % 400 for i in range(150)], rows=[(i * 7) % 60 for i in range(150)], Hq=4, Hkv=2, d=64, P=16),
    "question, large keys": dict(lens=[600], rows=[64], Hq=7, Hkv=1, d=128, P=16, k_scale=8.0),
    "question, small and strided queries": dict(lens=[500], rows=[64], Hq=4, Hkv=1, d=64, P=16, q_scale=2.0 ** -90, k_scale=20.0, stride=4 * 64 + 128, extra_rows=3),
    "group of 40": dict(lens=[200, 31, 0], rows=[1, 1, 1], Hq=40, Hkv=1, d=64, P=16),
    "group of 128": dict(lens=[300, 31, 0, 129], rows=[1, 2, 1, 1], Hq=128, Hkv=1, d=128, P=16),
    "128 heads on 128": dict(lens=[70, 200], rows=[1, 2], Hq=128, Hkv=128, d=64, P=16),
    "many under a window": dict(lens=[(i * 37) % 700 for i in range(300)], rows=[1 + i % 2 for i in range(300)], Hq=4, Hkv=1, d=64, P=32, window=50, sink=4),
    "many questions under a window": dict(lens=[(i * 53) % 700 for i in range(200)], rows=[(i * 7) % 60 for i in range(200)], Hq=4, Hkv=2, d=64, P=16, window=90, sink=20),
    "one of many": dict(lens=[0] * 700 + [900] + [40] * 200, rows=[0] * 700 + [2] + [0] * 200, Hq=8, Hkv=2, d=64, P=16),
    "few of many": dict(lens=[(i * 31) % 500 for i in range(1500)], rows=[i % 3 + 1 if i in (0, 1, 129, 130, 700, 1403, 1499) else 0 for i in range(1500)], Hq=4, Hkv=2, d=128, P=32),
    "questions of a few of many": dict(lens=[(i * 31) % 500 for i in range(1500)], rows=[i % 100 + 1 if i in (0, 1, 2, 3, 4, 129, 130, 700, 1403, 1499) else 0 for i in range(1500)], Hq=4, Hkv=2, d=64, P=16),
    "few of 128": dict(lens=[200] * 128, rows=[2 if i in (5, 6, 90, 127) else 0 for i in range(128)], Hq=4, Hkv=2, d=64, P=16),
    "single tokens beside a question": dict(lens=[300 + i for i in range(40)], rows=[1] * 20 + [70] + [1] * 18 + [5], Hq=7, Hkv=1, d=128, P=32),
    "single tokens beside a question, heads of 64": dict(lens=[300 + i for i in range(40)], rows=[2] * 30 + [33] + [0] * 8 + [90], Hq=8, Hkv=2, d=64, P=16, window=200, sink=9),
    "rows of no sequence": dict(lens=[300, 20, 0], rows=[0, 0, 0], Hq=4, Hkv=2, d=64, P=16, extra_rows=40),
    "scale": dict(lens=[100], rows=[1], Hq=4, Hkv=2, d=64, P=16, scale=0.5),
}


@pytest.mark.parametrize("name", CASES)
def test_against_the_definition(name):
    c = Case(**CASES[name], seed=len(name))
    c.check(*c.run())


@pytest.mark.parametrize("name", ["drafted tokens", "a question", "page ends", "as many rows as keys", "page ends, heads of 64", "no key among others", "window",
                                  "pages that are not there", "many without rows", "sink longer than the sequence", "single tokens beside a question",
                                  "rows of no sequence"])
def test_any_row_hint_gives_a_right_result(name):
    """max_rows chooses the kernel; the row counts on the device are what is computed."""
    c = Case(**CASES[name], seed=3)
    for most in (1, min(c.n_rows, 2), c.n_rows):
        c.check(*c.run(max_rows=most))


@pytest.mark.parametrize("rows", [[1, 2, 1], [64, 3, 200]])
def test_same_bits_twice_and_on_a_replayed_graph(rows):
    import torch
    c = Case([3000, 17, 900], rows, 28, 4, 128, 64, seed=9)
    most = max(rows)
    o, lse = c.run()
    o2, lse2 = c.run()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    pb = c.pb
    ws = torch.empty(pb.pevlm_packed_workspace_bytes(c.shape, c.pages, c.n_rows, most), dtype=torch.uint8, device="cuda")
    o3, lse3 = torch.zeros_like(o), torch.zeros_like(lse)
    call = lambda: pb.pevlm_packed_attn(c.shape, c.pages, 0, c.q, c.cache, c.table, c.d_lens, c.start, c.n_rows, most, o3, lse3, ws)
    side, graphs = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    for _ in range(2):  # two graphs that share the workspace, replayed in turn
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            call()
    for graph in graphs * 2:
        o3.zero_(); lse3.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, o3) and torch.equal(lse, lse3)


def test_lengths_that_change_between_replays():
    """Lengths are read on the device: a captured step serves whatever they have become."""
    import torch
    c = Case([400, 90, 200], [1, 1, 1], 8, 2, 64, 16, seed=4)
    pb = c.pb
    ws = torch.empty(pb.pevlm_packed_workspace_bytes(c.shape, c.pages, 3, 1), dtype=torch.uint8, device="cuda")
    o, lse = torch.zeros((3, 8, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((8, 3), device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        pb.pevlm_packed_attn(c.shape, c.pages, 0, c.q, c.cache, c.table, c.d_lens, c.start, 3, 1, o, lse, ws)
    full = c.lens.copy()
    for lens in (full, [1, 0, 200], [17, 89, 16]):
        c.d_lens.copy_(torch.tensor(np.array(lens), dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        c.lens = np.array(lens)
        k, v = c.k, c.v
        c.k, c.v = [x[:n] for x, n in zip(k, lens)], [x[:n] for x, n in zip(v, lens)]
        c.check(o, lse)
        c.k, c.v = k, v


@pytest.mark.parametrize("rows,window,sink", [([1, 3], 40, 5), ([2, 1], 100, 0), ([60, 90], 150, 20), ([70, 100], 33, 200)])
@pytest.mark.parametrize("Hq,Hkv,d", [(7, 1, 128), (4, 1, 64)])
def test_keys_that_no_row_sees_may_hold_anything(rows, window, sink, Hq, Hkv, d):
    """Pages between the sink and the window whose bytes are codes of -6 and scales that are NaN (pages given back, say)."""
    import torch
    c = Case([700, 900], rows, Hq, Hkv, d, 16, window=window, sink=sink, seed=5)
    o, lse = c.run()
    c.check(o, lse)
    for r, (L, n) in enumerate(zip(c.lens, c.rows)):
        for t in range(sink, int(L - n - window + 1)):
            page, u = int(c.table[r, t // 16]), t % 16
            h, k8, w, g = u // 8, u % 8, d // 64, d // 16
            tile = c.cache[page, :, 0]
            # the scales of token u, K's and V's
            tile[:, [16 * d + k8 * 2 * g + (i // w) * 2 * w + h * w + i % w for i in range(g)]] = 0xFF
            tile[:, [17 * d + i * 16 + (k8 // 2) * 4 + h * 2 + k8 % 2 for i in range(g)]] = 0xFF
    o2, lse2 = c.run()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("rows", [[2, 3], [3, 5], [64, 100]])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_row_that_is_no_number_stays_alone(rows, value):
    c = Case([500, 333], rows, 6, 2, 64, 16, seed=7)
    o, lse = c.run()
    at = rows[0] + 1  # the second row of the second sequence, one of its heads
    c.q[at, 64:128] = value
    o2, lse2 = c.run()
    if value != value:
        assert bool(o2[at, 1].isnan().all())
    o2[at, 1], lse2[1, at] = o[at, 1], lse[1, at]
    c.check(o2, lse2)


def test_calls_on_two_streams_at_once():
    """Each with its own workspace; both kernels take every SM."""
    import torch
    cases = [Case([9000, 40], [1, 2], 8, 2, 128, 64, seed=1), Case([3000], [200], 8, 2, 64, 16, seed=2)]
    calls, streams, got = [], [torch.cuda.Stream(), torch.cuda.Stream()], []
    want = [c.run() for c in cases]
    for c in cases:
        most = int(c.rows.max())
        ws = torch.empty(c.pb.pevlm_packed_workspace_bytes(c.shape, c.pages, c.n_rows, most), dtype=torch.uint8, device="cuda")
        calls.append((c, most, ws, torch.zeros((c.n_rows, c.Hq, c.d), dtype=torch.bfloat16, device="cuda"), torch.zeros((c.Hq, c.n_rows), device="cuda")))
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, (c, most, ws, o, lse) in zip(streams, calls):
            with torch.cuda.stream(stream):
                c.pb.pevlm_packed_attn(c.shape, c.pages, 0, c.q, c.cache, c.table, c.d_lens, c.start, c.n_rows, most, o, lse, ws)
    torch.cuda.synchronize()
    for (o, lse), (_, _, ws, o2, lse2) in zip(want, calls):
        assert cases[0].pb.pevlm_read_status(ws) == (0, 0)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("rows", [1, 70])
def test_no_query_and_the_smallest_scale(rows):
    """Rows of Q that are 0 weigh all that they see alike, and so does a scale that leaves nothing of the scores."""
    c = Case([100, 60], [rows, 2], 4, 2, 64, 16, scale=2.0 ** -40, seed=6)
    c.q.view(-1)[:64] = 0
    c.q_values = _values(c.q)[:c.used].reshape(c.used, 4, 64)
    c.check(*c.run())
    c = Case([100, 60], [rows, 2], 4, 2, 64, 16, q_scale=2.0 ** -120, scale=2.0 ** -30, seed=6)
    c.check(*c.run())


@pytest.mark.parametrize("rows", [[1, 2, 1], [1, 60, 2], [50, 60, 70]])
def test_the_most_sequences_that_a_table_may_have(rows):
    """Three of 2^20 have rows: the first, one in the middle and the last."""
    import torch
    c = Case([90, 16, 75], rows, 4, 2, 64, 16, seed=8)
    n, at = 2 ** 20, [0, 500001, 2 ** 20 - 1]
    table = torch.full((n, c.table.shape[1]), -1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(n, dtype=torch.int32, device="cuda")
    counts = torch.zeros(n, dtype=torch.int64, device="cuda")
    table[at], lens[at], counts[at] = c.table, c.d_lens, torch.tensor(rows, device="cuda")
    c.table, c.d_lens = table, lens
    c.start = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0)]).int()
    c.pages = c.pb.make_pages(c.pages.num_pages, 16, n, table.shape[1])
    c.check(*c.run())


def test_rows_without_lse():
    import torch
    c = Case([100], [2], 4, 2, 64, 16)
    o, lse = c.run()
    ws = torch.empty(c.pb.pevlm_packed_workspace_bytes(c.shape, c.pages, 2, 2), dtype=torch.uint8, device="cuda")
    o2 = torch.zeros_like(o)
    c.pb.pevlm_packed_attn(c.shape, c.pages, 0, c.q, c.cache, c.table, c.d_lens, c.start, 2, 2, o2, None, ws)
    assert torch.equal(o, o2)


def test_offsets_past_32_bits():
    """A cache of more than 4 GiB: pages at its far end."""
    import torch
    from paper_2506_19651_b200 import binding as pb
    Hq, Hkv, d, P = 8, 8, 128, 128
    s, big = pb.make_shape(0, 1, 0, 1, Hq, Hkv, d), pb.make_pages(31000, P, 1, 4)  # pages of 147,456 bytes: 8 heads, 128 tokens of 144
    assert pb.pevlm_packed_cache_bytes(s, big) > 2 ** 32
    cache = torch.empty(pb.pevlm_packed_cache_bytes(s, big), dtype=torch.uint8, device="cuda")
    torch.manual_seed(1)
    k, v = (torch.randn((300, Hkv, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn((1, Hq, d), device="cuda").to(torch.bfloat16)
    got = []
    for first in (0, 30996):
        table = torch.tensor([[first + 3, first, first + 2, 5]], dtype=torch.int32, device="cuda")
        at = torch.arange(300, device="cuda")
        slots = (table[0, at // P] * P + at % P).int()
        pb.pevlm_packed_store(s, big, k, v, slots, 300, cache)
        ko, vo = torch.empty_like(k), torch.empty_like(v)
        pb.pevlm_packed_load(s, big, cache, slots, 300, ko, vo)
        o, lse = torch.empty_like(q), torch.empty((Hq, 1), device="cuda")
        ws = torch.empty(pb.pevlm_packed_workspace_bytes(s, big, 1, 1), dtype=torch.uint8, device="cuda")
        pb.pevlm_packed_attn(s, big, 0, q, cache, table, torch.tensor([300], dtype=torch.int32, device="cuda"),
                             torch.tensor([0, 1], dtype=torch.int32, device="cuda"), 1, 1, o, lse, ws)
        got.append((ko, vo, o, lse))
    for a, b in zip(*got):
        assert torch.equal(a, b)
