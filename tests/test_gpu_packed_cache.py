"""Whole steps over the packed cache (layer.PackedCache): pages, RoPE, rows in 4 bits and attention together, against an allocator in
plain Python, the oracle's RoPE, the 64-bit quantiser and attention in 64 bits (tolerances: see test_gpu_packed_attn)."""
import numpy as np
import pytest

import packed_reference as R
from helpers import bits_to_f64, to_bits
from oracle import api as oracle
from test_gpu_packed_attn import _bf16, _values, visible

pytestmark = pytest.mark.gpu


class Model:
    """The same steps in 64 bits."""

    def __init__(self, cache, theta, window, sink):
        g = cache.pages
        self.a = R.Allocator(g.num_pages, g.page_len, g.num_seqs, g.max_pages)
        self.lens, self.table = np.zeros(g.num_seqs, np.int64), np.full((g.num_seqs, g.max_pages), -1)
        self.free, self.count = np.arange(g.num_pages), g.num_pages
        self.k, self.v = [None] * g.num_seqs, [None] * g.num_seqs
        self.theta, self.window, self.sink, self.max_rows = theta, window, sink, cache.max_rows

    def step(self, q, k, v, new, finished):
        """Bits of the rows; returns per row (o, lse, tolerance, tolerance of lse) or None where the sequence found no room."""
        self.lens, self.free, self.count = self.a.release(finished, self.lens, self.table, self.free, self.count)
        for r in np.nonzero(finished)[0]:
            self.k[r] = self.v[r] = None
        self.lens, self.table, self.count, start, slots, positions = self.a.assign(self.lens, new, self.table, self.free, self.count, self.max_rows)
        n = len(q)
        qr = bits_to_f64(oracle.rope(q, self.theta, pos=positions[:n]))
        kr = R.dequantise(*R.quantise(bits_to_f64(oracle.rope(k, self.theta, pos=positions[:n]))))
        vr = R.dequantise(*R.quantise(bits_to_f64(v)))
        out = [None] * n
        for s in range(len(new)):
            rows = range(start[s], start[s + 1])
            if len(rows) == 0 or start[s + 1] > len(slots) or slots[start[s]] < 0:
                continue
            for have, x in ((self.k, kr), (self.v, vr)):
                have[s] = x[rows] if have[s] is None else np.concatenate([have[s], x[rows]])
            G = q.shape[1] // k.shape[1]
            j = np.arange(self.lens[s])
            for i in rows:
                see = visible(positions[i], j, self.window, self.sink)
                kk, vv, qq = self.k[s][see], self.v[s][see], qr[i].reshape(k.shape[1], G, -1)
                scale = q.shape[2] ** -0.5
                sc = np.einsum("hgd,khd->hgk", qq, kk) * scale
                big = 64 * 2.0 ** -24 * (np.einsum("hgd,khd->hgk", np.abs(qq), np.abs(kk)) * scale).max()
                top = sc.max(-1, keepdims=True)
                p = np.exp(sc - top)
                l = p.sum(-1, keepdims=True)
                o = (np.einsum("hgk,khd->hgd", p, vv) / l).reshape(q.shape[1:])
                a = (np.einsum("hgk,khd->hgd", p, np.abs(vv)) / l).reshape(q.shape[1:])
                z = (top + np.log(l)).reshape(-1)
                out[i] = (o, z, 2.0 ** -8 * np.abs(o) + (2.0 ** -11 + 2.0 ** -22 + 2 * big) * a + len(j) * 2.0 ** -25 * np.abs(vv).max(), big + 2.0 ** -20 * (1 + np.abs(z)))
        return out, slots, positions, start


@pytest.mark.parametrize("Hq,Hkv,d,P,window,sink", [(8, 2, 64, 16, 0, 0), (7, 1, 128, 32, 40, 3), (28, 4, 128, 64, 0, 0)])
def test_steps(Hq, Hkv, d, P, window, sink):
    import torch
    from paper_2506_19651_b200.layer import PackedCache
    rng = np.random.default_rng(d + P)
    theta, n_seqs, max_rows = 1e6, 5, 256
    cache = PackedCache(n_seqs, 600, 40 if P == 16 else 24, P, max_rows, Hq, Hkv, d, theta, window=window, sink=sink)
    model = Model(cache, theta, window, sink)
    script = [  # new tokens, finished, padding rows behind the last sequence
        ([90, 33, 0, 1, 64], [0] * 5, 0), ([1, 1, 0, 1, 1], [0] * 5, 0), ([1, 4, 70, 0, 2], [0] * 5, 3), ([1, 1, 1, 1, 1], [0, 1, 0, 0, 0], 0),
        ([0, 55, 1, 3, 1], [0, 0, 0, 0, 1], 11), ([100, 1, 1, 1, 100], [0] * 5, 0), ([300, 1, 2, 1, 1], [1, 0, 1, 0, 0], 0)]
    for new, finished, padding in script:
        n = min(sum(new) + padding, max_rows)
        bits = [to_bits(_bf16(rng.standard_normal((n, h, d)))).reshape(n, h, d) for h in (Hq, Hkv, Hkv)]
        want, slots, positions, start = model.step(*bits, np.array(new), np.array(finished))
        dev = [torch.from_numpy(b.view(np.int16)).cuda().view(torch.bfloat16) for b in bits]
        kv = torch.cat([dev[2], dev[2]], 1)  # V as the upper half of a fused projection
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
        o, lse = cache.step(dev[0], dev[1], kv[:, Hkv:], i32(new), i32(finished) if any(finished) else None, most=max(new))
        assert np.array_equal(cache.slots.cpu().numpy(), slots) and np.array_equal(cache.positions.cpu().numpy(), positions)
        assert np.array_equal(cache.lens.cpu().numpy(), model.lens) and int(cache.free_count) == model.count
        got, z = _values(o), lse.double().cpu().numpy().T
        checked = 0
        for i, w in enumerate(want):
            if w is not None:
                assert (np.abs(got[i] - w[0]) <= w[2]).all() and (np.abs(z[i] - w[1]) <= w[3]).all(), (new, i)
                checked += 1
        assert checked > 0 or new[0] > max_rows  # rows past the first sequence too long find no room
    # what the cache holds of a sequence, read back
    s = int(model.lens.argmax())
    t = np.arange(model.lens[s])
    at = torch.from_numpy((model.table[s, t // P] * P + t % P).astype(np.int32)).cuda()
    k, v = cache.load(at)
    assert np.array_equal(_values(k), model.k[s]) and np.array_equal(_values(v), model.v[s])


def test_video_encoded_by_blocks_then_asked():
    """A video through the block-wise prefill, its roped keys and values packed, and a question over the packed cache: the same as the
    question attention over the bf16 cache to within what 4 bits leave (and exactly the packed cache's own attention, see above)."""
    import torch
    from paper_2506_19651_b200 import binding as pb
    from paper_2506_19651_b200.layer import LayerBuffers, PackedCache, layer_forward
    S, B, N, Q, Hq, Hkv, d, theta = 64, 128, 4, 24, 14, 2, 128, 1e6
    s = pb.make_shape(S, B, N, Q, Hq, Hkv, d, theta=theta)
    torch.manual_seed(3)
    q, k, v = (torch.randn((s.L, h, d), device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
    buf = layer_forward(LayerBuffers(s), q, k, v)
    cache = PackedCache(2, 1024, 40, 32, s.L, Hq, Hkv, d, theta)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    cache.extend(i32([0, s.n_video]))
    cache.store(buf.k_cache[:s.n_video], buf.v_cache[:s.n_video])
    o, lse = cache.step(q[s.n_video:], k[s.n_video:], v[s.n_video:], i32([0, Q]), most=Q)
    # the same question with a bf16 cache that holds the packed values
    table = cache.page_table[1].long()
    t = torch.arange(s.L, device="cuda")
    kd, vd = cache.load((table[t // 32] * 32 + t % 32).int())
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    pb.pevlm_query_attn(s, buf.q_question[:Q], kd, vd, o2, lse2, buf.ws_query)
    a = o.double() - o2.double()
    # both round to bf16; that of the bf16 cache its probabilities too (2^-8 of sum p |v| / sum p <= the largest |v|)
    assert float(a.abs().max()) <= 2.0 ** -7 * float(o2.double().abs().max()) + (2.0 ** -8 + 2.0 ** -11) * float(vd.double().abs().max())
    assert float((lse - lse2).abs().max()) < 1e-4
    # and 4 bits: a key is off by at most a sixth of its group's largest, on average far less
    assert float((o.double() - buf.o_question.double()).norm() / buf.o_question.double().norm()) < 0.35


def test_steps_without_rows():
    """A step that only gives pages back, and one of no rows at all."""
    import torch
    from paper_2506_19651_b200.layer import PackedCache
    c = PackedCache(2, 64, 6, 16, 32, 4, 2, 64, 1e4)
    rows = lambda n: [torch.randn((n, h, 64), device="cuda").to(torch.bfloat16) for h in (4, 2, 2)]
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    c.step(*rows(20), i32([17, 3]))
    assert c.lens.tolist() == [17, 3] and int(c.free_count) == 3
    o, lse = c.step(*rows(0), i32([0, 0]), i32([1, 0]))
    assert o.shape == (0, 4, 64) and lse.shape == (4, 0) and c.lens.tolist() == [0, 3] and int(c.free_count) == 5


def test_captured_decode_loop():
    """Decode steps as one graph that runs on: each replay takes the next token of every sequence."""
    import torch
    from paper_2506_19651_b200.layer import PackedCache
    Hq, Hkv, d, n = 8, 2, 64, 3
    make = lambda: PackedCache(n, 128, 16, 16, 64, Hq, Hkv, d, 1e4)
    torch.manual_seed(0)
    rand = lambda rows: [torch.randn((rows, h, d), device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv)]
    first, steps = rand(40), [rand(3) for _ in range(20)]
    new0, ones = torch.tensor([20, 15, 5], dtype=torch.int32, device="cuda"), torch.ones(n, dtype=torch.int32, device="cuda")
    eager, captured = make(), make()
    for c in (eager, captured):
        c.step(*first, new0)
    want = [eager.step(*x, ones, most=1) for x in steps]
    x = [t.clone() for t in steps[0]]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        o, lse = captured.step(*x, ones, most=1)
    for rows, (wo, wl) in zip(steps, want):
        with torch.cuda.stream(side):
            for t, r in zip(x, rows):
                t.copy_(r)
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, wo) and torch.equal(lse, wl)
    assert captured.lens.tolist() == [40, 35, 25]
