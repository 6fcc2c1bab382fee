"""Attention under a sliding window beside the first tokens against 64-bit arithmetic.

Tolerance of an output, derived: the result and the probabilities are rounded to bf16 (2^-8 of each at most; for few rows the result passes an
fp32 merge on the way), the running reference maximum leaves no other error; scores are sums of exact products in fp32: under 64 partial sums
of at most S = sum |q k| lose 2^-24 of it each.  With A = sum p |v| / sum p:  2^-8 |o| + (2^-8 + 2^-20 + 2 * 64 * 2^-24 S scale) A;
of the log-sum-exp 64 * 2^-24 S scale + 2^-20 (1 + |lse|)."""
import numpy as np
import pytest

from helpers import GuardedAllocator, bits_to_f64, to_bits

pytestmark = pytest.mark.gpu


def _bf16(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(torch.bfloat16)


def _values(t):
    return bits_to_f64(to_bits(t)).reshape(t.shape)


def definition(q, k, v, first, window, sink, scale):
    """q [n, Hq, d], k, v [keys, Hkv, d] in 64 bits -> o, lse [n, Hq], and the two parts of the tolerance."""
    n, Hq, d = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    pos, j = first + np.arange(n), np.arange(len(k))
    see = (j <= pos[:, None]) & ((j > pos[:, None] - window) | (j < sink))
    o, a, z, big = np.empty(q.shape), np.empty(q.shape), np.empty((n, Hq)), 0.0
    for h in range(Hq):
        kh, vh = k[:, h // G], v[:, h // G]
        s = q[:, h] @ kh.T * scale
        big = max(big, float((np.abs(q[:, h]) @ np.abs(kh).T).max() * scale))
        s = np.where(see, s, -np.inf)
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        l = p.sum(1, keepdims=True)
        o[:, h], a[:, h] = p @ vh / l, p @ np.abs(vh) / l
        z[:, h] = (top + np.log(l))[:, 0]
    score = 64 * 2.0 ** -24 * big
    return o, z, 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 2.0 ** -20 + 2 * score) * a, score + 2.0 ** -20 * (1 + np.abs(z))


def run(n, first, window, sink, Hq, Hkv, d, batch=1, slack=0, scale=0.0, seed=0, outliers=False, with_lse=True):
    import torch
    from paper_2506_19651_b200 import binding as pb
    rng = np.random.default_rng(seed)
    keys = first + n
    rows = keys + slack
    s = pb.make_shape(sink, 1, 0, 1, Hq, Hkv, d, scale=scale, batch=batch)
    q, k, v = _bf16(rng.standard_normal((batch, n, Hq, d))), rng.standard_normal((batch, rows, Hkv, d)), rng.standard_normal((batch, rows, Hkv, d))
    if outliers:
        k[:, :4] *= 8
        k[:, keys // 2] *= 8
    k[:, keys:], v[:, keys:] = np.nan, np.nan  # rows of the cache that nothing has been written to
    k, v = _bf16(k), _bf16(v)
    guard = GuardedAllocator()
    o, lse = guard((batch, n, Hq, d), torch.bfloat16), guard((batch, Hq, n), torch.float32)
    ws = guard((pb.pevlm_window_workspace_bytes(s, window, first, n),), torch.uint8)
    ws.fill_(0xFF)
    for _ in range(2):
        pb.pevlm_window_attn(s, window, q, k, v, first, n, rows, o, lse if with_lse else None, ws)
    assert pb.pevlm_read_status(ws) == (0, 0)
    guard.check()
    sc = scale or d ** -0.5
    for b in range(batch):
        want, z, tol, tol_z = definition(_values(q)[b], _values(k)[b, :keys], _values(v)[b, :keys], first, window, sink, sc)
        got = _values(o)[b]
        assert np.isfinite(got).all()
        over = np.abs(got - want) - tol
        assert over.max() <= 0, (b, np.unravel_index(over.argmax(), over.shape), over.max())
        if with_lse:
            assert (np.abs(lse[b].double().cpu().numpy().T - z) <= tol_z).all()
    return o, lse


# n, first, window, sink, Hq, Hkv, d
PREFILL = [
    (128, 0, 128, 0, 4, 2, 64), (300, 0, 64, 4, 4, 2, 64), (1000, 0, 1, 0, 2, 1, 128), (777, 0, 100, 5, 7, 1, 128), (513, 0, 128, 128, 4, 2, 128),
    (640, 0, 129, 127, 3, 1, 64), (900, 0, 300, 64, 28, 4, 128), (257, 0, 5000, 3, 4, 2, 64), (600, 0, 200, 1000, 4, 2, 64), (640, 0, 33, 300, 7, 1, 128),
    (200, 1, 150, 16, 14, 2, 128), (150, 700, 128, 8, 7, 1, 128), (129, 333, 77, 130, 5, 1, 64), (48, 1000, 256, 4, 28, 4, 128), (97, 2000, 2 ** 31 - 1, 2, 4, 2, 64),
    (33, 90, 60, 40, 8, 8, 64), (385, 0, 256, 0, 8, 1, 64), (100, 5, 3, 1, 32, 8, 128), (2100, 0, 777, 4, 2, 1, 128),
    # sinks that share the window's first tile and sinks just too long for it, windows of one tile
    (700, 0, 100, 17, 4, 2, 64), (700, 0, 100, 48, 7, 1, 128), (700, 0, 100, 49, 4, 2, 128), (500, 900, 90, 33, 3, 1, 64), (500, 900, 300, 47, 4, 2, 128),
    (40, 500, 10, 5, 8, 8, 64), (40, 500, 10, 48, 8, 8, 128), (40, 500, 1, 16, 8, 8, 128), (129, 500, 2, 1, 4, 4, 64), (300, 40, 9, 31, 5, 1, 128),
]
FEW = [
    (1, 0, 1, 0, 4, 2, 64), (1, 0, 10, 5, 7, 1, 128), (1, 15, 16, 0, 4, 2, 64), (1, 16, 16, 0, 4, 2, 64), (1, 5000, 100, 4, 28, 4, 128), (1, 5000, 4096, 64, 32, 8, 64),
    (4, 3000, 77, 16, 7, 1, 128), (8, 333, 5, 33, 4, 1, 64), (2, 600, 1, 1, 16, 1, 128), (32, 100, 50, 7, 2, 2, 64), (5, 0, 3, 1, 4, 1, 64), (1, 4000, 2 ** 31 - 1, 0, 4, 2, 128),
    (3, 500, 128, 1000, 4, 2, 64), (1, 1000, 999, 1, 4, 4, 128), (16, 1040, 1000, 48, 2, 1, 128),
]


@pytest.mark.parametrize("n,first,window,sink,Hq,Hkv,d", PREFILL)
def test_tiles(n, first, window, sink, Hq, Hkv, d):
    run(n, first, window, sink, Hq, Hkv, d, seed=n)


@pytest.mark.parametrize("n,first,window,sink,Hq,Hkv,d", FEW)
def test_few_rows(n, first, window, sink, Hq, Hkv, d):
    run(n, first, window, sink, Hq, Hkv, d, seed=n + first)


@pytest.mark.parametrize("n,first", [(300, 0), (260, 200), (1, 500), (3, 77)])
def test_batches_slack_and_outliers(n, first):
    run(n, first, 100, 4, 7, 1, 128, batch=3, slack=70, seed=1)
    run(n, first, 64, 6, 4, 2, 64, batch=2, slack=1, seed=2, outliers=True, scale=0.3)
    run(n, first, 64, 0, 4, 2, 64, batch=2, seed=2, with_lse=False)


@pytest.mark.parametrize("n,first,window,sink", [(1, 1000, 100, 5), (4, 777, 33, 0), (3, 500, 17, 20), (300, 900, 100, 5), (150, 2000, 130, 60), (40, 1000, 7, 0)])
@pytest.mark.parametrize("Hq,Hkv,d", [(7, 1, 128), (4, 2, 64)])
def test_keys_that_no_row_sees_may_hold_anything(n, first, window, sink, Hq, Hkv, d):
    """A stream that has left its old rows behind: NaN in every key between the sink and the first row's window."""
    import torch
    from paper_2506_19651_b200 import binding as pb
    torch.manual_seed(n)
    s, keys = pb.make_shape(sink, 1, 0, 1, Hq, Hkv, d), first + n
    q, k, v = (torch.randn((m, h, d), device="cuda").to(torch.bfloat16) for m, h in ((n, Hq), (keys, Hkv), (keys, Hkv)))
    ws = torch.zeros(pb.pevlm_window_workspace_bytes(s, window, first, n), dtype=torch.uint8, device="cuda")
    out = []
    for _ in range(2):
        o, lse = torch.zeros_like(q), torch.zeros((Hq, n), device="cuda")
        pb.pevlm_window_attn(s, window, q, k, v, first, n, keys, o, lse, ws)
        out.append((o, lse))
        k[sink:first - window + 1] = float("nan")
        v[sink:first - window + 1] = float("nan")
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1]) and bool(torch.isfinite(out[1][0]).all())


@pytest.mark.parametrize("n,first", [(3, 400), (200, 400)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_row_that_is_no_number_stays_alone(n, first, value):
    import torch
    from paper_2506_19651_b200 import binding as pb
    torch.manual_seed(n)
    Hq, Hkv, d, window, sink = 6, 2, 64, 100, 5
    s, keys = pb.make_shape(sink, 1, 0, 1, Hq, Hkv, d), first + n
    q, k, v = (torch.randn((m, h, d), device="cuda").to(torch.bfloat16) for m, h in ((n, Hq), (keys, Hkv), (keys, Hkv)))
    ws = torch.zeros(pb.pevlm_window_workspace_bytes(s, window, first, n), dtype=torch.uint8, device="cuda")
    want, z, tol, tol_z = definition(_values(q), _values(k), _values(v), first, window, sink, d ** -0.5)
    q[1, 4] = value
    o, lse = torch.zeros_like(q), torch.zeros((Hq, n), device="cuda")
    pb.pevlm_window_attn(s, window, q, k, v, first, n, keys, o, lse, ws)
    others = np.ones((n, Hq), bool)
    others[1, 4] = False
    got, got_z = _values(o), lse.double().cpu().numpy().T
    assert (np.abs(got - want) <= tol)[others].all() and (np.abs(got_z - z) <= tol_z)[others].all()


@pytest.mark.parametrize("n", [1, 40])
def test_more_sequences_than_a_launch_takes(n):
    """A window of one: each row's output is its own V."""
    import torch
    from paper_2506_19651_b200 import binding as pb
    torch.manual_seed(n)
    batch, first = 33000, 2
    s = pb.make_shape(0, 1, 0, 1, 1, 1, 64, batch=batch)
    q, k, v = (torch.randn((batch, m, 1, 64), device="cuda").to(torch.bfloat16) for m in (n, first + n, first + n))
    o, lse = torch.zeros_like(q), torch.zeros((batch, 1, n), device="cuda")
    ws = torch.zeros(pb.pevlm_window_workspace_bytes(s, 1, first, n), dtype=torch.uint8, device="cuda")
    pb.pevlm_window_attn(s, 1, q, k, v, first, n, first + n, o, lse, ws)
    assert pb.pevlm_read_status(ws) == (0, 0)
    assert bool((o == v[:, first:]).all()) and bool(lse.isfinite().all())


def test_window_of_everything_is_plain_causal():
    """With a window as long as the sequence the rows are those of the full causal prefill, bit for bit."""
    import torch
    from paper_2506_19651_b200 import binding as pb
    n, Hq, Hkv, d = 700, 14, 2, 128
    torch.manual_seed(0)
    q, k, v = (torch.randn((n, h, d), device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
    causal = pb.make_shape(0, n, 1, 0, Hq, Hkv, d, mask_mode=pb.MASK_FULL_CAUSAL)
    o, o2 = torch.empty_like(q), torch.empty_like(q)
    lse, lse2 = torch.empty((Hq, n), device="cuda"), torch.empty((Hq, n), device="cuda")
    ws = torch.zeros(1024, dtype=torch.uint8, device="cuda")
    pb.pevlm_parallel_prefill_attn(causal, q, k, v, o, lse, ws)
    pb.pevlm_window_attn(pb.make_shape(3, 1, 0, 1, Hq, Hkv, d), n, q, k, v, 0, n, n, o2, lse2, ws)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_captured_steps_share_a_workspace():
    import torch
    from paper_2506_19651_b200 import binding as pb
    Hq, Hkv, d, rows, sink, window = 28, 4, 128, 3000, 4, 500
    torch.manual_seed(0)
    s = pb.make_shape(sink, 1, 0, 1, Hq, Hkv, d)
    k, v = (torch.randn((rows, Hkv, d), device="cuda").to(torch.bfloat16) for _ in range(2))
    q = torch.randn((200, Hq, d), device="cuda").to(torch.bfloat16)
    o, lse = torch.empty_like(q), torch.empty((Hq * 200,), device="cuda")
    ws = torch.zeros(pb.pevlm_window_workspace_bytes(s, 1, 0, 1), dtype=torch.uint8, device="cuda")
    calls = [(2999, 1), (2800, 200), (700, 1)]
    want, graphs = [], []
    for first, n in calls:
        pb.pevlm_window_attn(s, window, q, k, v, first, n, rows, o, lse, ws)
        want.append(o[:n].clone())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for first, n in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            pb.pevlm_window_attn(s, window, q, k, v, first, n, rows, o, lse, ws)
    for i in (0, 1, 2, 1, 0, 2):
        o.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(o[:calls[i][1]], want[i])
