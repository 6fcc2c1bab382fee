"""A key/value cache in pages of 4-bit numbers, what fills it and what reads it, and attention under a sliding window.

Four kinds of case:
  pages   page tables, slots and positions of a serving step, built from the sequences' lengths (release, then assign)
  packed  rows of K and V written to their slots in 4 bits, and read back
  attn    attention of each sequence's last rows over the packed cache, optionally under a window
  window  attention of bf16 rows under a sliding window beside the first tokens, which stay visible

The packed format: a value is an e2m1 code (4 bits) times the e4m3 scale of its group of 16 along the head; a page of one
kv head is a run of tiles of 16 tokens, 18 * d bytes each (see `_tile_parts`).
"""
import math

import torch

own = False

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # of the e2m1 codes 0 to 7; bit 3 is the sign


def listed():
    return [
        # a decode step of 64 conversations: one new token each, a few of them done; launch latency counts
        dict(name="pages_decode", kind="pages", seqs=64, page=64, new=1, longest=16384, done=4),
        # a burst of arrivals: 700 requests of up to 1,568 new tokens (two blocks), few of them holding anything yet
        dict(name="pages_arrivals", kind="pages", seqs=700, page=16, new=1568, longest=4096, done=31),
        # the keys and values of one decode step of 64 sequences
        dict(name="packed_step", kind="packed", rows=64, Hkv=4, d=128, page=64, fused=True),
        # a 12.6K-token video, its tokens in order
        dict(name="packed_12k", kind="packed", rows=12608, Hkv=4, d=128, page=64, fused=False),
        # a stack's worth of short heads, an odd number of rows
        dict(name="packed_head64", kind="packed", rows=60001, Hkv=8, d=64, page=16, fused=True),
        # one generated token against a resident 50K-token video
        dict(name="attn_decode_50k", kind="attn", seqs=1, shortest=50240, longest=50240, rows=1, Hq=28, Hkv=4, d=128, page=64, window=0, sink=0),
        # one token for each of 64 conversations of very different lengths
        dict(name="attn_decode_batch", kind="attn", seqs=64, shortest=1, longest=16384, rows=1, Hq=28, Hkv=4, d=128, page=64, window=0, sink=0),
        # short heads, up to 4 drafted tokens a sequence, a window over the recent ones beside the first 64
        dict(name="attn_window_batch", kind="attn", seqs=16, shortest=3000, longest=32768, rows=4, Hq=32, Hkv=8, d=64, page=16, window=4096, sink=64),
        # a question of 256 tokens about a 74K-token video
        dict(name="attn_question_74k", kind="attn", seqs=1, shortest=73984, longest=73984, rows=256, Hq=28, Hkv=4, d=128, page=64, window=0, sink=0),
        # one token of a live stream: the first tokens and the last 4,096
        dict(name="window_decode", kind="window", first=50175, tokens=1, window=4096, sink=64, Hq=28, Hkv=4, d=128, batch=1),
        # a 12.6K-token video under a window of one block, odd sizes
        dict(name="window_12k", kind="window", first=0, tokens=12561, window=777, sink=4, Hq=28, Hkv=4, d=128, batch=1),
        # a 50K-token video, window of 2,048
        dict(name="window_50k", kind="window", first=0, tokens=50176, window=2048, sink=64, Hq=28, Hkv=4, d=128, batch=1),
    ]


def _between(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        most[c["kind"]] = {k: max(w[k], most.get(c["kind"], w)[k]) for k in w}
    while True:
        kind = rng.choice(["pages", "packed", "attn", "attn", "attn", "window", "window"])
        d = 64 if rng.random() < 0.3 else 128
        Hq, Hkv = rng.choice([(28, 4), (28, 4), (32, 8), (14, 2), (8, 2), (4, 2)])
        page = rng.choice([16, 32, 64, 128])
        window, sink = (_between(rng, 16, 4096), _between(rng, 1, 128)) if rng.random() < 0.5 else (0, 0)
        if kind == "pages":
            seqs = _between(rng, 1, 1500)
            c = dict(kind=kind, seqs=seqs, page=page, new=rng.choice([1, 1, 5, _between(rng, 1, 4096)]), longest=_between(rng, 1, 16384),
                     done=rng.randint(0, seqs // 4))
        elif kind == "packed":
            c = dict(kind=kind, rows=_between(rng, 1, 60001), Hkv=Hkv, d=d, page=page, fused=rng.random() < 0.5)
        elif kind == "attn":
            longest = _between(rng, 1, 73984)
            c = dict(kind=kind, seqs=_between(rng, 1, 64), shortest=_between(rng, 1, longest), longest=longest,
                     rows=rng.choice([1, 1, 2, 5, _between(rng, 1, 256)]), Hq=Hq, Hkv=Hkv, d=d, page=page, window=window, sink=sink)
        else:
            tokens = rng.choice([1, 3, _between(rng, 1, 50176), _between(rng, 64, 50176)])
            c = dict(kind=kind, first=rng.choice([0, _between(rng, 1, 50176)]), tokens=tokens, window=window or 1000, sink=sink, Hq=Hq, Hkv=Hkv,
                     d=d, batch=rng.choice([1, 1, 2, 3]))
        w = work(c)
        if all(w[k] <= most[kind][k] for k in w) and _scores(c) <= 3.8e9:
            return c


def _scores(c):
    """Numbers of the largest tensor that the plain form makes."""
    if c["kind"] == "attn":
        return c["seqs"] * c["longest"] * max(c["Hq"] * c["rows"], 2 * c["Hkv"] * c["d"])
    if c["kind"] == "window":
        chunk = _chunk(c)
        chunks = -(-c["tokens"] // chunk)
        return c["batch"] * c["Hq"] * chunks * chunk * (c["sink"] + chunk + c["window"])
    return 0


def _lengths(c):
    """Tokens that each sequence holds, spread over [shortest, longest]: the same in every state of a case."""
    n, lo, hi = c["seqs"], c["shortest"], c["longest"]
    return [int(round(lo + (hi - lo) * ((i * 37) % n) / max(1, n - 1))) for i in range(n)]


def _rows(c):
    """Rows of each sequence in this call: 1 to c["rows"], never more than it holds."""
    if c["rows"] == 1 or c["seqs"] == 1:
        return [min(c["rows"], x) for x in _lengths(c)]
    return [min(1 + (i * 5) % c["rows"], x) for i, x in enumerate(_lengths(c))]


def _visible(pos, window, sink):
    """Keys that a row at this position sees."""
    keys = pos + 1
    if window and window < keys:
        first = keys - window
        return window + min(sink, first)
    return keys


def work(c):
    """Each input byte read once and each output byte written once; 4 d flops for each visible (row, key) pair and head."""
    kind = c["kind"]
    if kind == "pages":
        # lengths in and out, flags, the slot and the position of every row there is room for, and an entry read and one
        # written for every page taken or given back (lengths and new rows are uniform: half of the longest on average)
        new = c["seqs"] * (1 if c["new"] == 1 else c["new"] / 2)
        taken, given = new / c["page"], c["done"] * c["longest"] / 2 / c["page"]
        return {"bytes": 4 * (5 * c["seqs"] + 2 * c["seqs"] * c["new"] + 2 * taken + 2 * given), "flops": 0}
    if kind == "packed":
        # bf16 rows in, 4.5 bits a value out, and both the other way round
        values = 2 * c["rows"] * c["Hkv"] * c["d"]
        return {"bytes": 2 * values * (2 + 4.5 / 8) + 8 * c["rows"], "flops": 0}
    Hq, Hkv, d, window, sink = c["Hq"], c["Hkv"], c["d"], c["window"], c["sink"]
    pairs = keys = rows = 0
    if kind == "attn":
        for length, n in zip(_lengths(c), _rows(c)):
            pairs += sum(_visible(p, window, sink) for p in range(length - n, length))
            keys += min(length, _visible(length - 1, window, sink) + n - 1)
            rows += n
        key_bytes = 2 * Hkv * d * 4.5 / 8
    else:
        first, n, b = c["first"], c["tokens"], c["batch"]
        full = max(0, first + n - max(first, window + sink))  # rows that see exactly window + sink keys
        pairs = b * (full * (window + sink) + sum(_visible(p, window, sink) for p in range(first, first + n - full)))
        keys = b * min(first + n, _visible(first + n - 1, window, sink) + n - 1)
        rows = b * n
        key_bytes = 2 * Hkv * d * 2
    return {"bytes": keys * key_bytes + rows * Hq * (4 * d + 4), "flops": 4 * d * Hq * pairs}


# ---------------------------------------------------------------- the packed format

def _tile_parts(cache, d):
    """The four parts of every tile of a cache [..., 18 d] as bytes, token-major: K codes [..., 16, d/2], V codes the same, K
    scales [..., 16, d/16], V scales the same.  In a tile K codes stand token by token; V codes by (half of the tokens, eighth
    of the head, token); the scales so that those one thread needs are neighbours."""
    n, lead = d // 16, cache.shape[:-1]
    kc, vc, ks, vs = cache.split([8 * d, 8 * d, d, d], dim=-1)
    b = len(lead)
    ax = list(range(b))
    kc = kc.reshape(*lead, 16, d // 2)
    vc = vc.reshape(*lead, 2, 8, 8, n).permute(*ax, b, b + 2, b + 1, b + 3).reshape(*lead, 16, d // 2)
    ks = ks.reshape(*lead, 8, 4, 2, n // 4).permute(*ax, b + 2, b, b + 1, b + 3).reshape(*lead, 16, n)
    vs = vs.reshape(*lead, n, 4, 2, 2).permute(*ax, b + 2, b + 1, b + 3, b).reshape(*lead, 16, n)
    return kc, vc, ks, vs


def _tiles(kc, vc, ks, vs, d):
    """The tiles of those parts: what _tile_parts takes apart."""
    n, lead = d // 16, kc.shape[:-2]
    b = len(lead)
    ax = list(range(b))
    vc = vc.reshape(*lead, 2, 8, 8, n).permute(*ax, b, b + 2, b + 1, b + 3)
    ks = ks.reshape(*lead, 2, 8, 4, n // 4).permute(*ax, b + 1, b + 2, b, b + 3)
    vs = vs.reshape(*lead, 2, 4, 2, n).permute(*ax, b + 3, b + 1, b, b + 2)
    return torch.cat([x.reshape(*lead, -1) for x in (kc, vc, ks, vs)], dim=-1)


def _nibbles(codes):
    """[..., n] bytes to [..., 2 n] codes, the low half of a byte first."""
    return torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)


def _quantise(x):
    """Codes [..., d] (a byte each) and scales [..., d/16] (e4m3) of x [..., d]."""
    g = x.float().unflatten(-1, (-1, 16))
    top = g.abs().amax(-1)
    scale = (top.double() / 6).clamp(2.0 ** -9, 448).float().to(torch.float8_e4m3fn)
    y = g.abs() / scale.float().unsqueeze(-1)
    # halfway between two magnitudes the even code is taken
    code = (y > 0.25).byte() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5)
    return (code + 8 * torch.signbit(g).byte()).flatten(-2), scale


def _values(codes, scales):
    """What codes [..., d] with scales [..., d/16] (e4m3) stand for."""
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=codes.device)
    return (table[codes.long()].unflatten(-1, (-1, 16)) * scales.float().unsqueeze(-1)).flatten(-2)


# ---------------------------------------------------------------- states

def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, st = c["kind"], {"c": c}
    if kind == "pages":
        n, P = c["seqs"], c["page"]
        lens = torch.randint(0, c["longest"] + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)
        new = torch.randint(0, c["new"] + 1, (n,), generator=gen, device="cuda", dtype=torch.int32) if c["new"] > 1 else torch.ones_like(lens)
        most = -(-(c["longest"] + c["new"]) // P)
        pages = n * most
        order = torch.randperm(pages, generator=gen, device="cuda").int()
        held = (lens + P - 1) // P
        start = held.cumsum(0) - held
        cols = torch.arange(most, device="cuda")
        table = torch.where(cols < held[:, None], order[(start[:, None] + cols).clamp(max=pages - 1)], -1).int()
        used = int(held.sum())
        free = torch.cat([order[used:], torch.full((used,), -1, dtype=torch.int32, device="cuda")])
        done = torch.zeros_like(lens)
        done[torch.randperm(n, generator=gen, device="cuda")[:c["done"]]] = 1
        new = torch.where(done != 0, 0, new).int()
        rows = n * c["new"]
        st |= {"lens": lens, "new": new, "table": table, "free": free, "count": _ints([pages - used]), "done": done, "pages": pages, "most": most,
               "lens_mid": torch.empty_like(lens), "lens_out": torch.empty_like(lens), "count_mid": _ints([0]), "count_out": _ints([0]),
               "row_start": torch.empty(n + 1, dtype=torch.int32, device="cuda"),
               "slots": torch.empty(rows, dtype=torch.int32, device="cuda"), "positions": torch.empty(rows, dtype=torch.int32, device="cuda")}
    elif kind == "packed":
        rows, Hkv, d, P = c["rows"], c["Hkv"], c["d"], c["page"]
        pages = -(-rows // P) + 3
        if c["fused"]:  # K and V as they leave one projection: row by row beside each other
            st["kv"] = _normal(gen, rows, 2, Hkv, d)
            st["k"], st["v"] = st["kv"][:, 0], st["kv"][:, 1]
        else:
            st["k"], st["v"] = _normal(gen, rows, Hkv, d), _normal(gen, rows, Hkv, d)
        st["k"][::7, :, :16] *= 8  # a few large channels, as keys have
        table = torch.randperm(pages, generator=gen, device="cuda").int()
        at = torch.arange(rows, device="cuda") + P // 2  # starts in the middle of a page
        st["slots"] = (table[at // P] * P + at % P).int()
        st["slots"][torch.rand(rows, generator=gen, device="cuda") < 0.002] = -1  # padding
        st["pages"] = pages
        st["cache"] = torch.zeros((pages, Hkv, P // 16, 18 * d), dtype=torch.uint8, device="cuda")
        st["k_out"] = torch.empty((rows, Hkv, d), dtype=torch.bfloat16, device="cuda")
        st["v_out"] = torch.empty_like(st["k_out"])
    elif kind == "attn":
        Hq, Hkv, d, P = c["Hq"], c["Hkv"], c["d"], c["page"]
        lens, rows = _lengths(c), _rows(c)
        held = [-(-x // P) for x in lens]
        pages, most = sum(held) + 2, max(held) + 1
        order = torch.randperm(pages, generator=gen, device="cuda").int()
        held = torch.tensor(held, device="cuda")
        start = held.cumsum(0) - held
        cols = torch.arange(most, device="cuda")
        st["table"] = torch.where(cols < held[:, None], order[(start[:, None] + cols).clamp(max=pages - 1)], -1).int()
        st["cache"] = torch.empty((pages, Hkv, P // 16, 18 * d), dtype=torch.uint8, device="cuda")
        step = max(1, (1 << 27) // (Hkv * P * d))
        for p in range(0, pages, step):  # the cache of N(0, 1) keys and values
            m = min(step, pages - p)
            (kc, ks), (vc, vs) = (_quantise(torch.randn((m, Hkv, P // 16, 16, d), generator=gen, device="cuda")) for _ in range(2))
            kc, vc = (x[..., 0::2] | x[..., 1::2] << 4 for x in (kc, vc))
            st["cache"][p:p + m] = _tiles(kc, vc, ks.view(torch.uint8), vs.view(torch.uint8), d)
        total = sum(rows)
        st["q"] = _normal(gen, total, Hq, d)
        st["lens"], st["pages"], st["most"] = _ints(lens), pages, most
        st["row_start"] = _ints([0] + torch.tensor(rows).cumsum(0).tolist())
        st["total"], st["max_rows"], st["max_len"] = total, max(rows), max(lens)
        st["o"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty((Hq, total), dtype=torch.float32, device="cuda")
    else:
        Hq, Hkv, d, b, n, first = c["Hq"], c["Hkv"], c["d"], c["batch"], c["tokens"], c["first"]
        st["q"] = _normal(gen, b * n, Hq, d)
        st["k"], st["v"] = _normal(gen, b * (first + n), Hkv, d), _normal(gen, b * (first + n), Hkv, d)
        st["o"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty((b, Hq, n), dtype=torch.float32, device="cuda")
    return st


# ---------------------------------------------------------------- one pass

def run(st):
    if own:
        return _run_own(st)
    return {"pages": _plain_pages, "packed": _plain_packed, "attn": _plain_attn, "window": _plain_window}[st["c"]["kind"]](st)


def _run_own(st):
    from paper_2506_19651_b200 import binding as pb
    c = st["c"]
    kind = c["kind"]
    if "shape" not in st:  # what a program keeps beside its inputs: shapes and a workspace
        if kind != "packed":
            st["geometry"] = pb.make_pages(st.get("pages", 1), c.get("page", 16), c.get("seqs", 1), st.get("most", 1))
        else:
            st["geometry"] = pb.make_pages(st["pages"], c["page"], 1, st["pages"])
        st["shape"] = pb.make_shape(c.get("sink", 0), 1, 0, 1, c.get("Hq", c.get("Hkv", 1)), c.get("Hkv", 1), c.get("d", 64), batch=c.get("batch", 1))
        if kind in ("attn", "window"):
            size = (pb.pevlm_packed_workspace_bytes(st["shape"], st["geometry"], st["total"], st["max_rows"]) if kind == "attn"
                    else pb.pevlm_window_workspace_bytes(st["shape"], c["window"], c["first"], c["tokens"]))
            st["ws"] = torch.zeros(size, dtype=torch.uint8, device="cuda")
    s, g = st["shape"], st["geometry"]
    if kind == "pages":
        pb.pevlm_pages_release(g, st["done"], st["lens"], st["table"], st["free"], st["count"], st["lens_mid"], st["count_mid"])
        pb.pevlm_pages_assign(g, st["lens_mid"], st["new"], st["table"], st["free"], st["count_mid"], st["lens_out"], st["count_out"],
                              st["row_start"], st["slots"], st["positions"], st["slots"].numel())
        return [st[k] for k in ("lens_out", "count_out", "row_start", "slots", "positions", "table", "free")]
    if kind == "packed":
        pb.pevlm_packed_store(s, g, st["k"], st["v"], st["slots"], c["rows"], st["cache"], st["k"].stride(0), st["v"].stride(0))
        pb.pevlm_packed_load(s, g, st["cache"], st["slots"], c["rows"], st["k_out"], st["v_out"])
        return [st["k_out"], st["v_out"]]
    if kind == "attn":
        pb.pevlm_packed_attn(s, g, c["window"], st["q"], st["cache"], st["table"], st["lens"], st["row_start"], st["total"], st["max_rows"],
                             st["o"], st["lse"], st["ws"])
    else:
        n = c["first"] + c["tokens"]
        pb.pevlm_window_attn(s, c["window"], st["q"], st["k"], st["v"], c["first"], c["tokens"], n, st["o"], st["lse"], st["ws"])
    return [st["o"], st["lse"]]


def _plain_pages(st):
    c = st["c"]
    n, P, rows = c["seqs"], c["page"], st["slots"].numel()
    lens, new, count = st["lens"].long(), st["new"].long(), st["count"].long()
    cols = torch.arange(st["most"], device="cuda")
    # release: the pages of the sequences that are done go on top of the free list, in order
    given = torch.where(st["done"] != 0, (lens + P - 1) // P, 0)
    at = count + (given.cumsum(0) - given)[:, None] + cols
    held = cols < given[:, None]
    free = torch.cat([st["free"].long(), lens.new_zeros(1)])
    free = free.scatter(0, torch.where(held, at, st["pages"]).flatten(), st["table"].long().flatten())[:-1]
    lens, count = torch.where(st["done"] != 0, 0, lens), count + given.sum()
    # assign: pages from the top of the free list, in the order of the sequences
    have = (lens + P - 1) // P
    need = (lens + new + P - 1) // P - have
    before = need.cumsum(0) - need
    fits = (need == 0) | (before + need <= count)
    col = cols - have[:, None]
    fresh = (col >= 0) & (col < need[:, None]) & fits[:, None]
    table = torch.where(fresh, free[(count - 1 - before[:, None] - col).clamp(0, st["pages"] - 1)], st["table"].long())
    ends = new.cumsum(0)
    row_start = torch.cat([ends.new_zeros(1), ends])
    row = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(ends, row, right=True)
    there = seq < n
    seq = seq.clamp(max=n - 1)
    pos = lens[seq] + row - row_start[seq]
    ok = there & fits[seq]
    slots = torch.where(ok, table[seq, (pos // P).clamp(max=st["most"] - 1)] * P + pos % P, -1)
    positions = torch.where(there, pos, 0)
    out = (torch.where(fits, lens + new, lens), count - torch.where(fits, need, 0).sum(), row_start, slots, positions, table, free)
    return [x.int() for x in out]


def _plain_packed(st):
    kept = (st["slots"] >= 0)[:, None, None]
    return [torch.where(kept, _values(*_quantise(st[x])), 0.0).to(torch.bfloat16) for x in ("k", "v")]


def _attend(q, k, v, mask, dtype):
    """q [b, h, rows, d], k, v [b, h, keys, d], mask broadcast over [b, h, rows, keys]: outputs and log-sum-exp in `dtype`."""
    s = q.to(dtype) @ k.to(dtype).transpose(-1, -2) / math.sqrt(q.shape[-1])
    s = s.masked_fill_(~mask, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = p @ v.to(dtype) / torch.where(total > 0, total, 1.0)
    return o, (top + total.log()).squeeze(-1)


def _plain_attn(st):
    c = st["c"]
    Hq, Hkv, d, P = c["Hq"], c["Hkv"], c["d"], c["page"]
    n, rows, G = c["seqs"], st["max_rows"], c["Hq"] // c["Hkv"]
    cols = -(-st["max_len"] // P)
    pages = st["cache"][st["table"][:, :cols].long().clamp(min=0)]  # [n, cols, Hkv, tiles, 18 d]
    kc, vc, ks, vs = _tile_parts(pages.transpose(1, 2).flatten(2, 3), d)
    k = _values(_nibbles(kc), ks.contiguous().view(torch.float8_e4m3fn)).flatten(2, 3)  # [n, Hkv, keys, d]
    v = _values(_nibbles(vc), vs.contiguous().view(torch.float8_e4m3fn)).flatten(2, 3)
    lens, row_start = st["lens"].long(), st["row_start"].long()
    here = row_start[1:] - row_start[:-1]
    i = torch.arange(rows, device="cuda")
    q = st["q"][(row_start[:-1, None] + i).clamp(max=st["total"] - 1)]  # [n, rows, Hq, d]
    q = q.reshape(n, rows, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * rows, d)
    pos = (lens - here)[:, None] + i
    j = torch.arange(k.shape[2], device="cuda")
    mask = (j <= pos[..., None]) & (j < lens[:, None, None])
    if c["window"]:
        mask &= (j > pos[..., None] - c["window"]) | (j < c["sink"])
    o, lse = _attend(q, k, v, mask[:, None].repeat(1, 1, G, 1), torch.float32)
    o = o.reshape(n, Hq, rows, d)
    lse = lse.reshape(n, Hq, rows)
    row = torch.arange(st["total"], device="cuda")
    seq = torch.searchsorted(row_start[1:], row, right=True)
    at = row - row_start[seq]
    return [o[seq, :, at].to(torch.bfloat16), lse[seq, :, at].T.contiguous()]


def _chunk(c):
    """Rows that the plain form takes together: as many as a window has, so that half of what it computes is seen."""
    return min(c["tokens"], max(64, min(1024, c["window"])))


def _plain_window(st):
    """Rows in chunks; the keys of a chunk are the sink and the run of keys that ends with its last row."""
    c = st["c"]
    Hq, Hkv, d, b, n, first, window, sink = (c[x] for x in ("Hq", "Hkv", "d", "batch", "tokens", "first", "window", "sink"))
    G, chunk = Hq // Hkv, _chunk(c)
    chunks = -(-n // chunk)
    run_ = chunk + window
    start = first - window + chunk * torch.arange(chunks, device="cuda")  # of each chunk's run
    j = start[:, None] + torch.arange(run_, device="cuda")
    inside = (j >= 0) & (j < first + n)

    def keys(x):
        x = x.reshape(b, first + n, Hkv, d)
        own_run = x[:, j.clamp(0, first + n - 1)]                  # [b, chunks, run, Hkv, d]
        shared = x[:, None, :min(sink, first + n)].expand(-1, chunks, -1, -1, -1)
        return torch.cat([shared, own_run], 2).permute(0, 1, 3, 2, 4).flatten(0, 1).float()

    row = torch.arange(chunks * chunk, device="cuda")
    q = st["q"].reshape(b, n, Hkv, G, d)[:, row.clamp(max=n - 1)]
    q = q.reshape(b, chunks, chunk, Hkv, G, d).permute(0, 1, 3, 4, 2, 5).reshape(b * chunks, Hkv, G * chunk, d)
    pos = first + row.reshape(chunks, chunk)[:, :, None]
    first_keys = torch.arange(min(sink, first + n), device="cuda")
    seen_run = inside[:, None] & (j[:, None] <= pos) & (j[:, None] > pos - window)
    seen_first = (first_keys <= pos) & (first_keys <= pos - window)  # the others of the sink are in the run
    mask = torch.cat([seen_first, seen_run], 2)[:, None].repeat(b, 1, G, 1)
    o, lse = _attend(q, keys(st["k"]), keys(st["v"]), mask, torch.float32)
    o = o.reshape(b, chunks, Hkv, G, chunk, d).permute(0, 1, 4, 2, 3, 5).reshape(b, chunks * chunk, Hq, d)[:, :n]
    lse = lse.reshape(b, chunks, Hq, chunk).permute(0, 2, 1, 3).reshape(b, Hq, chunks * chunk)[:, :, :n]
    return [o.reshape(b * n, Hq, d).to(torch.bfloat16), lse.contiguous()]


# ---------------------------------------------------------------- the definition in 64 bits

def _byte_values():
    """The 256 e4m3 numbers in 64 bits, from their bits."""
    b = torch.arange(256, device="cuda")
    e, m = (b >> 3) & 15, (b & 7).double()
    v = torch.where(e > 0, torch.ldexp(8 + m, e - 10), m * 2.0 ** -9)
    return torch.where(b >= 128, -v, v)


def exact(c, seed):
    def sequence(q, pos, k, v, length, window, sink, Hkv):
        """q [rows, Hq, d] at positions pos against k, v [keys, Hkv, d], all in 64 bits, a few rows at a time."""
        rows, Hq, d = q.shape
        G = Hq // Hkv
        o, lse = torch.empty_like(q), q.new_empty((Hq, rows))
        step = max(1, min(256, (1 << 28) // max(1, G * length)))
        for r in range(0, rows, step):
            at = pos[r:r + step]
            lo = 0
            if window:
                lo = max(0, int(at[0]) - window + 1)
            hi = int(at[-1]) + 1
            j = torch.arange(max(lo, 0), max(hi, 0), device=q.device)
            if window and lo > 0:
                j = torch.cat([torch.arange(min(sink, lo), device=q.device), j])
            see = j <= at[:, None]
            if window:
                see &= (j < sink) | (at[:, None] - j < window)
            for h in range(Hkv):
                heads = slice(h * G, (h + 1) * G)
                s = torch.einsum("rgd,kd->grk", q[r:r + step, heads], k[j, h]) * d ** -0.5
                s[:, ~see] = -math.inf
                z = torch.logsumexp(s, -1)
                lse[heads, r:r + step] = z
                w = torch.exp(s - torch.where(z == -math.inf, 0.0, z)[..., None])
                o[r:r + step, heads] = torch.einsum("grk,kd->rgd", w, v[j, h])
        return o, lse

    st = prepare(c, seed)
    kind = c["kind"]
    if kind == "pages":
        return None
    if kind == "packed":
        scales = _byte_values()[:127]
        grid = torch.tensor(MAGNITUDES, dtype=torch.float64, device="cuda")
        out = []
        for x in (st["k"], st["v"]):
            x = x.double().reshape(-1, 16)
            top = x.abs().amax(1).clamp(6 * 2.0 ** -9, 6 * 448.0)
            # nearest of the ascending scales, and of the magnitudes; halfway, the one with the even number
            def nearest(y, values):
                up = torch.searchsorted(values, y).clamp(1, len(values) - 1)
                below, above = y - values[up - 1], values[up] - y
                return torch.where((below < above) | ((below == above) & ((up - 1) % 2 == 0)), up - 1, up)
            s = scales[nearest(top, 6 * scales)]  # (a division of top by 6 would move it off the halfway points)
            code = nearest((x.abs() / s[:, None]).clamp(max=6.0), grid)
            y = (grid[code] * s[:, None] * torch.sign(x)).reshape(c["rows"], c["Hkv"], c["d"])
            out.append(torch.where((st["slots"] < 0)[:, None, None], torch.zeros_like(y), y))
        return out
    if kind == "attn":
        Hkv, d, P = c["Hkv"], c["d"], c["page"]
        number = _byte_values()
        grid = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), dtype=torch.float64, device="cuda")
        o = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
        row = 0
        for r, (length, n) in enumerate(zip(_lengths(c), _rows(c))):
            pages = st["cache"][st["table"][r, :-(-length // P)].long()]
            kv = []
            for codes, scale in zip(*(lambda p: ((p[0], p[1]), (p[2], p[3])))(_tile_parts(pages, d))):
                x = torch.stack([grid[(codes & 15).long()], grid[(codes >> 4).long()]], -1).flatten(-2)
                x = x * number[scale.long()].repeat_interleave(16, -1)       # [pages, Hkv, tiles, 16, d]
                kv.append(x.transpose(1, 2).transpose(2, 3).reshape(-1, Hkv, d)[:length])
            pos = torch.arange(length - n, length, device="cuda")
            o[row:row + n], lse[:, row:row + n] = sequence(st["q"][row:row + n].double(), pos, kv[0], kv[1], length, c["window"], c["sink"], Hkv)
            row += n
        return [o, lse]
    n, first, b = c["tokens"], c["first"], c["batch"]
    pos = torch.arange(first, first + n, device="cuda")
    o = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["lse"].shape, dtype=torch.float64, device="cuda")
    for i in range(b):
        k, v = (st[x][i * (first + n):(i + 1) * (first + n)].double() for x in ("k", "v"))
        o[i * n:(i + 1) * n], lse[i] = sequence(st["q"][i * n:(i + 1) * n].double(), pos, k, v, min(first + n, c["window"] + c["sink"] + 256), c["window"], c["sink"], c["Hkv"])
    return [o, lse]
