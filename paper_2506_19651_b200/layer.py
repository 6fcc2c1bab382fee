"""One pass of the whole hot path over one layer's tensors, as a user of the library calls it.

Host-side orchestration only (buffer allocation through torch, then the C-ABI calls).  A pass is one call
(pevlm_layer_forward); its steps, in the order of the method, are RoPE at global positions with K and V written to the
caches -> parallel prefill attention (Eq. 3-4) and question attention (Eq. 5).
"""
from __future__ import annotations

from . import binding as pb


def _workspace(alloc, n_bytes):
    """A workspace whose status header (its first 256 bytes) reads as clear before the first call; the rest needs no value."""
    import torch
    ws = alloc((n_bytes,), torch.uint8)
    ws[:256].zero_()
    return ws


def _one_sequence(shape):
    if shape.batch != 1:
        raise ValueError(f"a layer pass is over one sequence, not a batch of {shape.batch}: its buffers hold the rows of one")


class LayerBuffers:
    """Device buffers of one layer pass over one sequence, allocated once and reused across steps."""

    def __init__(self, shape: pb.Shape, device="cuda", alloc=None):
        """`alloc(shape, dtype, zero)` replaces torch.empty / torch.zeros (the tests pass an allocator that puts
        guard bytes around every buffer)."""
        import torch
        s = shape
        _one_sequence(s)
        nv, Q, L = s.n_video, s.query_len, s.L
        Hq, Hkv, d = s.num_q_heads, s.num_kv_heads, s.head_dim
        bf, f32 = torch.bfloat16, torch.float32
        if alloc is None:
            def alloc(shp, dtype, zero=False):
                return (torch.zeros if zero else torch.empty)(shp, dtype=dtype, device=device)
        self.shape = s
        self.q_video = alloc((max(nv, 1), Hq, d), bf)   # roped copy of the video queries
        self.q_question = alloc((max(Q, 1), Hq, d), bf)
        self.k_cache = alloc((L, Hkv, d), bf)
        self.v_cache = alloc((L, Hkv, d), bf)
        self.o_video = alloc((max(nv, 1), Hq, d), bf)
        self.lse_video = alloc((Hq, max(nv, 1)), f32)
        self.o_question = alloc((max(Q, 1), Hq, d), bf)
        self.lse_question = alloc((Hq, max(Q, 1)), f32)
        self.ws_prefill = _workspace(alloc, pb.pevlm_workspace_bytes(s, pb.WS_PREFILL))
        self.ws_query = _workspace(alloc, pb.pevlm_workspace_bytes(s, pb.WS_QUERY))


def layer_forward(buf: LayerBuffers, q, k, v, mark=None):
    """q [L,Hq,d], k, v [L,Hkv,d]: un-roped bf16 device tensors of the whole stream.
    Leaves O/LSE of the video rows and of the question rows in `buf`.  `mark(name)`, if
    given, is called before the first call and after each C-ABI call (for event timing); without it the pass is one
    call (pevlm_layer_forward)."""
    s = buf.shape
    nv, Q = s.n_video, s.query_len
    _one_sequence(s)
    if mark is None:
        if nv + Q == 0:  # an empty stream is no call's shape
            return buf
        pb.pevlm_layer_forward(s, q, k, v, buf.q_video, buf.q_question, buf.k_cache, buf.v_cache, buf.o_video,
                               buf.lse_video, buf.o_question, buf.lse_question, buf.ws_prefill, buf.ws_query)
        return buf
    mark("start")
    if nv > 0:
        # K goes straight into its cache slot; Q is roped into a scratch copy
        pb.pevlm_rope_qk(s, q[:nv], k[:nv], buf.q_video, buf.k_cache[:nv], 0, nv)
        mark("rope_video")
        pb.pevlm_assemble_kv(s, None, v[:nv], None, None, buf.k_cache, buf.v_cache)
        mark("assemble_video")
        pb.pevlm_parallel_prefill_attn(s, buf.q_video, buf.k_cache[:nv], buf.v_cache[:nv], buf.o_video,
                                       buf.lse_video, buf.ws_prefill)
        mark("prefill_attn")
    if Q > 0:
        pb.pevlm_rope_qk(s, q[nv:], k[nv:], buf.q_question, buf.k_cache[nv:], nv, Q)
        mark("rope_question")
        pb.pevlm_assemble_kv(s, None, None, None, v[nv:], buf.k_cache, buf.v_cache)
        mark("assemble_question")
        pb.pevlm_query_attn(s, buf.q_question, buf.k_cache, buf.v_cache, buf.o_question, buf.lse_question,
                            buf.ws_query)
        mark("query_attn")
    return buf


def ragged_layer_forward(q, k, v, S, B, N, B_last, Q, theta, scale=0.0, alloc=None):
    """Layer pass over a video whose length is not a multiple of the block length: N context blocks, the
    first N-1 of B tokens, the last one of B_last < B tokens (the uniform partition of Sec. 3.2.1 with the
    remainder as one shorter block).  q [L,Hq,d], k, v [L,Hkv,d] un-roped device tensors of the whole
    stream, L = S + (N-1)*B + B_last + Q.  Returns (o_video, lse_video, o_question, lse_question, workspaces), the workspaces
    (for pevlm_read_status) being those of sink and full blocks, of the last block and of the question; the first two are one.

    One call (pevlm_layer_forward with the length of the last block); positions are the global ones.
    `alloc(shape, dtype, zero)` replaces torch.empty / torch.zeros (see LayerBuffers).
    """
    import torch
    Hq, Hkv, d = q.shape[1], k.shape[1], q.shape[2]
    nv = S + (N - 1) * B + B_last
    L = nv + Q
    assert N >= 1 and 1 <= B_last <= B and q.shape[0] == L
    bf, f32 = torch.bfloat16, torch.float32
    s = pb.make_shape(S, B, N, Q, Hq, Hkv, d, theta=theta, scale=scale)
    if alloc is None:
        # (new_empty takes type and device from the tensor: half of torch.empty's time on the host)
        def alloc(shp, dtype, zero=False):
            return q.new_empty(shp) if dtype is q.dtype else q.new_empty(shp, dtype=dtype)
    q_roped = alloc((L, Hq, d), bf)
    k_cache = alloc((L, Hkv, d), bf)
    v_cache = alloc((L, Hkv, d), bf)
    o_video = alloc((nv, Hq, d), bf)
    lse_video = alloc((Hq, nv), f32)
    o_question = alloc((max(Q, 1), Hq, d), bf)
    lse_question = alloc((Hq, max(Q, 1)), f32)
    # the launch writes the status words; a question that is not there leaves its own as it was
    ws_prefill = alloc((pb.pevlm_workspace_bytes(s, pb.WS_PREFILL),), torch.uint8)
    ws_query = (alloc((pb.pevlm_workspace_bytes(s, pb.WS_QUERY),), torch.uint8) if Q > 0
                else _workspace(alloc, pb.pevlm_workspace_bytes(s, pb.WS_QUERY)))
    pb.pevlm_layer_forward(s, q, k, v, q_roped, q_roped[nv:], k_cache, v_cache, o_video, lse_video, o_question, lse_question,
                           ws_prefill, ws_query, last_len=B_last)
    return o_video, lse_video, o_question, lse_question, [ws_prefill, ws_prefill, ws_query]


def _need_rows(n, q, k, v):
    """The calls get addresses only: that there are n rows behind them is seen to here."""
    if q.shape[0] < n or k.shape[0] < n or v.shape[0] < n:
        raise ValueError(f"{q.shape[0]}, {k.shape[0]}, {v.shape[0]} rows of q, k, v where {n} are read")


class StreamingWindow:
    """A sliding window of W context blocks over a fixed sink (the streaming use the paper names as
    future work, Sec. 5).  The cache is [sink | W block slots | question]; block t of the stream is encoded
    once, at its global positions S + t*B ..., against the sink alone (Eq. 4) and replaces the oldest
    block (slot t mod W).  A question attends to the sink and the blocks now in the window (Eq. 5 over the
    window); key order inside the cache does not matter to it because every key carries its own position.
    """

    def __init__(self, S, B, W, Q_max, Hq, Hkv, d, theta, scale=0.0, device="cuda"):
        import torch
        self.S, self.B, self.W, self.Q_max, self.theta, self.scale = S, B, W, Q_max, theta, scale
        self.Hq, self.Hkv, self.d = Hq, Hkv, d
        self.rows = S + W * B + Q_max
        bf, f32 = torch.bfloat16, torch.float32
        self.k_cache = torch.zeros((self.rows, Hkv, d), dtype=bf, device=device)
        self.v_cache = torch.zeros((self.rows, Hkv, d), dtype=bf, device=device)
        self.q_rows = max(S, B, Q_max)
        self.q_buf = torch.empty((self.q_rows, Hq, d), dtype=bf, device=device)
        self.s_sink = self._shape(S, 1, 0, 0)
        self.s_block = self._shape(S, B, 1, 0)
        alloc = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=device)
        self.ws_sink = _workspace(alloc, pb.pevlm_workspace_bytes(self.s_sink, pb.WS_PREFILL))
        self.ws_block = _workspace(alloc, pb.pevlm_workspace_bytes(self.s_block, pb.WS_PREFILL))
        self.ws_query = _workspace(alloc, pb.pevlm_workspace_bytes(self._shape(S + W * B, 1, 0, Q_max), pb.WS_QUERY))
        self.blocks_seen = 0
        self._f32 = torch.empty((0,), dtype=f32, device=device)

    def _outputs(self, n):
        """o [n,Hq,d] and lse [Hq,n] (new_empty, which takes type and device from a tensor, costs the host half of torch.empty)."""
        return self.k_cache.new_empty((n, self.Hq, self.d)), self._f32.new_empty((self.Hq, n))

    def _shape(self, S, B, N, Q):
        return pb.make_shape(S, B, N, Q, self.Hq, self.Hkv, self.d, theta=self.theta, scale=self.scale)

    def _row(self, cache, row):
        """Address of a cache row (what cache[row:] would point to, without building the view)."""
        return cache.data_ptr() + row * self.Hkv * self.d * 2

    def set_sink(self, q, k, v):
        """Encode the sink (Eq. 3).  Returns (o [S,Hq,d], lse [Hq,S])."""
        S = self.S
        _need_rows(S, q, k, v)
        o, lse = self._outputs(S)
        pb.pevlm_rope_qkv(self.s_sink, q, k, v, self.q_buf, self.k_cache, self.v_cache, 0, S)
        pb.pevlm_parallel_prefill_attn(self.s_sink, self.q_buf, self.k_cache, self.v_cache, o, lse, self.ws_sink)
        return o, lse

    def append_block(self, q, k, v):
        """Encode the next block of the stream into the slot of the oldest one.  Returns (o [B,Hq,d], lse [Hq,B])."""
        S, B = self.S, self.B
        _need_rows(B, q, k, v)
        t = self.blocks_seen
        row0 = S + (t % self.W) * B
        o, lse = self._outputs(B)
        pb.pevlm_rope_qkv(self.s_block, q, k, v, self.q_buf, self._row(self.k_cache, row0), self._row(self.v_cache, row0), S + t * B, B)
        pb.pevlm_block_attn(self.s_block, self.q_buf, self.k_cache, self.v_cache, row0, self.rows, o, lse, self.ws_block)
        self.blocks_seen = t + 1
        return o, lse

    def ask(self, q, k, v):
        """Question of Qn <= Q_max tokens at the positions that follow the stream so far, against the sink
        and the blocks in the window (Eq. 5).  Returns (o [Qn,Hq,d], lse [Hq,Qn])."""
        Qn = q.shape[0]
        held = min(self.blocks_seen, self.W)
        nv = self.S + held * self.B
        if k.shape[0] < Qn or v.shape[0] < Qn:
            _need_rows(Qn, q, k, v)
        room = self.rows - nv  # more than Q_max while the window fills
        if Qn > room or Qn > self.q_rows:
            room = min(room, self.q_rows)
            raise ValueError(f"a question of {Qn} rows where {room} fit")
        s = self._shape(nv, 1, 0, Qn)
        o, lse = self._outputs(Qn)
        pb.pevlm_rope_qkv(s, q, k, v, self.q_buf, self._row(self.k_cache, nv), self._row(self.v_cache, nv),
                          self.S + self.blocks_seen * self.B, Qn)
        pb.pevlm_query_attn(s, self.q_buf, self.k_cache, self.v_cache, o, lse, self.ws_query)
        return o, lse


class PackedCache:
    """Keys and values of one layer of many sequences, in pages and in 4 bits: what a server keeps of its videos between questions
    (a 74K-token video of 4 kv heads of 128: 42.6 MB a layer instead of 151.5).  Lengths, page tables, slots and positions live on the
    GPU, so a step may be captured into a graph and replayed with whatever `new_lens` and `finished` hold by then.

    `max_rows` rows at most a step, of all sequences one after another (step() keeps room for as many roped rows of Q and K); `window` > 0 leaves each row the last `window`
    positions and its sequence's first `sink` ones, whose pages all stay the sequence's until it is finished.  Steps follow one another on one stream: the workspace and the roped rows are the object's.  A sequence that finds no pages, or
    whose rows are not all among those that the step brings, keeps its length; its rows get slot -1, output 0 and LSE -inf (see pevlm_pages_assign_rows)."""

    def __init__(self, num_seqs, max_tokens, num_pages, page_len, max_rows, Hq, Hkv, d, theta, window=0, sink=0, scale=0.0, device="cuda"):
        import torch
        if max_rows < 1:
            raise ValueError(f"a step of {max_rows} rows")
        if not 0 <= window < 2 ** 31:
            raise ValueError(f"a window of {window} positions")
        self.pages = pb.make_pages(num_pages, page_len, num_seqs, -(-max_tokens // page_len))
        self.shape = pb.make_shape(sink, 1, 0, 1, Hq, Hkv, d, theta=theta, scale=scale)
        n_bytes = pb.pevlm_packed_cache_bytes(self.shape, self.pages)
        if n_bytes == 0:
            raise ValueError(f"no packed cache of {num_pages} pages of {page_len} tokens for {num_seqs} sequences of {max_tokens}, {Hq}/{Hkv} heads of {d}")
        self.Hq, self.Hkv, self.d, self.window, self.max_rows = Hq, Hkv, d, window, max_rows
        ints = lambda n: torch.zeros(n, dtype=torch.int32, device=device)
        self.cache = torch.zeros(n_bytes, dtype=torch.uint8, device=device)
        self.page_table = torch.full((num_seqs, self.pages.max_pages), -1, dtype=torch.int32, device=device)
        self.free_list = torch.arange(num_pages, dtype=torch.int32, device=device)
        self.lens, self._lens = ints(num_seqs), ints(num_seqs)  # after a step; between its two calls
        self._key_lens = ints(num_seqs)                         # as attend() takes them: 0 for a sequence that was turned away
        self.free_count, self._free_count = torch.full((1,), num_pages, dtype=torch.int32, device=device), ints(1)
        self.row_start, self.slots, self.positions = ints(num_seqs + 1), ints(max_rows) - 1, ints(max_rows)
        self._none = ints(num_seqs)
        self._room = None  # rows of the last extend()
        self._q, self._k = (torch.empty((max_rows, h, d), dtype=torch.bfloat16, device=device) for h in (Hq, Hkv))
        self._lse = torch.empty(0, dtype=torch.float32, device=device)
        n_bytes = pb.pevlm_packed_workspace_bytes(self.shape, self.pages, max_rows, max_rows)
        if n_bytes == 0:
            raise ValueError(f"steps of {max_rows} rows of {Hq}/{Hkv} heads")
        self.workspace = torch.zeros(n_bytes, dtype=torch.uint8, device=device)

    def _rows(self, *tensors):
        n = tensors[0].shape[0]
        if n > self.max_rows or any(t.shape[0] != n for t in tensors):
            raise ValueError(f"{', '.join(str(t.shape[0]) for t in tensors)} rows where at most {self.max_rows} fit, the same of each")
        return n

    def _at_hand(self, *tensors):
        """The calls go to the current device and take addresses: all of it has to be there."""
        import torch
        at = self.cache.device
        if at.type != "cuda" or at.index != torch.cuda.current_device():
            raise ValueError(f"a cache on {at}, which is not the current device")
        for t in tensors:
            if t is not None and t.device != at:
                raise ValueError(f"a tensor on {t.device} beside a cache on {at}")

    def _row_stride(self, t, heads):
        """Elements from one row to the next of rows whose heads stand one after another (the calls get addresses only)."""
        if t.dtype is not self._q.dtype or t.dim() != 3 or t.shape[1:] != (heads, self.d):
            raise ValueError(f"rows of {tuple(t.shape)} ({t.dtype}) where bf16 [n, {heads}, {self.d}] is read")
        if t.stride(2) != 1 or (heads > 1 and t.stride(1) != self.d) or (t.shape[0] > 1 and t.stride(0) < heads * self.d):
            raise ValueError(f"rows with strides {t.stride()}: the {heads} heads of a row have to stand one after another, and rows apart")
        return t.stride(0) if t.shape[0] > 1 else 0

    def _aligned(self, *tensors):
        """What the calls would refuse only after a page call has been made."""
        for t in tensors:
            if t.shape[0] > 0 and (t.data_ptr() % 16 != 0 or t.shape[0] > 1 and t.stride(0) % 8 != 0):
                raise ValueError(f"rows at {t.data_ptr():#x}, {t.stride(0)} elements apart: they are read 16 bytes at a time")

    def _int_per_sequence(self, *tensors):
        for t in tensors:
            if t is not None and (t.numel() != self.pages.num_seqs or t.dtype is not self.lens.dtype or not t.is_contiguous()):
                raise ValueError(f"{t.numel()} of {t.dtype} where an int32 for each of {self.pages.num_seqs} sequences is read")

    def extend(self, new_lens, finished=None, rows=None):
        """Gives back the pages of the `finished` sequences and makes room for new_lens (int32, on the GPU, one for each sequence) more tokens
        of each: row_start, slots and positions say where the rows of the step go; they have to be stored before anything attends to them.  `rows`: as many as store() will bring; a sequence whose
        rows are not all among them is turned away.  Without it there is room for max_rows, and a store() of fewer makes the page call again."""
        if rows is not None and not 0 <= rows <= self.max_rows:
            raise ValueError(f"a step of {rows} rows where at most {self.max_rows} fit")
        self._int_per_sequence(new_lens, finished)
        self._at_hand(new_lens, finished)
        self._room = 0  # nothing to store should one of the two calls be refused
        pb.pevlm_pages_release(self.pages, self._none if finished is None else finished, self.lens, self.page_table, self.free_list,
                               self.free_count, self._lens, self._free_count)
        self._assign(new_lens, self.max_rows if rows is None else rows)

    def _assign(self, new_lens, rows):
        """From the lengths and the free pages between the two page calls of extend(), which the second one leaves as they are."""
        pb.pevlm_pages_assign_rows(self.pages, self._lens, new_lens, self.page_table, self.free_list, self._free_count, self.lens,
                                   self.free_count, self.row_start, self.slots, self.positions, self.max_rows, rows, self._key_lens)
        self._room = rows

    def store(self, k, v):
        """Rows of roped K and of V [n, Hkv, d] (rows may be strided) into the slots of the last extend(): all rows of its step, since a sequence
        whose rows are not all there is turned away (see extend)."""
        n = self._rows(k, v)
        strides = self._row_stride(k, self.Hkv), self._row_stride(v, self.Hkv)
        if self._room is not None and n > self._room:
            raise ValueError(f"{n} rows for a step of {self._room}")
        self._aligned(k, v)
        self._at_hand(k, v)
        if self._room is not None and n < self._room:
            self._assign(self.row_start.diff(), n)  # row_start has kept the new lengths
        pb.pevlm_packed_store(self.shape, self.pages, k, v, self.slots, n, self.cache, *strides)

    def attend(self, q, most=None):
        """Attention of roped q [n, Hq, d], the rows of the last extend().  `most`: rows of one sequence, if the caller knows (64 single tokens of up
        to 16K keys: 72 us, 106 without, where either kernel is launched).
        Rows of a sequence that was turned away have output 0 and LSE -inf, rows of no sequence are not written.  Returns (o [n,Hq,d], lse [Hq,n])."""
        n = self._rows(q)
        stride = self._row_stride(q, self.Hq)
        self._at_hand(q)
        o, lse = q.new_empty((n, self.Hq, self.d)), self._lse.new_empty((self.Hq, n))
        pb.pevlm_packed_attn(self.shape, self.pages, self.window, q, self.cache, self.page_table, self._key_lens, self.row_start, n,
                             n if most is None else min(most, n), o, lse, self.workspace, stride)
        return o, lse

    def step(self, q, k, v, new_lens, finished=None, most=None):
        """One step of the layer from un-roped rows: extend(), RoPE at the rows' positions, store(), attend().  A step that is refused changes nothing."""
        n = self._rows(q, k, v)
        for t, heads in ((q, self.Hq), (k, self.Hkv), (v, self.Hkv)):
            self._row_stride(t, heads)
        if not q.is_contiguous() or not k.is_contiguous():
            raise ValueError("RoPE reads the rows of q and k one after another")
        self._aligned(q, k, v)
        if most is not None and most < 0:
            raise ValueError(f"at most {most} rows of a sequence")
        self._int_per_sequence(new_lens, finished)
        self._at_hand(q, k, v)
        self.extend(new_lens, finished, n)
        if n > 0:
            pb.pevlm_rope_qk(self.shape, q, k, self._q, self._k, 0, n, self.positions)
        self.store(self._k[:n], v)
        return self.attend(self._q[:n], most)

    def load(self, slots):
        """K and V [n, Hkv, d] (bf16) as the cache holds them at the given slots (int32, on the GPU)."""
        if slots.dtype is not self.lens.dtype or not slots.is_contiguous():
            raise ValueError(f"slots of {slots.dtype} where int32 are read")
        self._at_hand(slots)
        n = slots.numel()
        k, v = (self._k.new_empty((n, self.Hkv, self.d)) for _ in range(2))
        pb.pevlm_packed_load(self.shape, self.pages, self.cache, slots, n, k, v)
        return k, v
