"""Device-side plumbing around the C ABI: a compressed cache held in torch
device memory (buffer, segment offsets, head modes, sequence lengths) with
thin methods that queue the library calls.  All arithmetic of the method
runs in the library's kernels.
"""
from __future__ import annotations

import math
from typing import Optional, Sequence

import numpy as np

from . import binding as B


def _torch():
    import torch
    if not torch.cuda.is_available():
        raise RuntimeError("a ROCm GPU is required for the compressed-KV path")
    return torch


def torch_dtype(dtype: str):
    torch = _torch()
    # inputs, queries and outputs: FP8-coefficient caches take bf16 tensors
    return {"bf16": torch.bfloat16, "bf16_e4m3": torch.bfloat16, "f32": torch.float32}[dtype]


def _input_dtype(dims: B.Dims):
    return torch_dtype({B.F32: "f32", B.BF16: "bf16", B.BF16_E4M3: "bf16_e4m3"}[dims.dtype])


def to_device(x: np.ndarray, dtype: str, device="cuda"):
    """float32 numpy values (exactly representable in ``dtype``) -> device tensor."""
    torch = _torch()
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32))
    return t.to(device=device).to(torch_dtype(dtype))


def _allocate(stream, make):
    """``make()``, a tensor that ``stream`` (None: the current one) is to write, from that stream's memory: a block of the
    current stream's may still be in use by what is queued there.  A reader on another stream waits for ``stream`` as for
    any tensor of it."""
    if stream is None:
        return make()
    with _torch().cuda.stream(stream):
        return make()


class CompressedCache:
    """One compressed cache: ``batch`` sequences, modes ``[batch][n_blocks][Hkv]``."""

    def __init__(self, dims: B.Dims, seq_lens: Sequence[int], modes: np.ndarray, device="cuda"):
        torch = _torch()
        self.dims = dims
        self.seq_lens_host = [int(t) for t in seq_lens]
        self.batch = len(self.seq_lens_host)
        self.max_seq_len = max(self.seq_lens_host) if self.seq_lens_host else 0
        self.block_first, self.block_size = B.blocks(dims)
        m = np.ascontiguousarray(modes, dtype=np.uint8).reshape(self.batch, len(self.block_size), dims.n_kv_heads)
        self.modes_host = m
        self.offsets_host, self.total_bytes = B.layout(dims, self.seq_lens_host, m)
        self.buf = torch.empty(max(self.total_bytes, 256), dtype=torch.uint8, device=device)
        self.offsets = torch.from_numpy(self.offsets_host.astype(np.int64)).to(device)
        self.modes = torch.from_numpy(m).to(device)
        self.seq_lens = torch.tensor(self.seq_lens_host, dtype=torch.int32, device=device)
        self.ws = torch.empty(B.decode_workspace(dims, self.batch, self.max_seq_len) // 4 + 64,
                              dtype=torch.float32, device=device)
        self.bounds = None                                  # the index of a sparse decode (``index``)
        self.indexed = [t == 0 for t in self.seq_lens_host]
        self.compressed = [False] * self.batch

    def compress(self, seq: int, k_layers, v_layers, stream=None, token_scores=None, k_select=None):
        """Write sequence ``seq`` from per-layer device tensors ``[Hkv][T][d]`` (``token_scores``
        from the probe when residual heads hold a token-level set; ``k_select`` the probe's K
        selections of the same keys, reused instead of selecting again).  A sequence that is written
        again has to be indexed again, after it, before a sparse decode reads it."""
        if self.compressed[seq]:
            self.indexed[seq] = self.seq_lens_host[seq] == 0
        self.compressed[seq] = True
        B.compress(self.dims, self.seq_lens_host[seq], k_layers, v_layers, self.modes[seq],
                   self.offsets[seq], self.buf, stream, token_scores, k_select)

    def allocate_bounds(self, stream=None):
        """The memory of ``index`` (its first call asks for it; a cache of empty sequences only needs no call)."""
        if self.bounds is not None:
            return
        torch = _torch()
        blocks = max(1, -(-self.max_seq_len // B.BLOCK_TOKENS))
        shape = (self.batch, self.dims.n_kv_heads, blocks, 2, self.dims.head_dim)
        self.bounds = [torch.empty(shape, dtype=_input_dtype(self.dims), device=self.buf.device)
                       for _ in range(self.dims.n_layers)]
        if stream is not None:  # the memory is the current stream's, whose work may still use what lay there before
            stream.wait_stream(torch.cuda.current_stream(self.buf.device))

    def index(self, seq: int, k_layers, stream=None):
        """Key bounds of sequence ``seq``, from the keys that ``compress`` takes: what a sparse decode
        (``Generation`` with ``select``) chooses its blocks by.  ``bounds[l] [batch][Hkv][blocks][2][d]``;
        blocks behind a sequence are left unwritten, as nothing reads them."""
        self.allocate_bounds(stream)
        if self.seq_lens_host[seq]:
            B.key_bounds(self.dims, self.seq_lens_host[seq], k_layers, [b[seq] for b in self.bounds],
                         self.bounds[0].shape[2], stream)
        self.indexed[seq] = True

    def decode(self, layer: int, q, out=None, sm_scale: Optional[float] = None, stream=None):
        """One decode step of ``layer`` for queries ``q [batch][Hq][d]``; returns ``out``."""
        if out is None:
            out = _allocate(stream, lambda: _torch().empty_like(q))
        scale = 1.0 / math.sqrt(self.dims.head_dim) if sm_scale is None else sm_scale
        B.decode_attn(self.dims, self.batch, self.seq_lens, self.max_seq_len, self.modes, self.offsets,
                      self.buf, layer, q, out, scale, self.ws, stream)
        return out

    def host_bytes(self) -> np.ndarray:
        return self.buf[: self.total_bytes].cpu().numpy()


def probe(dims: B.Dims, seq_len: int, k_layers, qp_layers, n_probe: int, stream=None):
    """Queue fdkv_probe and return the device tensor of errors ``[n_blocks][Hkv][n_err]`` and what
    compress of the same keys takes from the probe: for a token-level residual set the token
    scores ``[n_blocks][Hkv][T]``, otherwise the K selections of the pairs."""
    torch = _torch()
    dev = k_layers[0].device
    ws = torch.empty(B.probe_workspace(dims, seq_len, n_probe), dtype=torch.uint8, device=dev)
    nb = len(B.blocks(dims)[0])
    err = torch.empty((nb, dims.n_kv_heads, dims.n_err), dtype=torch.float32, device=dev)
    scores, ksel = None, None
    if dims.residual == B.RES_TOKENS:
        scores = torch.empty((nb, dims.n_kv_heads, seq_len), dtype=torch.float32, device=dev)
    else:
        ksel = torch.empty(max(B.selection_bytes(dims, seq_len), 1), dtype=torch.uint8, device=dev)
    B.probe(dims, seq_len, k_layers, qp_layers, n_probe, err, ws, stream, scores, ksel)
    return err, (scores if scores is not None else ksel)


def _same_cache(a: B.Dims, b: B.Dims) -> bool:
    """Dims of one cache layout (all of it but the query heads)."""
    here = B.Dims.from_buffer_copy(b)
    here.n_q_heads = a.n_q_heads
    return bytes(a) == bytes(here)


class Generation:
    """A compressed cache being extended by decoding (the end of Section 3's
    method): compressed spans (prefill first) followed by an exact tail of
    ``tail_cap`` rows per (sequence, KV head) and layer, which ``refresh``
    compresses into a new span with freshly probed and routed modes.

    A decode step of one token, layer by layer: ``append(layer, k, v)`` puts
    the token's K / V rows at the tail's next row, ``decode(layer, q)``
    attends over every span and the tail including that row; ``advance()``
    then moves the tail position once for all layers.  ``append_rotated``
    stands in for ``append`` where the rows still need their norms and their
    rotation by position.

    ``shared``, a cache of one sequence, is a prefix that all sequences of the
    batch continue: it is held and read once for all of them (``prefix`` may
    then be None, with ``batch`` given).  ``select = (n_first, n_last, n_sel)``
    makes the decode sparse: of ``prefix``, whose sequences have been indexed
    (``CompressedCache.index``), a step reads per KV head the first and last
    blocks of 64 tokens and those that can hold the largest logits, ``n_sel``
    in all; every other span and the tail are read whole.  With either, a
    step's last bits depend on the batch and on the lengths that its launch is
    sized for (fdkv_decode_parts); without, a bf16 sequence's do not.
    """

    def __init__(self, dims: B.Dims, prefix: Optional["CompressedCache"], tail_cap: int, device="cuda",
                 shared: Optional["CompressedCache"] = None, select: Optional[Sequence[int]] = None,
                 batch: Optional[int] = None):
        torch = _torch()
        if prefix is None and (shared is None or batch is None or select is not None):
            raise ValueError("a generation without a prefix of its own takes a shared one and its batch, and selects nothing")
        if prefix is not None and batch not in (None, prefix.batch):
            raise ValueError("the batch is the prefix's")
        if shared is not None and shared.batch != 1:
            raise ValueError("a shared prefix is a cache of one sequence")
        if shared is not None or select is not None:
            if not all(_same_cache(c.dims, dims) for c in (shared, prefix) if c is not None):
                raise ValueError("a prefix of other dimensions, or compressed another way, than the generation")
        if select is not None and not all(prefix.indexed):
            raise ValueError("a sparse decode selects by the prefix's key bounds: index its sequences first")
        if select is not None:
            n_first, n_last, n_sel = select = tuple(int(n) for n in select)
            if n_first < 0 or n_last < 0 or n_sel < max(1, n_first + n_last):
                raise B.FdkvError(-1, f"Generation, select = {select}")
            if n_sel > B.MAX_SELECTED or prefix.batch * dims.n_kv_heads > B.MAX_SELECT_UNITS:
                raise B.FdkvError(-2, f"Generation, select = {select}, batch {prefix.batch}")
        self.dims = dims
        self.batch = prefix.batch if prefix is not None else int(batch)
        self.spans = [prefix] if prefix is not None else []
        self.shared = shared
        self.select = select
        if select is not None:
            prefix.allocate_bounds()
        self.cap = int(tail_cap)
        tdt = _input_dtype(dims)
        shape = (self.batch, dims.n_kv_heads, self.cap, dims.head_dim)
        self.tail_k = [torch.zeros(shape, dtype=tdt, device=device) for _ in range(dims.n_layers)]
        self.tail_v = [torch.zeros(shape, dtype=tdt, device=device) for _ in range(dims.n_layers)]
        self.n_tail = 0                                     # rows held before the current step
        self.pos = torch.zeros(self.batch, dtype=torch.int32, device=device)      # row the step writes
        self.lens = torch.zeros(self.batch, dtype=torch.int32, device=device)     # rows the step attends
        self._ws = None
        if self.select is not None:
            heads = (self.batch, dims.n_kv_heads)
            self.blocks = torch.empty(heads + (self.select[2],), dtype=torch.int32, device=device)    # of the last decode
            self.counts = torch.empty(heads, dtype=torch.int32, device=device)
            n = B.block_select_workspace(dims, self.batch, prefix.max_seq_len)
            self._select_ws = torch.empty(n // 4 + 64, dtype=torch.float32, device=device)
        self._refresh_ws()
        self._begin_step()

    def _refresh_ws(self):
        torch = _torch()
        if self.shared is not None or self.select is not None:
            def part(kind, s, **chosen):
                return B.part(kind, s.seq_lens, s.max_seq_len, s.modes, s.offsets, s.buf, **chosen)
            self._parts = [] if self.shared is None else [part(B.PART_SHARED, self.shared)]
            for i, s in enumerate(self.spans):
                if i == 0 and self.select is not None:
                    self._parts.append(part(B.PART_BLOCKS, s, blocks=self.blocks, counts=self.counts, n_sel=self.select[2]))
                else:
                    self._parts.append(part(B.PART_OWN, s))
            n = B.decode_parts_workspace(self.dims, self.batch, self._parts, self.cap)
            self._ws = torch.empty(n // 4 + 64, dtype=torch.float32, device=self.pos.device)
            return
        n = B.decode_spans_workspace(self.dims, self.batch, [s.max_seq_len for s in self.spans], self.cap)
        self._ws = torch.empty(n // 4 + 64, dtype=torch.float32, device=self.pos.device)
        self._span_desc = [B.Span(int(s.seq_lens.data_ptr()), s.max_seq_len, int(s.modes.data_ptr()),
                                  int(s.offsets.data_ptr()), int(s.buf.data_ptr())) for s in self.spans]

    def _begin_step(self):
        self.pos.fill_(self.n_tail)
        self.lens.fill_(self.n_tail + 1)

    @property
    def full(self) -> bool:
        return self.n_tail >= self.cap

    def append(self, layer: int, k_new, v_new, stream=None):
        """This step's K / V rows ``[batch][Hkv][d]`` of ``layer`` into the tail."""
        if self.full:
            raise RuntimeError("the tail is full: refresh before appending")
        B.append(self.dims, self.batch, self.pos, self.cap, k_new, v_new, self.tail_k[layer], self.tail_v[layer],
                 stream)

    def append_rotated(self, layer: int, rope: B.Rope, q, k_new, v_new, q_norm=None, k_norm=None, eps: float = 1e-6,
                       stream=None, out=None):
        """``append`` of rows as the projections leave them: queries ``q [batch][Hq][d]`` and keys are
        normed per head (where weights are given) and turned by ``rope``, keys and values go into the
        tail.  Heads may lie in one fused projection's rows.  Returns the queries for ``decode`` (``out``)."""
        if self.full:
            raise RuntimeError("the tail is full: refresh before appending")
        if out is None:
            out = _allocate(stream, lambda: _torch().empty(q.shape, dtype=q.dtype, device=q.device))
        B.rope_append(self.dims, rope, q, k_new, v_new, out, None, self.pos, self.tail_k[layer], self.tail_v[layer],
                      q_norm, k_norm, eps, stream)
        return out

    def decode(self, layer: int, q, out=None, sm_scale: Optional[float] = None, stream=None):
        if out is None:
            out = _allocate(stream, lambda: _torch().empty_like(q))
        scale = 1.0 / math.sqrt(self.dims.head_dim) if sm_scale is None else sm_scale
        tail = B.Tail(int(self.lens.data_ptr()), self.cap, int(self.tail_k[layer].data_ptr()),
                      int(self.tail_v[layer].data_ptr()))
        if self.shared is None and self.select is None:
            B.decode_spans(self.dims, self.batch, self._span_desc, tail, layer, q, out, scale, self._ws, stream)
            return out
        if self.select is not None:
            if scale < 0:
                raise ValueError("a sparse decode selects the largest q . k, which a negative scale turns into the least")
            s = self.spans[0]
            if False in s.indexed:
                raise RuntimeError("a sequence of the prefix was compressed again: index it before a sparse decode")
            B.block_select(self.dims, self.batch, s.seq_lens, s.max_seq_len, s.bounds[layer], q, *self.select,
                           self.blocks, self.counts, self._select_ws, stream)
        B.decode_parts(self.dims, self.batch, self._parts, tail, layer, q, out, scale, self._ws, stream)
        return out

    def advance(self):
        """End of a decode step: the appended rows become part of the tail."""
        self.n_tail += 1
        if not self.full:
            self._begin_step()

    def refresh(self, probe_rows, n_probe: int, lam: float = 0.0, budget_bytes: int = 0):
        """Compress the full tail into a new span.  ``probe_rows[l]`` holds the most
        recent decode queries of layer ``l`` as ``[batch][Hq][n_probe][d]``; each
        sequence's span is probed on its own tail keys and routed with ``lam`` (or
        ``budget_bytes`` per sequence).  Returns the new span's modes."""
        torch = _torch()
        nb = len(B.blocks(self.dims)[0])
        T = self.n_tail
        modes = np.zeros((self.batch, nb, self.dims.n_kv_heads), dtype=np.uint8)
        scores = []
        for s in range(self.batch):
            kl = [self.tail_k[l][s, :, :T] if T < self.cap else self.tail_k[l][s] for l in range(self.dims.n_layers)]
            kl = [t.contiguous() for t in kl]
            ql = [probe_rows[l][s].contiguous() for l in range(self.dims.n_layers)]
            err, extra = probe(self.dims, T, kl, ql, n_probe)
            scores.append(extra)
            modes[s], _, _ = B.route(self.dims, T, err.cpu().numpy(), lam=lam, budget_bytes=budget_bytes,
                                     allow_infeasible=True)
        span = CompressedCache(self.dims, [T] * self.batch, modes, device=self.pos.device)
        for s in range(self.batch):
            kl = [self.tail_k[l][s, :, :T].contiguous() for l in range(self.dims.n_layers)]
            vl = [self.tail_v[l][s, :, :T].contiguous() for l in range(self.dims.n_layers)]
            if self.dims.residual == B.RES_TOKENS:
                span.compress(s, kl, vl, token_scores=scores[s])
            else:
                span.compress(s, kl, vl, k_select=scores[s])
        torch.cuda.synchronize()
        self.spans.append(span)
        self.n_tail = 0
        self._refresh_ws()
        self._begin_step()
        return modes


class PagedCache:
    """Exact rows of up to ``batch`` sequences in pages, before (or instead of)
    their compression: prompts as they come in, in pieces of any length, and
    the tokens decoded after them, in one pool of ``n_pages`` pages of ``page``
    rows a layer.  The rows of dims of ``bf16_e4m3`` are held in FP8 with an exponent a
    row.

    A prompt, or its next piece: ``rows = begin(counts)`` takes pages for
    ``counts[s]`` new tokens of every sequence s, ``prompt(rows, layer, q, k, v)``
    stores a layer's rows and attends (causally, over the sequence's earlier
    rows too), and ``end(rows)`` makes them part of the sequences.  A decode step:
    ``begin_step()`` takes a row for each active sequence, ``append(layer, k, v)``
    and ``decode(layer, q)`` store and attend layer by layer, ``advance()`` ends
    it.  ``cancel()`` gives up what has begun, a prompt's rows or a step, whatever
    calls of it were made or failed, and leaves the sequences as they were.
    ``read`` gives a sequence's rows back as ``probe`` and
    ``CompressedCache.compress`` take them, and ``release`` its pages to others.
    ``decode(..., prefix=cache)`` also attends over a compressed prefix that the
    paged rows continue; ``begin_step(prefix=cache)`` then takes a row for the
    sequences that hold tokens of it alone, too.

    ``append`` and ``decode`` of one step can be captured in a graph once and
    replayed every step between ``begin_step`` and ``advance``, which change the
    positions, lengths and tables that the graph reads: captured calls are sized
    for ``max_len`` rows, others for the longest sequence.  All calls go to the
    current stream, and the calls and replays of one cache to one stream (they
    share a workspace).
    """

    def __init__(self, dims: B.Dims, batch: int, max_len: int, n_pages: Optional[int] = None, page: int = 64, device="cuda"):
        torch = _torch()
        self.dims, self.batch, self.page = dims, int(batch), int(page)
        self.max_len = int(max_len)
        most = max(1, -(-self.max_len // self.page))
        self.n_pages = self.batch * most if n_pages is None else int(n_pages)
        shape = (self.n_pages, dims.n_kv_heads, self.page, dims.head_dim)
        c8 = dims.dtype == B.BF16_E4M3
        tdt = torch.uint8 if c8 else _input_dtype(dims)
        self.table = torch.full((self.batch, most), -1, dtype=torch.int32, device=device)
        self.pools = []
        for _ in range(dims.n_layers):
            kv = [torch.zeros(shape, dtype=tdt, device=device) for _ in range(2)]
            exps = [torch.zeros(shape[:3], dtype=torch.uint8, device=device) if c8 else None for _ in range(2)]
            self.pools.append(B.pages(dims, *kv, self.table, *exps))
        self.free = list(range(self.n_pages - 1, -1, -1))
        self.held = [[] for _ in range(self.batch)]         # pages of each sequence
        self.lens_host = [0] * self.batch                   # rows held before the current step
        self.active = [False] * self.batch
        self._by_default = False                            # the active sequences of the step were not named
        self._captured = None                               # the prefix of a captured step
        self._open = None                                   # rows of begin (or True: a step) that have not ended
        self.pos = torch.full((self.batch,), -1, dtype=torch.int32, device=device)  # row that a step writes
        self.lens = torch.zeros(self.batch, dtype=torch.int32, device=device)       # rows that a step attends
        self._ws = torch.empty(B.paged_attn_workspace(dims, self.batch, self.max_len) // 4 + 64, dtype=torch.float32,
                               device=device)

    def _room(self, counts):
        """The pages that each sequence needs for ``counts[s]`` more rows, once it is sure that they can be had."""
        if self._open is not None:
            raise RuntimeError("end the rows, or advance the step, that have begun (or cancel)")
        if len(counts) != self.batch or min(counts) < 0:
            raise ValueError("a number of new rows for each sequence")
        want = [-(-(n + c) // self.page) for n, c in zip(self.lens_host, counts)]
        if any(n + c > self.max_len for n, c in zip(self.lens_host, counts)):
            raise RuntimeError(f"a sequence holds {self.max_len} rows at most")
        if sum(max(0, w - len(h)) for w, h in zip(want, self.held)) > len(self.free):
            raise RuntimeError("the pool has no pages left: release sequences, or compress them")
        return want

    def _take(self, want):
        """``want[s]`` pages for every sequence s, or none where that fails."""
        torch = _torch()
        try:
            for s, w in enumerate(want):
                first = len(self.held[s])
                if w > first:
                    new = [self.free.pop() for _ in range(w - first)]
                    self.held[s] += new
                    self.table[s, first:w] = torch.tensor(new, dtype=torch.int32).to(self.table.device)
        except BaseException:
            self._give_back()
            raise

    def _give_back(self):
        """Pages behind the rows that their sequences hold are free."""
        for s in reversed(range(self.batch)):               # (the order that they were taken in, backwards)
            keep = -(-self.lens_host[s] // self.page)
            if len(self.held[s]) > keep:
                self.free += reversed(self.held[s][keep:])
                del self.held[s][keep:]
                self.table[s, keep:].fill_(-1)

    def release(self, seq: int):
        """Sequence ``seq`` ends: its pages are free, it holds no rows."""
        if self._open is not None:
            raise RuntimeError("end the rows, or advance the step, that have begun (or cancel)")
        self.free += reversed(self.held[seq])
        self.held[seq] = []
        self.lens_host[seq] = 0
        self.active[seq] = False
        self.table[seq].fill_(-1)
        self.pos[seq].fill_(-1)
        self.lens[seq].fill_(0)

    def _pass(self, call, layer: int, k, v, seqs, rows):
        """``call``, page_write or page_read, over as many rows at a time as it takes."""
        most = max(1, B.MAX_PAGE_GROUPS // self.dims.n_kv_heads) * 8
        if len(rows) <= most:
            call(self.dims, self.pools[layer], k, v, seqs, rows)
            return
        for a in range(0, len(rows), most):
            at = slice(a, a + most)
            call(self.dims, self.pools[layer], k[at], v[at], seqs[at], rows[at])

    # ------------------------------------------------------------ prompts
    def begin(self, counts: Sequence[int]):
        """Takes pages for ``counts[s]`` new tokens of every sequence (packed in the order of the sequences in the calls
        that follow) and returns what ``prompt`` needs to know of them."""
        torch = _torch()
        counts = [int(c) for c in counts]
        want = self._room(counts)

        class Rows:
            pass
        r, dev = Rows(), self.table.device
        part = [s for s in range(self.batch) if counts[s]]
        past = [self.lens_host[s] for s in part]
        new = [counts[s] for s in part]
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        k_lens = np.array([a + b for a, b in zip(past, new)], dtype=np.int32)
        firsts = np.concatenate([[0], np.cumsum(k_lens)]).astype(np.int32)

        def put(x):
            return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(dev)

        def spans(first, count):
            return np.concatenate([np.arange(a, a + n) for a, n in zip(first, count)]) if len(count) else np.zeros(0)
        r.counts, r.n, r.total, r.earlier = counts, int(starts[-1]), int(firsts[-1]), sum(past)
        r.starts, r.k_lens, r.k_starts = put(starts), put(k_lens), put(firsts[:-1])
        r.seqs, r.rows = put(np.repeat(part, new)), put(spans(past, new))
        if r.earlier:                                       # every row of the sequences, and where the new ones lie among them
            r.all_seqs, r.all_rows = put(np.repeat(part, k_lens)), put(spans([0] * len(part), k_lens))
            r.new_at = torch.from_numpy(spans(firsts[:-1] + past, new).astype(np.int64)).to(dev)
        n = B.prompt_attn_workspace(self.dims, r.n, len(part), r.total) if r.n else 0
        r.ws = torch.empty(n // 4 + 64, dtype=torch.float32, device=dev)
        self._take(want)
        self._open = r
        return r

    def prompt(self, rows, layer: int, q, k, v, out=None, sm_scale: Optional[float] = None):
        """Stores the new rows ``k`` / ``v [n][Hkv][d]`` of ``layer`` and returns the attention of ``q [n][Hq][d]`` over them
        and the earlier rows of their sequences.  (The new rows take part as they are given, earlier ones as held;
        a compressed prefix takes no part.)"""
        torch = _torch()
        if rows is not self._open:
            raise RuntimeError("not the rows that have begun")
        d = self.dims
        if q.shape != (rows.n, d.n_q_heads, d.head_dim) or (out is not None and out.shape != q.shape) or \
                not k.shape == v.shape == (rows.n, d.n_kv_heads, d.head_dim):
            raise ValueError(f"q and out are [{rows.n}][Hq][d], k and v [{rows.n}][Hkv][d]: the rows that have begun")
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if rows.n == 0:
            return out
        scale = 1.0 / math.sqrt(self.dims.head_dim) if sm_scale is None else sm_scale
        self._pass(B.page_write, layer, k, v, rows.seqs, rows.rows)
        keys = k.transpose(0, 1)[None], v.transpose(0, 1)[None]
        if rows.earlier:
            shape = (self.dims.n_kv_heads, rows.total, self.dims.head_dim)
            keys = [torch.empty(shape, dtype=k.dtype, device=k.device) for _ in range(2)]
            self._pass(B.page_read, layer, *(x.transpose(0, 1) for x in keys), rows.all_seqs, rows.all_rows)
            if self.dims.dtype == B.BF16_E4M3:
                for both, given in zip(keys, (k, v)):
                    both[:, rows.new_at] = given.transpose(0, 1)
            keys = [x[None] for x in keys]
        B.prompt_attn(self.dims, q, *keys, rows.starts, rows.k_lens, out, scale, rows.ws, k_starts=rows.k_starts)
        return out

    def end(self, rows):
        """The rows of ``begin`` become part of their sequences."""
        if rows is not self._open:
            raise RuntimeError("not the rows that have begun")
        self._open = None
        for s, c in enumerate(rows.counts):
            self.lens_host[s] += c

    # ------------------------------------------------------------ steps
    def _check_prefix(self, prefix: CompressedCache):
        if prefix.batch != self.batch or not _same_cache(prefix.dims, self.dims) or prefix.dims.n_q_heads != self.dims.n_q_heads:
            raise ValueError("a prefix of another batch, other dimensions, or compressed another way")

    def _check_active(self, prefix: CompressedCache, active):
        """A sequence that holds tokens of the prefix alone may be at its first step, or at its end: it is not passed over
        unless the caller says so."""
        alone = [s for s, (t, a) in enumerate(zip(prefix.seq_lens_host, active)) if t and not a]
        if alone:
            raise RuntimeError(f"sequences {alone} hold tokens of the prefix alone: begin the step with it, or name the active ones")

    def begin_step(self, active: Optional[Sequence[bool]] = None, prefix: Optional[CompressedCache] = None):
        """A step of the ``active`` sequences begins: each takes a row.  Default: those that hold rows, or tokens of
        ``prefix``, the compressed cache that the step's ``decode`` is called with."""
        torch = _torch()
        by_default = active is None
        if prefix is not None:
            self._check_prefix(prefix)
        if by_default:
            active = [n > 0 for n in self.lens_host]
            if prefix is not None:
                active = [a or t > 0 for a, t in zip(active, prefix.seq_lens_host)]
            elif self._captured is not None:
                self._check_active(self._captured, active)
        active = [bool(a) for a in active]
        want = self._room([int(a) for a in active])
        now = torch.tensor([[n if a else -1 for n, a in zip(self.lens_host, active)],
                            [n + 1 if a else 0 for n, a in zip(self.lens_host, active)]], dtype=torch.int32).to(self.pos.device)
        self._take(want)
        self._open, self.active, self._by_default = True, active, by_default
        self.pos.copy_(now[0])
        self.lens.copy_(now[1])

    def _in_step(self):
        """Positions and lengths on the device are those of the last step until the next one begins.  (A graph may be
        captured at any time.)"""
        if self._open is not True and not _torch().cuda.is_current_stream_capturing():
            raise RuntimeError("no step has begun")

    def append(self, layer: int, k_new, v_new):
        """This step's K / V rows ``[batch][Hkv][d]`` of ``layer`` (those of sequences that are not active are passed over)."""
        self._in_step()
        B.page_write(self.dims, self.pools[layer], k_new, v_new, None, self.pos)

    def decode(self, layer: int, q, out=None, sm_scale: Optional[float] = None, prefix: Optional[CompressedCache] = None):
        """The step's attention ``[batch][Hq][d]`` of ``layer``: over every active sequence's paged rows, and the tokens of
        ``prefix``, a compressed cache of the same batch (of sequences that were not named active: over the prefix alone)."""
        torch = _torch()
        if q.numel() != self.batch * self.dims.n_q_heads * self.dims.head_dim or (out is not None and out.numel() != q.numel()):
            raise ValueError("decode: q and out are [batch][Hq][d]")
        if out is None:
            out = torch.empty_like(q)
        scale = 1.0 / math.sqrt(self.dims.head_dim) if sm_scale is None else sm_scale
        most = self.max_len
        if not torch.cuda.is_current_stream_capturing():
            most = min(most, -(-max(n + a for n, a in zip(self.lens_host, self.active)) // 256) * 256)
        more, n_more = None, 0
        if prefix is not None:
            self._check_prefix(prefix)
        self._in_step()
        if prefix is not None:
            if self._open is True and self._by_default:
                self._check_active(prefix, self.active)
            if torch.cuda.is_current_stream_capturing():
                self._captured = prefix
            if prefix.max_seq_len:
                B.decode_partial(prefix.dims, self.batch, prefix.seq_lens, prefix.max_seq_len, prefix.modes, prefix.offsets,
                                 prefix.buf, layer, q, scale, prefix.ws)
                more, n_more = prefix.ws, -(-prefix.max_seq_len // B.DECODE_CHUNK)
        B.paged_attn(self.dims, self.pools[layer], self.lens, most, q, out, scale, self._ws, more=more, n_more=n_more)
        return out

    def advance(self):
        """End of a decode step: the appended rows become part of their sequences."""
        if self._open is not True:
            raise RuntimeError("no step has begun")
        self._open = None
        for s, a in enumerate(self.active):
            self.lens_host[s] += int(a)
        self.active = [False] * self.batch

    def cancel(self):
        """What has begun, a prompt's rows or a step, is given up: the sequences hold what they held before it."""
        if self._open is None:
            raise RuntimeError("nothing has begun")
        if self._open is True:                              # (a step that is replayed now writes no row)
            self.pos.fill_(-1)
            self.lens.fill_(0)
        self._open = None
        self.active = [False] * self.batch
        self._give_back()

    # ------------------------------------------------------------ rows back
    def read(self, layer: int, seq: int):
        """K and V rows ``[Hkv][T][d]`` of a sequence, as held."""
        torch = _torch()
        seq = range(self.batch)[seq]                        # (a token of sequence -1 is of none)
        T, dev = self.lens_host[seq], self.table.device
        k, v = (torch.empty((self.dims.n_kv_heads, T, self.dims.head_dim), dtype=_input_dtype(self.dims), device=dev) for _ in range(2))
        if T:
            rows = torch.arange(T, dtype=torch.int32, device=dev)
            self._pass(B.page_read, layer, k.transpose(0, 1), v.transpose(0, 1), torch.full_like(rows, seq), rows)
        return k, v
