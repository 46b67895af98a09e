"""Self-attention of a transformer layer in 8-bit codes, prompts and single tokens, through the C ABI.

The paper has no counterpart; the block shows the library's 8-bit transformer calls together,
as a server would use them:

    qkv = x W_qkv^T + b_qkv        palquant_linear_q8: 8-bit codes, one scale for each token and channel
    cache <- k, v                  palquant_kv8_append: 8-bit codes, one scale for each page and head
    mixed = attention(q, cache)    palquant_kv8_attention: grouped heads, causal, optional window
    y = mixed W_out^T              palquant_linear_q8

A block serves a fixed set of sequences.  forward() takes any number of new tokens for each of
them (none, one, a chunk or a whole prompt), appends them to the cache and attends from them
to everything cached so far; sequences of different lengths share a call.  reset() ends a
sequence and makes its pages free for the next one.  q, k and v are read where the first layer
wrote them (columns of its output), so nothing is copied between the four calls.

    block = AttentionBlock8(w_qkv, w_out, heads=32, kv_heads=8, sequences=4, max_len=4096)
    y = block.forward(prompts, [900, 17, 2048, 1])    # [2966, hidden]
    y = block.forward(tokens, [1, 1, 1, 1])           # [4, hidden]
"""
from __future__ import annotations

import contextlib

import torch

from . import binding as B

_INDEX_BUFFERS = 16
_TYPES = {torch.float32: B.PQ_F32, torch.float16: B.PQ_F16, torch.bfloat16: B.PQ_BF16}


@contextlib.contextmanager
def _in_turn(device, stream: torch.cuda.Stream | None, *tensors):
    """Inside, `stream` (None: the current one) is current: after what the caller's stream holds and before what it is given
    next.  `tensors`, the caller's, are held until it is done with them."""
    caller = torch.cuda.current_stream(device)
    if stream is None or stream == caller:
        yield caller
        return
    stream.wait_stream(caller)
    for t in tensors:
        t.record_stream(stream)
    with torch.cuda.stream(stream):
        yield stream
    caller.wait_stream(stream)


def _give(device, *tensors) -> None:
    """Tensors made on another stream, held until the current one is done with them."""
    current = torch.cuda.current_stream(device)
    for t in tensors:
        t.record_stream(current)


def weight_codes(w: torch.Tensor, stream: torch.cuda.Stream | None = None):
    """Signed 8-bit codes [N, K] and one scale for each output channel (row) of w: the token quantiser on the rows.  It runs
    on `stream` (None: the current one), after what the current stream holds and before what it is given next."""
    if w.dim() != 2 or w.dtype not in _TYPES or w.stride(1) != 1:
        raise ValueError("w: a float matrix with contiguous rows")
    with _in_turn(w.device, stream, w) as run:
        codes = torch.empty(w.shape, dtype=torch.int8, device=w.device)
        scales = torch.empty(w.shape[0], device=w.device)
        B.palquant_quantize_tokens(w, _TYPES[w.dtype], w.stride(0), w.shape[0], w.shape[1], B.PQ_CODES_INT8, codes,
                                   w.shape[1], scales, run)
    _give(w.device, codes, scales)
    return codes, scales


class AttentionBlock8:
    def __init__(self, w_qkv: torch.Tensor, w_out: torch.Tensor, heads: int, kv_heads: int, sequences: int, max_len: int,
                 b_qkv: torch.Tensor | None = None, page_tokens: int = 64, window: int = 0,
                 stream: torch.cuda.Stream | None = None):
        """w_qkv [(heads + 2 kv_heads) D, hidden] (the rows of q, then k, then v) and w_out [hidden, heads D] on the
        GPU; their type is the activations'.  b_qkv: a value for each row of w_qkv."""
        if w_qkv.dim() != 2 or w_qkv.dtype not in _TYPES or sequences < 1 or max_len < 1 or window < 0 or page_tokens not in (16, 32, 64, 128):
            raise ValueError("w_qkv: a float matrix; at least one sequence and token; window >= 0; page_tokens: 16, 32, 64 or 128")
        if heads < 1 or kv_heads < 1 or heads % kv_heads or w_qkv.shape[0] % (heads + 2 * kv_heads):
            raise ValueError("heads: a multiple of kv_heads; w_qkv: heads + 2 kv_heads blocks of rows")
        self.heads, self.kv_heads, self.window = heads, kv_heads, window
        self.D = w_qkv.shape[0] // (heads + 2 * kv_heads)
        self.hidden = w_qkv.shape[1]
        if self.D % 16 or not 16 <= self.D <= 256:
            raise ValueError("w_qkv: heads of D, a multiple of 16 from 16 to 256")
        if b_qkv is not None and b_qkv.numel() != w_qkv.shape[0]:
            raise ValueError("b_qkv: a value for each row of w_qkv")
        if w_out.shape != (self.hidden, heads * self.D) or w_out.dtype != w_qkv.dtype:
            raise ValueError("w_out: [hidden, heads D], of w_qkv's type")
        self.dtype, self.dev, self.stream = w_qkv.dtype, w_qkv.device, stream
        self.sequences, self.max_len = sequences, max_len
        given = [t for t in (w_qkv, w_out, b_qkv) if t is not None and t.is_cuda]
        with _in_turn(self.dev, stream, *given) as run:
            self.b_qkv = None if b_qkv is None else b_qkv.to(self.dev, torch.float32).contiguous().view(-1)
            w_qkv, w_out = w_qkv.contiguous(), w_out.contiguous()
            self.w_qkv, self.s_qkv = weight_codes(w_qkv, run)
            self.w_out, self.s_out = weight_codes(w_out, run)
            pages = -(-max_len // page_tokens)
            n = sequences * pages
            self.k, self.v = (torch.zeros((n, kv_heads, page_tokens, self.D), dtype=torch.int8, device=self.dev)
                              for _ in range(2))
            self.k_scale, self.v_scale = (torch.zeros((n, kv_heads), device=self.dev) for _ in range(2))
            self.cache = B.kv8_cache(self.k, self.v, self.k_scale, self.v_scale)
            self.table = torch.arange(n, dtype=torch.int32, device=self.dev).view(sequences, pages)
            # a call's positions, page-locked: a copy from pageable memory would wait for the device.  Used in turn, each
            # again once its last copy is over (the host waits only when it is that many calls ahead)
            self._index = torch.empty((_INDEX_BUFFERS, 3 * sequences + 1), dtype=torch.int32, pin_memory=True)
            self._copied = [torch.cuda.Event() for _ in range(_INDEX_BUFFERS)]
            self._calls = 0
            self._own = [t for t in (self.b_qkv, self.w_qkv, self.s_qkv, self.w_out, self.s_out, self.k, self.v, self.k_scale,
                                     self.v_scale, self.table) if t is not None]
            self._ran, self._over = run, torch.cuda.Event()  # the last call's stream, and its end there
            self._over.record(run)
        self.lens = [0] * sequences  # tokens cached, on the host: no call waits for the device to know them

    def _follow(self, run: torch.cuda.Stream) -> None:
        """With no stream of its own the block runs on its callers': after its last call, which held another stream, and
        with its memory held for this one too."""
        if run != self._ran:
            run.wait_event(self._over)
            for t in self._own:
                t.record_stream(run)
            self._ran = run

    def _to_device(self, values, run) -> torch.Tensor:
        """Positions on the device, without waiting for it."""
        i = self._calls % _INDEX_BUFFERS
        self._calls += 1
        self._copied[i].synchronize()  # (returns at once before the first record)
        self._index[i] = torch.tensor(values, dtype=torch.int32)
        index = self._index[i].to(self.dev, non_blocking=True)
        self._copied[i].record(run)
        return index

    def _scratch(self, n: int) -> torch.Tensor:
        """A call's workspace, of its stream's pool."""
        return torch.empty(n, dtype=torch.uint8, device=self.dev)

    def _linear(self, x, w, s_w, bias, y, run):
        d = B.linear_desc(x, w, y)
        work = self._scratch(B.palquant_linear_q8_scratch_bytes(d))
        B.palquant_linear_q8(x, w, s_w, bias, y, d, work, work.numel(), run)

    def reset(self, sequence: int) -> None:
        self.lens[sequence] = 0

    def forward(self, x: torch.Tensor, counts) -> torch.Tensor:
        """x [sum(counts), hidden]: counts[b] new tokens of every sequence b, one sequence after the other; returns y
        of x's shape.  It runs on the block's stream (None: the current one), after what the current stream holds and
        before what it is given next; with the current stream another than the last call's, after that call too."""
        counts = [int(c) for c in counts]
        if len(counts) != self.sequences or min(counts) < 0 or x.shape != (sum(counts), self.hidden) \
                or x.dtype != self.dtype or x.device != self.dev:
            raise ValueError("counts: one for each sequence; x: [sum(counts), hidden] of the weights' type, on their device")
        after = [n + c for n, c in zip(self.lens, counts)]
        if max(after) > self.max_len:
            raise ValueError(f"a sequence would pass max_len = {self.max_len}")
        if not sum(counts):
            return torch.empty_like(x)
        Hq, Hkv, D, tokens = self.heads, self.kv_heads, self.D, x.shape[0]
        with _in_turn(self.dev, self.stream, x) as run:
            self._follow(run)
            ends = [0]
            for c in counts:
                ends.append(ends[-1] + c)
            index = self._to_device(ends + self.lens + after, run)
            cu, start, lens = index.split([self.sequences + 1, self.sequences, self.sequences])
            qkv = torch.empty((tokens, (Hq + 2 * Hkv) * D), dtype=self.dtype, device=self.dev)
            self._linear(x, self.w_qkv, self.s_qkv, self.b_qkv, qkv, run)
            q, k, v = qkv.view(tokens, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], 1)
            B.palquant_kv8_append(self.cache, k, v, B.kv8_tokens(k, v, cu, start, self.table, max(counts)), run)
            mixed = torch.empty((tokens, Hq, D), dtype=self.dtype, device=self.dev)
            a = B.kv8_attn(q, mixed, cu, lens, self.table, max(counts), max(after), D ** -0.5, True, self.window)
            work = self._scratch(B.palquant_kv8_attention_scratch_bytes(self.cache, a))
            B.palquant_kv8_attention(self.cache, q, mixed, a, work, work.numel(), run)
            y = torch.empty((tokens, self.hidden), dtype=self.dtype, device=self.dev)
            self._linear(mixed.view(tokens, Hq * D), self.w_out, self.s_out, None, y, run)
            self._over.record(run)
        if self.stream is not None:
            _give(self.dev, y, qkv, mixed)
        self.lens = after
        self.qkv, self.mixed = qkv, mixed  # the last call's, for inspection
        return y
