"""Self-attention of a transformer layer in 8-bit codes, prompts and single tokens, through the C ABI.

The paper has no counterpart; the block shows the library's transformer calls together,
as a server would use them:

    qkv = x W_qkv^T + b_qkv        palquant_linear_q8: 8-bit codes, one scale for each token and channel; or
                                   palquant_linear_w4: 4-bit weights, one scale for each channel and group
    q, k <- norm, rotation         palquant_qk_norm_rope, in place (with rope or norm weights)
    cache <- k, v                  palquant_kv8_append: 8-bit codes, one scale for each page and head
    mixed = attention(q, cache)    palquant_kv8_attention: grouped heads, causal, optional window;
                                   palquant_kv8_attention_sinks: a window that keeps the first tokens in sight
    y = mixed W_out^T              as the first

A block serves a fixed set of sequences.  forward() takes any number of new tokens for each of
them (none, one, a chunk or a whole prompt), appends them to the cache and attends from them
to everything cached so far; sequences of different lengths share a call.  reset() ends a
sequence and makes its pages free for the next one.  q, k and v are read where the first layer
wrote them (columns of its output), so nothing is copied between the four calls.

    block = AttentionBlock8(w_qkv, w_out, heads=32, kv_heads=8, sequences=4, max_len=4096)
    y = block.forward(prompts, [900, 17, 2048, 1])    # [2966, hidden]
    y = block.forward(tokens, [1, 1, 1, 1])           # [4, hidden]

draft() runs drafted tokens, a tree of them for each sequence, which see the text and their ancestors
(palquant_kv8_attention_tree); accept() keeps one path of each tree.

    y = block.draft(tokens, [[-1, 0, 0, 2], [], [-1], [-1, -1]])   # each draft's parent, -1: it follows the text
    block.accept([[0, 2, 3], [], [0], []])
"""
from __future__ import annotations

import contextlib

import numpy as np
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


def weight_codes4(w: torch.Tensor, group: int = 128, scales: torch.dtype = torch.float16, stream: torch.cuda.Stream | None = None):
    """w [N, K] quantised to 4 bits with a scale for each row and `group` (32, 64 or 128) of its columns, and packed: (descriptor,
    packed bytes) for palquant_linear_w4.  `scales` is the type that the scales are held in: a group whose largest weight is below 7 of the
    type's smallest normal numbers becomes zeros, for float16 4.3e-4 (weights that quiet want bfloat16 or float32 scales).  It runs on
    `stream` as weight_codes does."""
    if w.dim() != 2 or w.dtype not in _TYPES or w.stride(1) != 1:
        raise ValueError("w: a float matrix with contiguous rows")
    desc = B.w4_weights(w.shape[0], w.shape[1], group, scales)
    nbytes = B.palquant_w4_packed_bytes(desc)
    if not nbytes:
        raise ValueError("group: 32, 64 or 128; w: rows of up to 131072")
    with _in_turn(w.device, stream, w) as run:
        packed = torch.empty(nbytes, dtype=torch.uint8, device=w.device)
        B.palquant_w4_quantize(w, _TYPES[w.dtype], w.stride(0), desc, packed, nbytes, run)
    _give(w.device, packed)
    return desc, packed


def _depths(parents, limit: int) -> list[int]:
    """How deep each draft of one sequence's tree stands (0: it follows the text)."""
    depths: list[int] = []
    for i, parent in enumerate(parents):
        if not -1 <= parent < i:
            raise ValueError("parents: of each draft one before it, or -1")
        depths.append(depths[parent] + 1 if parent >= 0 else 0)
    if len(depths) > limit:
        raise ValueError("parents: more drafts than the sequence has room for")
    return depths


def tree_bits(parents) -> torch.Tensor:
    """The rows of palquant_kv8_attention_tree for trees of drafts, one after the other: parents[b][i] is the draft that draft
    i of sequence b follows, one before it, or -1 for the text.  int32 [drafts, words] on the CPU."""
    words = max(1, -(-max((len(of) for of in parents), default=0) // 32))
    rows = []
    for of in parents:
        _depths(of, len(of))
        masks: list[int] = []
        for i, parent in enumerate(of):
            masks.append((masks[parent] if parent >= 0 else 0) | 1 << i)
        rows += [[m >> 32 * w & 0xFFFFFFFF for w in range(words)] for m in masks]
    return torch.from_numpy(np.array(rows, dtype=np.uint32).reshape(-1, words).view(np.int32))


class AttentionBlock8:
    def __init__(self, w_qkv: torch.Tensor, w_out: torch.Tensor, heads: int, kv_heads: int, sequences: int, max_len: int,
                 b_qkv: torch.Tensor | None = None, page_tokens: int = 64, window: int = 0,
                 stream: torch.cuda.Stream | None = None, *, sinks: int = 0, rope=None, rope_interleaved: bool = False,
                 q_norm: torch.Tensor | None = None, k_norm: torch.Tensor | None = None, norm_eps: float = 1e-6,
                 weight_bits: int = 8, weight_group: int = 128, weight_scales: torch.dtype = torch.float16):
        """w_qkv [(heads + 2 kv_heads) D, hidden] (the rows of q, then k, then v) and w_out [hidden, heads D] on the
        GPU; their type is the activations'.  b_qkv: a value for each row of w_qkv.

        sinks: first tokens that a window keeps in sight.  rope: frequencies, in radians a position, of the rotation of the
        first 2 len(rope) elements of every query and key head (pairs half of them apart, or neighbours with
        rope_interleaved).  q_norm, k_norm [D]: weights of a norm of every query and key head before the rotation (both
        or none).  weight_bits 4: the weights in 4 bits with a scale for each channel and weight_group of inputs, held as
        weight_scales (float16 takes groups whose largest weight is below 4.3e-4 for zeros: see weight_codes4)."""
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
        if sinks < 0 or (sinks and not window):
            raise ValueError("sinks: of a window")
        if weight_bits not in (4, 8) or weight_group not in (32, 64, 128) or weight_scales not in _TYPES:
            raise ValueError("weight_bits: 4 or 8; weight_group: 32, 64 or 128; weight_scales: float32, float16 or bfloat16")
        rope = None if rope is None else [float(f) for f in rope]
        if rope is not None and (2 * len(rope) > self.D or not np.isfinite(rope).all()):
            raise ValueError("rope: finite frequencies, one for each pair of a head's elements at most")
        if (q_norm is None) != (k_norm is None) or not norm_eps >= 0 or any(
                n is not None and (n.shape != (self.D,) or n.dtype != q_norm.dtype or n.dtype not in _TYPES) for n in (q_norm, k_norm)):
            raise ValueError("q_norm, k_norm: [D] of one float type, both or none; norm_eps: 0 and up")
        if w_out.shape != (self.hidden, heads * self.D) or w_out.dtype != w_qkv.dtype:
            raise ValueError("w_out: [hidden, heads D], of w_qkv's type")
        self.dtype, self.dev, self.stream = w_qkv.dtype, w_qkv.device, stream
        self.sequences, self.max_len = sequences, max_len
        self.sinks, self.weight_bits, self.norm_eps, self.rope_interleaved = sinks, weight_bits, float(norm_eps), bool(rope_interleaved)
        given = [t for t in (w_qkv, w_out, b_qkv, q_norm, k_norm) if t is not None and t.is_cuda]
        with _in_turn(self.dev, stream, *given) as run:
            self.b_qkv = None if b_qkv is None else b_qkv.to(self.dev, torch.float32).contiguous().view(-1)
            w_qkv, w_out = w_qkv.contiguous(), w_out.contiguous()
            if weight_bits == 4:
                # (descriptor, packed) of each; no scales beside them
                (self.w_qkv_desc, self.w_qkv), (self.w_out_desc, self.w_out) = (weight_codes4(w, weight_group, weight_scales, run) for w in (w_qkv, w_out))
                self.s_qkv = self.s_out = None
            else:
                self.w_qkv, self.s_qkv = weight_codes(w_qkv, run)
                self.w_out, self.s_out = weight_codes(w_out, run)
            self.turns = None if not rope else B.rope_turns(rope, self.dev)
            self.q_norm, self.k_norm = (None if n is None else n.to(self.dev).contiguous() for n in (q_norm, k_norm))
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
                                     self.v_scale, self.table, self.turns, self.q_norm, self.k_norm) if t is not None]
            self._ran, self._over = run, torch.cuda.Event()  # the last call's stream, and its end there
            self._over.record(run)
        self.lens = [0] * sequences  # tokens cached, on the host: no call waits for the device to know them
        self._drafted = None         # the last call's trees and keys and values, if it was draft()

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

    def _upload(self, values: np.ndarray) -> torch.Tensor:
        """Host values on the device, without waiting for it (the page-locked copy is held until it has been read)."""
        return torch.from_numpy(values).pin_memory().to(self.dev, non_blocking=True)

    def _linear(self, x, w, s_w, bias, y, run):
        if self.weight_bits == 4:
            desc = self.w_qkv_desc if w is self.w_qkv else self.w_out_desc
            d = B.linear_w4_desc(x, desc, y)
            work = self._scratch(B.palquant_linear_w4_scratch_bytes(desc, d))
            B.palquant_linear_w4(x, w, bias, y, desc, d, work, work.numel(), run)
            return
        d = B.linear_desc(x, w, y)
        work = self._scratch(B.palquant_linear_q8_scratch_bytes(d))
        B.palquant_linear_q8(x, w, s_w, bias, y, d, work, work.numel(), run)

    def _turn(self, q, k, positions, run) -> None:
        """Norm and rotation of new queries and keys where the first layer wrote them."""
        if self.turns is None and self.q_norm is None:
            return
        d = B.qk_norm_rope(q, k, q, k, positions, self.turns, self.q_norm, self.k_norm, self.norm_eps, self.rope_interleaved,
                           norm=self.q_norm is not None)
        B.palquant_qk_norm_rope(q, k, q, k, d, run)

    def _new_tokens(self, x, counts):
        """What forward() and draft() take: counts of new tokens, and the sequences' lengths with them."""
        counts = [int(c) for c in counts]
        if len(counts) != self.sequences or min(counts) < 0 or x.shape != (sum(counts), self.hidden) \
                or x.dtype != self.dtype or x.device != self.dev:
            raise ValueError("counts: one for each sequence; x: [sum(counts), hidden] of the weights' type, on their device")
        after = [n + c for n, c in zip(self.lens, counts)]
        if max(after) > self.max_len:
            raise ValueError(f"a sequence would pass max_len = {self.max_len}")
        return counts, after

    def _run(self, x, counts, after, positions, parents, run):
        """The block's calls for new tokens at their positions (None: one after the other); parents: the drafts' trees, or None."""
        Hq, Hkv, D, tokens = self.heads, self.kv_heads, self.D, x.shape[0]
        ends = [0]
        for c in counts:
            ends.append(ends[-1] + c)
        index = self._to_device(ends + self.lens + after, run)
        cu, start, lens = index.split([self.sequences + 1, self.sequences, self.sequences])
        if self.turns is None:
            positions = None
        elif positions is not None:
            positions = self._upload(positions)
        elif counts == [1] * self.sequences:
            positions = start  # single tokens stand where their sequences end
        else:
            positions = self._upload(np.concatenate([np.arange(n, n + c, dtype=np.int32) for n, c in zip(self.lens, counts)]))
        qkv = torch.empty((tokens, (Hq + 2 * Hkv) * D), dtype=self.dtype, device=self.dev)
        self._linear(x, self.w_qkv, self.s_qkv, self.b_qkv, qkv, run)
        q, k, v = qkv.view(tokens, Hq + 2 * Hkv, D).split([Hq, Hkv, Hkv], 1)
        self._turn(q, k, positions, run)
        B.palquant_kv8_append(self.cache, k, v, B.kv8_tokens(k, v, cu, start, self.table, max(counts)), run)
        mixed = torch.empty((tokens, Hq, D), dtype=self.dtype, device=self.dev)
        a = B.kv8_attn(q, mixed, cu, lens, self.table, max(counts), max(after), D ** -0.5, True, self.window)
        if parents is not None:
            tree = B.kv8_tree(self._upload(tree_bits(parents).numpy()), a)
            work = self._scratch(B.palquant_kv8_attention_tree_scratch_bytes(self.cache, a, tree))
            B.palquant_kv8_attention_tree(self.cache, q, mixed, a, tree, work, work.numel(), run)
        elif self.sinks:
            work = self._scratch(B.palquant_kv8_attention_sinks_scratch_bytes(self.cache, a, self.sinks))
            B.palquant_kv8_attention_sinks(self.cache, q, mixed, a, self.sinks, work, work.numel(), run)
        else:
            work = self._scratch(B.palquant_kv8_attention_scratch_bytes(self.cache, a))
            B.palquant_kv8_attention(self.cache, q, mixed, a, work, work.numel(), run)
        y = torch.empty((tokens, self.hidden), dtype=self.dtype, device=self.dev)
        self._linear(mixed.view(tokens, Hq * D), self.w_out, self.s_out, None, y, run)
        return y, qkv, mixed

    def reset(self, sequence: int) -> None:
        self.lens[sequence] = 0
        self._drafted = None

    def forward(self, x: torch.Tensor, counts) -> torch.Tensor:
        """x [sum(counts), hidden]: counts[b] new tokens of every sequence b, one sequence after the other; returns y
        of x's shape.  It runs on the block's stream (None: the current one), after what the current stream holds and
        before what it is given next; with the current stream another than the last call's, after that call too."""
        counts, after = self._new_tokens(x, counts)
        if not sum(counts):
            return torch.empty_like(x)
        return self._call(x, counts, after, None, None)

    def _call(self, x, counts, after, positions, parents) -> torch.Tensor:
        self._drafted = None
        with _in_turn(self.dev, self.stream, x) as run:
            self._follow(run)
            y, qkv, mixed = self._run(x, counts, after, positions, parents, run)
            self._over.record(run)
        if self.stream is not None:
            _give(self.dev, y, qkv, mixed)
        if parents is None:
            self.lens = after
        self.qkv, self.mixed = qkv, mixed  # the last call's, for inspection
        return y

    def draft(self, x: torch.Tensor, parents) -> torch.Tensor:
        """x [drafts, hidden]: drafted tokens of every sequence, one sequence after the other; parents[b][i] is the draft of
        sequence b, one before it, that its draft i follows, or -1 where it follows the text.  Each stands one position
        after its parent and sees the text and its ancestors; returns y of x's shape, streams as with forward().  The
        drafts take the cache's places after the texts, which stay as long as they were: accept() keeps some, any
        other call forgets them.  (A page that holds the end of a text keeps the scale that its loudest drafts asked for.)
        Not with a window: drafts' places in the cache are not their positions."""
        if self.window:
            raise ValueError("drafts: not with a window")
        parents = [[int(p) for p in of] for of in parents]
        counts, after = self._new_tokens(x, [len(of) for of in parents])
        positions = [n + d for n, of in zip(self.lens, parents) for d in _depths(of, self.max_len)]
        if not sum(counts):
            self._drafted = None
            return torch.empty_like(x)
        y = self._call(x, counts, after, np.array(positions, dtype=np.int32), parents)
        self._drafted = parents
        return y

    def accept(self, paths) -> None:
        """Keep drafts of the last call, which was draft(): paths[b] are drafts of sequence b, the first one's parent the text and
        each other's the one before it; the text goes on with them.  An empty path keeps none."""
        if self._drafted is None:
            raise ValueError("accept: after draft()")
        paths = [[int(i) for i in path] for path in paths]
        if len(paths) != self.sequences:
            raise ValueError("paths: one for each sequence")
        rows, first = [], 0
        for path, of in zip(paths, self._drafted):
            for before, i in zip([-1] + path, path):
                if not 0 <= i < len(of) or of[i] != before:
                    raise ValueError("paths: each draft's parent is the one before it")
            rows += [first + i for i in path]
            first += len(of)
        counts = [len(path) for path in paths]
        after = [n + c for n, c in zip(self.lens, counts)]
        if rows:
            qkv = self.qkv
            with _in_turn(self.dev, self.stream, qkv) as run:
                self._follow(run)
                qkv.record_stream(run)
                ends = [0]
                for c in counts:
                    ends.append(ends[-1] + c)
                index = self._to_device(ends + self.lens + after, run)
                cu, start, _ = index.split([self.sequences + 1, self.sequences, self.sequences])
                kept = qkv.index_select(0, self._upload(np.array(rows, dtype=np.int64)))
                _, k, v = kept.view(len(rows), -1, self.D).split([self.heads, self.kv_heads, self.kv_heads], 1)
                B.palquant_kv8_append(self.cache, k, v, B.kv8_tokens(k, v, cu, start, self.table, max(counts)), run)
                self._over.record(run)
        self.lens, self._drafted = after, None
