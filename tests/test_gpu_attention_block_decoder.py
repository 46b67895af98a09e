"""The attention block with 4-bit weights, norms and rotation, a window with sinks, and trees of drafts, its calls run together.

As in the block's other tests every stage is checked against the oracle on the values that the stage before left on the
device, within the bounds of its own tests; norms and rotation are done in place, so they are checked from x on: queries and keys within the
bounds of the first layer and of the norm after it."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import tokens as ref  # noqa: E402
from test_gpu_attention_block import HALF_ULP, TYPES, _check_linear, _f32  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2208_01944_gb300 import binding
    yield binding
    assert binding.palquant_sync_check() == binding.PQ_OK


def _make(kind, hidden, heads, kv_heads, D, sequences, max_len, **kw):
    from paper_2208_01944_gb300.attention_block import AttentionBlock8

    g = torch.Generator().manual_seed(hidden + heads)
    w = [(torch.randn(*s, generator=g) * s[1] ** -0.5).to(TYPES[kind]).cuda()
         for s in (((heads + 2 * kv_heads) * D, hidden), (hidden, heads * D))]
    return AttentionBlock8(*w, heads, kv_heads, sequences, max_len, **kw), w


def _frequencies(D):
    return [10000.0 ** (-2.0 * i / D) for i in range(D // 2)]


def _check_w4(x, w, group, y, kind, bias=None):
    codes, scales = ref.w4_quantize(_f32(w), group, lambda v: v.astype(np.float16).astype(np.float32), np.float32(2.0 ** -14))
    want, size = ref.linear_w4(_f32(x), codes, scales, group, None if bias is None else _f32(bias))
    tol = HALF_ULP[kind] * np.abs(want) + (74 + w.shape[1] / 128) * 2.0 ** -23 * size + (2.0 ** -25 if kind == "f16" else 0)
    assert np.all(np.abs(_f32(y).astype(np.float64) - want) <= tol)


def _check_mixed(block, q, rows, mixed, k, v, kind, seen):
    D = block.D
    want, spread, top = ref.attention(q[rows], k, v, float(np.float32(D ** -0.5)), seen=seen)
    tol = HALF_ULP[kind] * np.abs(want) + ((2.0 ** -21 if kind == "f32" else 2.0 ** -11) + 2.0 ** -20 * (2 + top)) * spread
    tol = tol + 2.0 ** -20 * np.abs(v).max(initial=0) + (2.0 ** -25 if kind == "f16" else 0)
    assert np.all(np.abs(mixed[rows] - want) <= tol)


def _cached(B, block, s, n):
    """What the cache holds of sequence s's first n tokens, fp32."""
    k, v = (torch.empty(n, block.kv_heads, block.D, device="cuda") for _ in range(2))
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    B.palquant_kv8_read(block.cache, k, v, B.kv8_tokens(k, v, i32(0, n), i32(0), block.table[s:s + 1].contiguous(), n))
    return _f32(k), _f32(v)


def _split(block, x):
    rows = _f32(x).reshape(x.shape[0], -1, block.D)
    return rows[:, :block.heads], rows[:, block.heads:block.heads + block.kv_heads], rows[:, block.heads + block.kv_heads:]


@pytest.mark.parametrize("kind,hidden,heads,kv_heads,D,group,window,sinks,interleaved,norm", [
    ("bf16", 512, 8, 2, 64, 128, 0, 0, False, True), ("f16", 320, 4, 4, 80, 32, 50, 3, True, True),
    ("f32", 200, 6, 1, 32, 64, 20, 17, False, False), ("bf16", 1024, 16, 4, 128, 64, 100, 4, False, True)])
def test_prompts_chunks_and_single_tokens(B, kind, hidden, heads, kv_heads, D, group, window, sinks, interleaved, norm):
    f = _frequencies(D)
    g = torch.Generator().manual_seed(3)
    weights = [(1 + 0.3 * torch.randn(D, generator=g)).to(TYPES[kind]).cuda() for _ in range(2)] if norm else [None, None]
    block, (w_qkv, w_out) = _make(kind, hidden, heads, kv_heads, D, 3, 400, page_tokens=32, window=window, sinks=sinks, rope=f,
                                  rope_interleaved=interleaved, q_norm=weights[0], k_norm=weights[1], weight_bits=4, weight_group=group)
    plain, _ = _make(kind, hidden, heads, kv_heads, D, 3, 400, weight_bits=4, weight_group=group)  # no norm, no rotation: the first layer's output
    lens = [0, 0, 0]
    for counts in ([150, 1, 0], [1, 1, 200], [1, 1, 1], [0, 33, 70], [1, 1, 1]):
        x = torch.randn(sum(counts), hidden, generator=g).to(TYPES[kind]).cuda()
        y = block.forward(x, counts)
        plain.reset(0), plain.reset(1), plain.reset(2)
        plain.forward(x, counts)
        _check_w4(x, w_qkv, group, plain.qkv, kind)
        positions = np.concatenate([np.arange(n, n + c) for n, c in zip(lens, counts)])
        (q0, k0, v0), (q, k, v) = _split(block, plain.qkv), _split(block, block.qkv)
        assert np.array_equal(v, v0)
        for before, after, weight in ((q0, q, weights[0]), (k0, k, weights[1])):
            want, size = ref.norm_rope(before, None if weight is None else _f32(weight), 1e-6, positions, f, interleaved, norm)
            tol = HALF_ULP[kind] * np.abs(want) + (12 + D / 64) * 2.0 ** -23 * size + (2.0 ** -25 if kind == "f16" else 0)
            assert np.all(np.abs(after.astype(np.float64) - want) <= tol)
        mixed, row = _f32(block.mixed).astype(np.float64), 0
        for s, n in enumerate(counts):
            lens[s] += n
            if n:
                _check_mixed(block, q, slice(row, row + n), mixed, *_cached(B, block, s, lens[s]), kind, ref.sees_sinks(n, lens[s], window, sinks))
            row += n
        _check_w4(block.mixed.view(len(x), -1), w_out, group, y, kind)
        assert block.lens == lens


@pytest.mark.parametrize("kind,bits", [("bf16", 8), ("f16", 4)])
def test_drafts_and_what_is_accepted(B, kind, bits):
    heads, kv_heads, D, hidden = 8, 2, 64, 256
    f = _frequencies(D)
    block, (w_qkv, w_out) = _make(kind, hidden, heads, kv_heads, D, 3, 300, page_tokens=16, rope=f, weight_bits=bits)
    g = torch.Generator().manual_seed(5)
    draw = lambda n: torch.randn(n, hidden, generator=g).to(TYPES[kind]).cuda()  # noqa: E731
    block.forward(draw(161), [100, 0, 61])
    trees = [[-1, 0, 0, 2, 1, 3], [-1, -1, 1], []]
    for paths in ([[0, 2, 3], [1, 2], []], [[], [0], []], [[0, 1, 4], [], []]):
        lens = list(block.lens)
        x = draw(9)
        y = block.draft(x, trees)
        assert block.lens == lens
        q, k, v = _split(block, block.qkv)
        mixed, row = _f32(block.mixed).astype(np.float64), 0
        for s, tree in enumerate(trees):
            n = len(tree)
            if n:
                seen = np.zeros((n, lens[s] + n), bool)
                seen[:, :lens[s]] = True
                for i, parent in enumerate(tree):
                    seen[i, lens[s] + i] = True
                    if parent >= 0:
                        seen[i] |= seen[parent]
                _check_mixed(block, q, slice(row, row + n), mixed, *_cached(B, block, s, lens[s] + n), kind, seen)
            row += n
        if bits == 8:
            _check_linear(block.mixed.view(9, -1), w_out, None, y, kind)
        else:
            _check_w4(block.mixed.view(9, -1), w_out, 128, y, kind)
        block.accept(paths)
        row = 0
        for s, (path, tree) in enumerate(zip(paths, trees)):
            assert block.lens[s] == lens[s] + len(path)
            if path:  # the accepted tokens' keys and values, each within half a step of its page's scale
                for got, new, scales in zip(_cached(B, block, s, block.lens[s]), (k, v), (block.k_scale, block.v_scale)):
                    at = np.arange(lens[s], block.lens[s])
                    step = _f32(scales)[_pages(block, s)[at // 16]]
                    assert np.all(np.abs(got[at] - new[[row + i for i in path]]) <= 0.5001 * step[:, :, None] + 2.0 ** -24)
            row += len(tree)
        with pytest.raises(ValueError):
            block.accept(paths)
    y = block.forward(draw(3), [1, 1, 1])  # and the texts go on
    assert torch.isfinite(y.float()).all()


def _pages(block, s):
    return block.table[s].cpu().numpy()


def test_a_chain_of_drafts_is_what_forward_gives(B):
    """The same tokens drafted as a chain and fed as a chunk: the same codes, positions and views (the order of the sums differs)."""
    outs = []
    for draft in (False, True):
        block, _ = _make("bf16", 256, 4, 2, 64, 2, 200, page_tokens=32, rope=_frequencies(64))
        g = torch.Generator().manual_seed(9)
        block.forward(torch.randn(41, 256, generator=g).bfloat16().cuda(), [40, 1])
        x = torch.randn(8, 256, generator=g).bfloat16().cuda()
        y = block.draft(x, [[-1, 0, 1, 2, 3], [-1, 0, 1]]) if draft else block.forward(x, [5, 3])
        if draft:
            block.accept([[0, 1, 2, 3, 4], [0, 1, 2]])
        outs.append((_f32(block.mixed), _f32(y), block.k.clone(), block.k_scale.clone(), list(block.lens)))
    (m0, y0, k0, s0, l0), (m1, y1, k1, s1, l1) = outs
    assert l0 == l1 and torch.equal(k0, k1) and torch.equal(s0, s1)
    assert np.abs(m0 - m1).max() <= 2.0 ** -7 * np.abs(m0).max()  # two roundings to bfloat16


@pytest.mark.parametrize("own_stream", [False, True])
def test_drafts_do_not_wait_for_the_device(B, own_stream):
    block, _ = _make("bf16", 256, 4, 2, 64, 2, 200, rope=_frequencies(64), weight_bits=4, stream=torch.cuda.Stream() if own_stream else None)
    xs = [torch.randn(n, 256, generator=torch.Generator().manual_seed(n)).bfloat16().cuda() for n in (21, 5, 2, 5)]
    trees, paths = [[-1, 0, 0], [-1, -1]], [[0, 2], [1]]

    def run():
        out = [block.forward(xs[0], [20, 1])]
        for _ in range(2):
            out.append(block.draft(xs[1], trees))
            block.accept(paths)
            out.append(block.forward(xs[2], [1, 1]))
        return out

    run()
    torch.cuda.synchronize()
    for s in (0, 1):
        block.reset(s)
    torch.cuda._sleep(500_000_000)
    mode = torch.cuda.get_sync_debug_mode()
    torch.cuda.set_sync_debug_mode("error")
    try:
        ahead = run()
    finally:
        torch.cuda.set_sync_debug_mode(mode)
    torch.cuda.synchronize()
    for s in (0, 1):
        block.reset(s)
    for got, want in zip(ahead, run()):
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_refusals(B):
    block, _ = _make("bf16", 256, 4, 2, 64, 2, 100)
    x = torch.zeros(4, 256, dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: block.accept([[], []]), lambda: block.draft(x, [[-1, 0, 1, 2]]), lambda: block.draft(x, [[-1, 0, 1, 3], []]),
                lambda: block.draft(x, [[-1, 0, 1, -2], []]), lambda: block.draft(x, [[-1, 0, 1], []]),
                lambda: block.draft(x.new_zeros(101, 256), [[-1] * 101, []])):
        with pytest.raises(ValueError):
            bad()
    block.draft(x, [[-1, 0, 1], [-1]])
    for bad in ([[0, 1, 2], [1]], [[1], []], [[0, 2], []], [[0], [0], []], [[0, 0], []]):
        with pytest.raises(ValueError):
            block.accept(bad)
    assert block.lens == [0, 0]
    block.accept([[0, 1], []])
    assert block.lens == [2, 0]
    block.draft(x, [[-1, 0, 1], [-1]])
    block.forward(x[:2], [1, 1])  # forgets the drafts
    with pytest.raises(ValueError):
        block.accept([[0], []])
    windowed, _ = _make("bf16", 256, 4, 2, 64, 2, 100, window=10)
    with pytest.raises(ValueError):
        windowed.draft(x, [[-1, 0, 1], [-1]])
    assert block.draft(x[:0], [[], []]).shape == (0, 256)


@pytest.mark.parametrize("scales", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", list(TYPES))
def test_quiet_weights_in_4_bits(B, kind, scales):
    """Weights of deviation 1e-5: no group of them is lost where the scales are not held in half precision."""
    from paper_2208_01944_gb300.attention_block import AttentionBlock8

    g = torch.Generator().manual_seed(17)
    w = [(torch.randn(*s, generator=g) * 1e-5).to(TYPES[kind]).cuda() for s in ((8 * 64, 256), (256, 4 * 64))]
    block = AttentionBlock8(*w, 4, 2, 1, 100, weight_bits=4, weight_group=64, weight_scales=scales)
    x = torch.randn(50, 256, generator=g).to(TYPES[kind]).cuda()
    block.forward(x, [50])
    codes, s = ref.w4_quantize(_f32(w[0]), 64, lambda v: torch.from_numpy(v).to(scales).float().numpy())
    assert (s > 0).all()
    want, size = ref.linear_w4(_f32(x), codes, s, 64)
    tol = HALF_ULP[kind] * np.abs(want) + (74 + 2) * 2.0 ** -23 * size + (2.0 ** -25 if kind == "f16" else 0)
    assert np.all(np.abs(_f32(block.qkv).astype(np.float64) - want) <= tol)
