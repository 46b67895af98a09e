"""The 8-bit attention block: its four calls chained over prompts, chunks and single tokens.

Every stage is checked against the oracle on the values that the stage before left on the device: the codes and scales in
the cache exactly, the two dense layers and the attention within the bounds of their own tests.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import tokens as ref  # noqa: E402

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _f32(t):
    return t.float().cpu().numpy()


def _block(kind, hidden, heads, kv_heads, D, sequences, max_len, page_tokens, window, bias, stream=None):
    from paper_2208_01944_gb300.attention_block import AttentionBlock8

    g = torch.Generator().manual_seed(hidden + heads)
    w = [(torch.randn(*s, generator=g) * s[1] ** -0.5).to(TYPES[kind]).cuda()
         for s in (((heads + 2 * kv_heads) * D, hidden), (hidden, heads * D))]
    b = torch.randn(w[0].shape[0], generator=g).cuda() if bias else None
    torch.cuda.synchronize()
    return AttentionBlock8(*w, heads, kv_heads, sequences, max_len, b, page_tokens, window, stream), w, b


def _check_linear(x, w, bias, y, kind):
    qw, sw = ref.quantize_tokens(_f32(w))
    q, s = ref.quantize_tokens(_f32(x))
    want = ref.linear_value(ref.linear(q, qw), s, sw)
    tol = np.abs(want) * 3 * 2.0 ** -24
    if bias is not None:
        want = want + _f32(bias).astype(np.float64)
        tol = tol + (np.abs(want) + tol) * 2.0 ** -24
    tol = tol + (np.abs(want) + tol) * HALF_ULP[kind] + (2.0 ** -25 if kind == "f16" else 0) + 2.0 ** -140
    assert np.all(np.abs(_f32(y).astype(np.float64) - want) <= tol)


@pytest.mark.parametrize("kind,hidden,heads,kv_heads,D,page_tokens,window,bias", [
    ("bf16", 512, 8, 2, 64, 64, 0, False), ("f16", 320, 4, 4, 80, 32, 50, True), ("f32", 200, 6, 1, 32, 16, 0, True),
    ("bf16", 1024, 16, 4, 128, 64, 0, False)])
def test_prompts_chunks_and_single_tokens(kind, hidden, heads, kv_heads, D, page_tokens, window, bias):
    sequences, max_len = 3, 400
    block, (w_qkv, w_out), b = _block(kind, hidden, heads, kv_heads, D, sequences, max_len, page_tokens, window, bias)
    T, table = page_tokens, block.table.cpu().numpy()
    k, v = (np.zeros(block.k.shape, np.int8) for _ in range(2))
    ks, vs = (np.zeros(block.k_scale.shape, np.float32) for _ in range(2))
    lens = [0] * sequences
    g = torch.Generator().manual_seed(7)
    for step, counts in enumerate([[150, 1, 0], [1, 1, 300], [1, 1, 1], [0, 33, 70], [1, 1, 1]]):
        if step == 3:
            block.reset(0)
            lens[0] = 0
            counts = [65, 33, 20]
        x = torch.randn(sum(counts), hidden, generator=g).to(TYPES[kind]).cuda()
        y = block.forward(x, counts)
        _check_linear(x, w_qkv, b, block.qkv, kind)
        qkv = _f32(block.qkv).reshape(-1, heads + 2 * kv_heads, D)
        mixed, row = _f32(block.mixed).astype(np.float64), 0
        for s, n in enumerate(counts):
            new = qkv[row:row + n]
            if n:
                ref.append(k, ks, table[s], lens[s], new[:, heads:heads + kv_heads])
                ref.append(v, vs, table[s], lens[s], new[:, heads + kv_heads:])
            lens[s] += n
            if n:
                K, V = (ref.read(c, cs, table[s], 0, lens[s]) for c, cs in ((k, ks), (v, vs)))
                want, spread, top = ref.attention(new[:, :heads], K, V, float(np.float32(D ** -0.5)), True, window)
                tol = HALF_ULP[kind] * np.abs(want) + ((2.0 ** -21 if kind == "f32" else 2.0 ** -11) + 2.0 ** -20 * (2 + top)) * spread
                tol = tol + 2.0 ** -20 * np.abs(V).max() + (2.0 ** -25 if kind == "f16" else 0)
                assert np.all(np.abs(mixed[row:row + n] - want) <= tol)
            row += n
        live = np.concatenate([table[s, :-(-lens[s] // T)] for s in range(sequences)])
        assert np.array_equal(block.k_scale.cpu().numpy()[live], ks[live]) and np.array_equal(block.v_scale.cpu().numpy()[live], vs[live])
        assert np.array_equal(block.k.cpu().numpy()[live], k[live]) and np.array_equal(block.v.cpu().numpy()[live], v[live])
        _check_linear(block.mixed.view(len(x), -1), w_out, None, y, kind)
        assert block.lens == lens


def test_the_stream_of_the_block_and_repeated_runs():
    """The same calls on another stream give the same bits."""
    outs = []
    for stream in (None, torch.cuda.Stream(), None):
        block, _, _ = _block("bf16", 256, 4, 2, 64, 2, 200, 32, 0, False, stream)
        x = torch.randn(101, 256, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
        torch.cuda.synchronize()
        ys = [block.forward(x, [100, 1]), block.forward(x[:2], [1, 1])]
        torch.cuda.synchronize()
        outs.append(torch.cat(ys))
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_refusals():
    block, (w_qkv, w_out), _ = _block("bf16", 256, 4, 2, 64, 2, 100, 32, 0, False)
    x = torch.zeros(4, 256, dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: block.forward(x, [4]), lambda: block.forward(x, [5, -1]), lambda: block.forward(x, [1, 1]),
                lambda: block.forward(x.float(), [2, 2]), lambda: block.forward(x.new_zeros(101, 256), [101, 0]),
                lambda: type(block)(w_qkv, w_out, 4, 3, 2, 100), lambda: type(block)(w_qkv, w_out[:, 1:], 4, 2, 2, 100)):
        with pytest.raises(ValueError):
            bad()
    assert block.lens == [0, 0] and block.forward(x[:0], [0, 0]).shape == (0, 256)
