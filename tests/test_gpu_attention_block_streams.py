"""The attention block on streams that change: results as on one stream, and memory of its own that no other stream is given."""
import pytest

from test_gpu_attention_block import _block

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PAUSE = 200_000_000  # cycles of a stream's own, about a tenth of a second


def _x(tokens, hidden, seed):
    return torch.randn(tokens, hidden, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


def test_weight_codes_follow_the_weights_and_are_followed():
    """On another stream: after the weights are there, and before the current stream reads the codes."""
    from paper_2208_01944_gb300.attention_block import weight_codes

    w = torch.randn(300, 200, generator=torch.Generator().manual_seed(1)).cuda()
    want = weight_codes(w)
    late, side = torch.zeros_like(w), torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(PAUSE)
    late.copy_(w)
    got = weight_codes(late, side)
    copies = [t.clone() for t in got]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, copies))


@pytest.mark.parametrize("bias", [False, True])
def test_calls_from_changing_streams_keep_their_order(bias):
    """Each call sees what the one before cached, whichever stream that was given to."""
    outs = []
    for change in (False, True):
        block, _, _ = _block("bf16", 256, 4, 2, 64, 2, 400, 32, 0, bias)
        xs = [_x(21, 256, 1), _x(2, 256, 2), _x(300, 256, 3), _x(2, 256, 4)]
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        ys = []
        for i, (x, counts) in enumerate(zip(xs, ([20, 1], [1, 1], [100, 200], [1, 1]))):
            with torch.cuda.stream(side if change and i % 2 else torch.cuda.default_stream()):
                torch.cuda._sleep(PAUSE // 10) if change and not i % 2 else None  # what the next call would overtake
                ys.append(block.forward(x, counts))
        torch.cuda.synchronize()
        outs.append(torch.cat(ys))
    assert torch.equal(outs[0], outs[1])


def test_no_stream_is_given_memory_that_another_still_uses(monkeypatch):
    """A workspace made for a call on one stream, used by a call on another, outgrown there: while the second stream still
    has its calls to run, allocations of the first do not get it."""
    from paper_2208_01944_gb300 import binding as B

    used = []
    real = B.palquant_linear_q8

    def spy(x, w, s_w, bias, y, d, work, nbytes, stream):
        used.append((work.data_ptr(), work.data_ptr() + work.numel()))
        return real(x, w, s_w, bias, y, d, work, nbytes, stream)

    monkeypatch.setattr(B, "palquant_linear_q8", spy)
    block, _, _ = _block("bf16", 256, 4, 2, 64, 2, 400, 32, 0, False)
    xs = [_x(40, 256, 1), _x(40, 256, 2), _x(300, 256, 3)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    block.forward(xs[0], [20, 20])
    side.wait_stream(torch.cuda.current_stream())
    done = torch.cuda.Event()
    with torch.cuda.stream(side):
        torch.cuda._sleep(PAUSE)
        used.clear()
        block.forward(xs[1], [20, 20])
        block.forward(xs[2], [150, 150])
        done.record()
    own = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in [512 * k for k in range(1, 200)] * 3]
    pending = not done.query()
    assert pending and used
    for t in own:
        a, b = t.data_ptr(), t.data_ptr() + t.numel()
        assert not any(a < hi and lo < b for lo, hi in used)


def test_outputs_kept_for_inspection_outlive_the_next_call():
    """block.qkv and block.mixed are the current stream's to read, as the result is, also after the block has let them go."""
    side = torch.cuda.Stream()
    block, _, _ = _block("bf16", 256, 4, 2, 64, 2, 200, 32, 0, False, side)
    x = _x(100, 256, 1)
    torch.cuda.synchronize()
    block.forward(x, [50, 50])
    held = [(t.data_ptr(), t.data_ptr() + t.numel() * 2) for t in (block.qkv, block.mixed)]
    copies = []
    torch.cuda._sleep(PAUSE)
    copies += [block.qkv.clone(), block.mixed.clone()]  # to be read after the pause
    block.qkv = block.mixed = None
    with torch.cuda.stream(side):
        own = [torch.empty(t.numel(), dtype=t.dtype, device="cuda") for t in copies for _ in range(8)]
    for t in own:
        a, b = t.data_ptr(), t.data_ptr() + t.numel() * 2
        assert not any(a < hi and lo < b for lo, hi in held)
    torch.cuda.synchronize()
