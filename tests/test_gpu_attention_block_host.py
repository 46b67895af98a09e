"""What the attention block asks of the host: its calls are handed to the device without waiting for it."""
import pytest

from test_gpu_attention_block import _block

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _x(tokens, hidden, seed):
    return torch.randn(tokens, hidden, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()


@pytest.mark.parametrize("own_stream", [False, True])
def test_forward_does_not_wait_for_the_device(own_stream):
    block, _, _ = _block("bf16", 256, 4, 2, 64, 2, 200, 32, 0, False, torch.cuda.Stream() if own_stream else None)
    xs = [_x(21, 256, 1)] + [_x(2, 256, 2 + i) for i in range(6)]
    block.forward(xs[0], [20, 1])
    torch.cuda.synchronize()
    done = torch.cuda.Event()
    torch.cuda._sleep(1_000_000_000)  # half a second of the current stream, which the block's stream waits for
    mode = torch.cuda.get_sync_debug_mode()
    torch.cuda.set_sync_debug_mode("error")
    try:
        ys = [block.forward(x, [1, 1]) for x in xs[1:]]
        done.record()
        ahead = not done.query()
    finally:
        torch.cuda.set_sync_debug_mode(mode)
    assert ahead
    # and each call read its own positions, although the host was calls ahead
    again, _, _ = _block("bf16", 256, 4, 2, 64, 2, 200, 32, 0, False)
    again.forward(xs[0], [20, 1])
    for x, y in zip(xs[1:], ys):
        torch.cuda.synchronize()
        assert torch.equal(again.forward(x, [1, 1]), y)


def test_more_calls_ahead_than_buffers():
    """Positions go through a fixed number of page-locked buffers in turn: none is filled again before it was copied."""
    outs = []
    for ahead in (True, False):
        block, _, _ = _block("bf16", 256, 4, 2, 64, 2, 200, 32, 0, False)
        xs = [_x(2, 256, 50 + i) for i in range(70)]
        torch.cuda.synchronize()
        if ahead:
            torch.cuda._sleep(100_000_000)
        ys = []
        for x in xs:
            ys.append(block.forward(x, [1, 1]))
            if not ahead:
                torch.cuda.synchronize()
        outs.append(torch.cat(ys))
    assert torch.equal(outs[0], outs[1])
