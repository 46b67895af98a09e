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
