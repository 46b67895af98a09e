"""Windows as long as the texts and longer, up to the largest 32-bit one, where some queries stand before the first token.
The bounds are those of the other attention tests."""
import numpy as np
import pytest

from test_gpu_kv8 import Cache, _attend, _check

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2208_01944_gb300 import binding
    yield binding
    assert binding.palquant_sync_check() == binding.PQ_OK


@pytest.mark.parametrize("kind", ["f32", "f16"])
@pytest.mark.parametrize("window", [0x7FFFFFFF, 0x7FFFFFF0, 400, 399, 301, 300, 299])
@pytest.mark.parametrize("n,lens", [([20, 3, 1], [9, 0, 300]), ([330, 150], [300, 40])], ids=str)
def test_windows_that_hide_nothing(B, n, lens, window, kind):
    c = Cache(B, lens, 2, 64, 32, seed=sum(n))
    q, o, scale = _attend(B, c, n, lens, 4, kind, True, window, seed=1)
    _check(c, q, o, n, lens, kind, True, window, scale)
    if window >= max(lens):
        assert np.array_equal(o, _attend(B, c, n, lens, 4, kind, True, 0, seed=1)[1])
