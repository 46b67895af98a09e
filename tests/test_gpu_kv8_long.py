"""Prompts over texts of many steps of the tile kernel: 128 tokens a step, its ring of looked-up pages (8 steps) wraps.

A block walks a whole text where there are more row tiles than SMs (sequences x cache heads x tiles of 256 query rows): forty
sequences of four heads, all but one of them short.  The bounds are those of the other attention tests."""
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


CASES = [  # queries and tokens of the long text, Hq, D, T, causal, window
    (200, 2700, 4, 128, 64, True, 0),   # two tiles of 128 rows, 22 steps
    (60, 2561, 4, 64, 16, True, 0),     # eight pages a step
    (90, 5000, 8, 96, 128, True, 0),    # 40 steps, two heads a cache head
    (70, 3100, 4, 128, 32, False, 0),
    (200, 6000, 4, 48, 64, True, 2600),
]


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_many_steps(B, case, kind):
    n, length, Hq, D, T, causal, window = case
    counts, lens = [1] * 40, [5 + b for b in range(40)]
    counts[17], lens[17] = n, length
    c = Cache(B, lens, 4, D, T, seed=D)
    outs = [_attend(B, c, counts, lens, Hq, kind, causal, window, seed=n) for _ in range(3)]
    q, o, scale = outs[0]
    _check(c, q, o, counts, lens, kind, causal, window, scale)
    assert all(np.array_equal(o, other[1]) for other in outs[1:])  # and the same bits in every call
