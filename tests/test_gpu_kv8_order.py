"""Attention over more sequences than find room at one time: they are taken the longest first, whatever their order, and every one of
them exactly once.  Equal lengths, sequences without tokens or without queries, and as many sequences as are put in order and one more.
The bounds are those of the other attention tests."""
import numpy as np
import pytest

from oracle import tokens as ref
from test_gpu_kv8 import Cache, _attend, _check
from test_gpu_kv8_views import _check as _check_seen
from test_gpu_kv8_views import _queries, _tree

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2208_01944_gb300 import binding
    yield binding
    assert binding.palquant_sync_check() == binding.PQ_OK


def _lengths(B, most, seed):
    """Ragged, many of them equal, some empty."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, most + 1, B)
    lens[rng.random(B) < 0.3] = most // 2
    lens[rng.random(B) < 0.1] = 0
    lens[B - 3] = 2100
    return [int(n) for n in lens]


@pytest.mark.parametrize("sequences,H,causal", [(45, 8, True), (40, 8, False), (128, 3, True), (129, 3, True), (20, 16, True)])
@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_single_tokens(B, sequences, H, causal, kind):
    lens = _lengths(sequences, 200, sequences)
    n = [0 if b % 11 == 3 else 1 for b in range(sequences)]
    c = Cache(B, lens, H, 32, 16, seed=sequences)
    q, o, scale = _attend(B, c, n, lens, 2 * H, kind, causal, 0, seed=7)
    _check(c, q, o, n, lens, kind, causal, 0, scale)


@pytest.mark.parametrize("sequences,H,most", [(45, 8, 9), (26, 8, 24), (100, 2, 24), (45, 8, 1)])
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
def test_drafts(B, sequences, H, most, kind):
    rng = np.random.default_rng(most)
    n = [int(v) for v in rng.integers(0, most + 1, sequences)]
    n[sequences // 2] = most
    lens = [max(a, b) for a, b in zip(n, _lengths(sequences, 300, most))]
    c = Cache(B, lens, H, 64, 32, seed=sequences)
    # each draft sees itself and about half of the drafts before it
    bits = np.zeros((sum(n), 1), np.uint32)
    at = np.concatenate([[0], np.cumsum(n)])
    for b in range(sequences):
        for i in range(n[b]):
            bits[at[b] + i] = (int(rng.integers(0, 1 << i)) if i else 0) | 1 << i
    q, o = _queries(sum(n), 4 * H, 64, kind, 5)
    _tree(B, c, q, o, n, lens, torch.from_numpy(bits.view(np.int32)).cuda())
    _check_seen(c, q, o, n, lens, kind, lambda b: ref.sees_tree(n[b], lens[b], bits[at[b]:at[b + 1]]))
