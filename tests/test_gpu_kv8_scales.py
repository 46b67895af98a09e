"""Attention over pages whose value scales are far apart, against the oracle in double.

Bound, with u the output type's half ulp, spread = sum p |v| and lv the largest |log2 scale| of the row's pages:
  u |o|                                          the rounding to the type,
+ 2^-11 spread (16-bit), 2^-21 spread (fp32)     the probabilities as one or two halves,
+ 2^-20 (2 + max |score|) spread                 scores, exponentials and sums in fp32,
+ 2^-22 lv spread                                log2 of a scale and its sum with the score, in fp32,
+ 2^-26 of the largest |v|                       weights below the halves' normal range: 2^-31 of the largest weight each,
                                                 32 times for texts of a few hundred tokens of like weight,
+ 2^-25 (f16)                                    half a step of the subnormal halves."""
import numpy as np
import pytest

from oracle import tokens as ref
from test_gpu_kv8 import HALF_ULP, Cache, _attend

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2208_01944_gb300 import binding
    yield binding
    assert binding.palquant_sync_check() == binding.PQ_OK


def _upload(c):
    for d, h in zip(c.dev, (c.k, c.v, c.ks, c.vs)):
        d.copy_(torch.from_numpy(h))


def _compare(c, q, o, length, kind, scale, columns=slice(None), big=None):
    k, v = ref.read(c.k, c.ks, c.table[0], 0, length), ref.read(c.v, c.vs, c.table[0], 0, length)
    want, spread, top = ref.attention(q, k, v, scale)
    lv = np.abs(np.log2(c.vs[c.vs > 0])).max()
    tol = HALF_ULP[kind] * np.abs(want) + ((2.0 ** -21 if kind == "f32" else 2.0 ** -11) + 2.0 ** -20 * (2 + top) + 2.0 ** -22 * lv) * spread
    tol = tol + 2.0 ** -26 * (np.abs(v).max() if big is None else big) + (2.0 ** -25 if kind == "f16" else 0)
    assert np.all(np.abs(o - want)[..., columns] <= tol[..., columns])
    return want


@pytest.mark.parametrize("kind,loudest", [("f32", 1e-3), ("f32", 1e-6), ("f32", 1e-9), ("bf16", 1e-3), ("bf16", 1e-6), ("bf16", 1e-9),
                                          ("f16", 1e-2), ("f16", 1e-4)])
@pytest.mark.parametrize("n", [1, 150])
@pytest.mark.parametrize("zeros", [[0], [3], [0, 1, 2, 9]], ids=str)
def test_zero_pages_beside_quiet_values(B, zeros, n, kind, loudest):
    """Pages of zero values, first, in the middle and last, with scores above the others': they count in the sum only."""
    T, length = 32, 320
    c = Cache(B, [length], 2, 64, T, seed=n)
    rng = np.random.default_rng(n)
    c.vs[:] = (loudest / 127 * rng.uniform(0.3, 1, c.vs.shape)).astype(np.float32)
    for i in zeros:
        page = c.table[0, i]
        c.v[page], c.vs[page] = 0, 0.0
        c.ks[page] *= 2
    _upload(c)
    q, o, scale = _attend(B, c, [n], [length], 8, kind, True, 0, seed=n, loud=0.2)
    want = _compare(c, q, o, length, kind, scale)
    assert np.abs(want).max() > 0.01 * loudest  # (the other pages are seen)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 150])
def test_only_zero_pages(B, n, kind):
    c = Cache(B, [320], 2, 64, 32, seed=3)
    c.v[:], c.vs[:] = 0, 0.0
    _upload(c)
    _, o, _ = _attend(B, c, [n], [320], 8, kind, True, 0, seed=n)
    assert not o.any()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 150])
@pytest.mark.parametrize("ends", [(-40, -40), (40, 40), (-20, 40)], ids=str)
def test_scales_at_the_ends_of_the_range(B, ends, n, kind):
    """Value scales of 2^-40 and 2^40, a page of zeros beside them: the sum of the weights keeps every page's share."""
    T, length = 32, 320
    c = Cache(B, [length], 2, 64, T, seed=5)
    c.vs[:] = np.float32(2.0) ** ends[0]
    c.vs[c.table[0, 4]] = np.float32(2.0) ** ends[1]
    c.v[c.table[0, 7]], c.vs[c.table[0, 7]] = 0, 0.0
    _upload(c)
    q, o, scale = _attend(B, c, [n], [length], 8, kind, True, 0, seed=n, loud=0.2)
    _compare(c, q, o, length, kind, scale)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 150])
def test_quiet_pages_beside_a_loud_one(B, n, kind):
    """One page 2^19 times as loud as the others, in the first eight columns alone.  The other columns hold what the quiet
    pages add, whose weights are 2^-18 to 2^-20 of the largest: normal halves once they are scaled by 2^6, so the bound
    there has no part of the loud page's values."""
    T, length = 32, 320
    c = Cache(B, [length], 2, 64, T, seed=7)
    c.ks[:] = 1 / 60
    c.vs[:] = np.float32(2.0 ** -10)
    loud = c.table[0, 0]  # every query sees it
    c.vs[loud] = np.float32(2.0 ** 9)
    c.v[loud, :, :, 8:] = 0
    _upload(c)
    q, o, scale = _attend(B, c, [n], [length], 8, kind, True, 0, seed=n, loud=0.05)
    quiet = np.ones(64, bool)
    quiet[:8] = False
    _compare(c, q, o, length, kind, scale, quiet, 0.0)
