"""Norms of query and key heads with the rotation by position, against the oracle in double.

Bound of an output made of magnitudes `size` = |a| + |b|: u |y| for the rounding to the type (u its half step; half precision
below its normal numbers 2^-25), and in fp32 two roundings of a normed value, half the error of D squares' sum (D / 32 + 7
additions and a product each), that of the root and the reciprocal, cosine and sine (2^-22 with their angle's rounding), a
product and a sum: (12 + D / 64) 2^-23 size."""
import numpy as np
import pytest

from oracle import tokens as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2208_01944_gb300 import binding
    yield binding
    assert binding.palquant_sync_check() == binding.PQ_OK


def _check(x, y, weight, eps, positions, frequencies, interleaved, kind, norm=True):
    D = x.shape[2]
    want, size = ref.norm_rope(x.float().cpu().numpy(), None if weight is None else weight.float().cpu().numpy(), eps,
                               positions.cpu().numpy(), frequencies, interleaved, norm)
    got = y.float().cpu().numpy().astype(np.float64)
    tol = HALF_ULP[kind] * np.abs(want) + (12 + D / 64) * 2.0 ** -23 * size + (2.0 ** -25 if kind == "f16" else 0)
    assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) - tol)


def _frequencies(R, theta=10000.0):
    return [theta ** (-2.0 * i / R) for i in range(R // 2)]


CASES = [  # tokens, Hq, Hkv, D, R, interleaved
    (1, 32, 8, 128, 128, False), (1, 1, 1, 2, 2, False), (3, 1, 2, 1, 0, False), (7, 6, 3, 80, 40, True), (7, 6, 3, 80, 40, False),
    (33, 5, 1, 64, 64, False), (33, 5, 1, 64, 64, True), (20, 4, 4, 256, 128, False), (20, 4, 4, 256, 256, True), (9, 2, 2, 96, 96, False),
    (9, 3, 1, 96, 48, True), (5, 2, 1, 1024, 1024, False), (5, 2, 1, 1023, 1022, True), (4, 3, 2, 37, 36, False), (4, 3, 2, 37, 14, True),
    (130, 12, 2, 112, 32, False), (6, 2, 2, 512, 64, False), (2, 100, 3, 32, 32, False), (700, 3, 1, 128, 64, False), (11, 2, 1, 16, 2, False),
    (3, 2, 1, 48, 16, False), (1000, 8, 2, 64, 16, True),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("case", CASES, ids=str)
def test_norm_and_rotation(B, case, kind):
    tokens, Hq, Hkv, D, R, interleaved = case
    rng = np.random.default_rng(D + R)
    dtype = TYPES[kind]
    qkv = torch.from_numpy((rng.normal(size=(tokens, Hq + 2 * Hkv, D)) * np.exp(rng.normal(size=(tokens, Hq + 2 * Hkv, 1)))).astype(np.float32)).to(dtype).cuda()
    q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
    q_out, k_out = torch.full((tokens, Hq, D), 7.0, dtype=dtype, device="cuda"), torch.full((tokens, Hkv, D), 7.0, dtype=dtype, device="cuda")
    wq, wk = (torch.from_numpy((1 + 0.3 * rng.normal(size=D)).astype(np.float32)).to(dtype).cuda() for _ in range(2))
    positions = torch.from_numpy(rng.integers(-5, 100000, tokens).astype(np.int32)).cuda()
    f = _frequencies(R)
    turns = B.rope_turns(f, "cuda") if R else None
    d = B.qk_norm_rope(q, k, q_out, k_out, positions, turns, wq, wk, 1e-6, interleaved)
    before = qkv.clone()
    B.palquant_qk_norm_rope(q, k, q_out, k_out, d)
    assert torch.equal(qkv, before)
    _check(q, q_out, wq, 1e-6, positions, f, interleaved, kind)
    _check(k, k_out, wk, 1e-6, positions, f, interleaved, kind)
    # in place, where the projection wrote them: the same values, and the values' heads are not touched
    B.palquant_qk_norm_rope(q, k, q, k, B.qk_norm_rope(q, k, q, k, positions, turns, wq, wk, 1e-6, interleaved))
    assert torch.equal(q, q_out) and torch.equal(k, k_out) and torch.equal(qkv[:, Hq + Hkv:], before[:, Hq + Hkv:])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("interleaved", [False, True])
def test_strides_and_odd_addresses(B, interleaved, kind):
    """Heads first, each row an odd element into its own; weights of another type."""
    tokens, Hq, Hkv, D = 13, 3, 2, 64
    rng = np.random.default_rng(1)

    def heads(H, fill):
        t = torch.full((H, tokens, D + 3), fill, dtype=TYPES[kind], device="cuda")
        t[:, :, 1:D + 1] = torch.from_numpy(rng.normal(size=(H, tokens, D)).astype(np.float32)).cuda()
        return t, t[:, :, 1:D + 1].transpose(0, 1)

    (qa, q), (ka, k), (qo_all, qo), (ko_all, ko) = heads(Hq, 3.0), heads(Hkv, 3.0), heads(Hq, 5.0), heads(Hkv, 5.0)
    w = torch.from_numpy((1 + 0.3 * rng.normal(size=D)).astype(np.float32)).cuda()
    positions = torch.arange(tokens, dtype=torch.int32, device="cuda") * 977
    f = _frequencies(32, 500000.0)
    B.palquant_qk_norm_rope(q, k, qo, ko, B.qk_norm_rope(q, k, qo, ko, positions, B.rope_turns(f, "cuda"), w, None, 1e-5, interleaved))
    _check(q, qo, w, 1e-5, positions, f, interleaved, kind)
    _check(k, ko, None, 1e-5, positions, f, interleaved, kind)
    for t in (qo_all, ko_all):
        assert bool((t[:, :, 0] == 5).all()) and bool((t[:, :, D + 1:] == 5).all())


def test_queries_alone_rotation_alone_and_norm_alone(B):
    x = torch.randn(50, 4, 128, device="cuda").to(torch.bfloat16)
    y = torch.empty_like(x)
    positions = torch.arange(50, dtype=torch.int32, device="cuda")
    f = _frequencies(128)
    turns = B.rope_turns(f, "cuda")
    B.palquant_qk_norm_rope(x, None, y, None, B.qk_norm_rope(x, None, y, None, positions, turns, norm=False))
    _check(x, y, None, 0, positions, f, False, "bf16", norm=False)
    assert torch.equal(y[0], x[0])  # position 0 turns nothing
    B.palquant_qk_norm_rope(None, x, None, y, B.qk_norm_rope(None, x, None, y, eps=0.0))
    _check(x, y, None, 0.0, positions, [], False, "bf16")


@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions_and_both_signs(B, interleaved):
    """Angles of positions up to the ends of 32 bits: exact to far below fp32's step."""
    positions = torch.tensor([0, 1, -1, 1000003, -1000003, 2 ** 31 - 1, -2 ** 31, 123456789], dtype=torch.int32, device="cuda")
    f = [1.0, 0.7310585786300049, -0.25, 1e-3, 1e-7, 6.5, 2 * np.pi, 0.0]
    x = torch.randn(8, 2, 16, device="cuda")
    y = torch.empty_like(x)
    B.palquant_qk_norm_rope(x, None, y, None, B.qk_norm_rope(x, None, y, None, positions, B.rope_turns(f, "cuda"), norm=False, interleaved=interleaved))
    # the oracle's own angle is a double product: off by up to 2^-53 of it, 2^31 * 6.5 * 2^-53 = 2^-19 at the far end.  Its
    # angles are taken modulo a turn in integers instead: frequency as an exact fraction, pi to 80 digits.
    from fractions import Fraction
    two_pi = 2 * Fraction(31415926535897932384626433832795028841971693993751058209749445923078164062862090, 10 ** 79)
    x64, got = x.double().cpu().numpy(), y.double().cpu().numpy()
    for t, p in enumerate(positions.tolist()):
        for j, freq in enumerate(f):
            angle = float((Fraction(freq) * p) % two_pi)
            a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + 8)
            c, s = np.cos(angle), np.sin(angle)
            size = np.abs(x64[t, :, a]) + np.abs(x64[t, :, b])
            assert np.all(np.abs(got[t, :, a] - (x64[t, :, a] * c - x64[t, :, b] * s)) <= 2.0 ** -21 * size)
            assert np.all(np.abs(got[t, :, b] - (x64[t, :, b] * c + x64[t, :, a] * s)) <= 2.0 ** -21 * size)


def test_extremes_stay_in_their_head(B):
    x = torch.randn(4, 3, 64, device="cuda")
    x[0, 1, 5], x[1, 0, 40], x[2, 2] = float("nan"), float("inf"), 0.0
    x[3, 0] *= 2.0 ** 58
    x[3, 1] *= 2.0 ** -60
    y = torch.empty_like(x)
    positions = torch.arange(4, dtype=torch.int32, device="cuda")
    f = _frequencies(64)
    B.palquant_qk_norm_rope(x, None, y, None, B.qk_norm_rope(x, None, y, None, positions, B.rope_turns(f, "cuda"), eps=1e-12))
    assert torch.isnan(y[0, 1]).all() and torch.isnan(y[1, 0]).any() and not y[2, 2].any()
    keep = torch.ones(4, 3, dtype=torch.bool)
    keep[0, 1] = keep[1, 0] = False
    want, size = ref.norm_rope(x.cpu().numpy()[keep.numpy()][:, None], None, 1e-12, positions.cpu().numpy().repeat(3)[keep.numpy().ravel()], f, False)
    assert np.all(np.abs(y.cpu().numpy()[keep.numpy()][:, None] - want) <= 14 * 2.0 ** -23 * size + 2.0 ** -24 * np.abs(want) + 1e-45)


def test_many_tokens(B):
    """More blocks than stand at one time, a last one that is not full; every token its own position."""
    tokens = 40003
    x = torch.randn(tokens, 3, 32, device="cuda").half()
    y = torch.full_like(x, 7.0)
    positions = torch.randperm(tokens, device="cuda").to(torch.int32)
    f = _frequencies(32)
    w = torch.rand(32, device="cuda").half() + 0.5
    B.palquant_qk_norm_rope(x[:, :2], x[:, 2:], y[:, :2], y[:, 2:], B.qk_norm_rope(x[:, :2], x[:, 2:], y[:, :2], y[:, 2:], positions, B.rope_turns(f, "cuda"), w, w))
    _check(x, y, w, 1e-6, positions, f, False, "f16")


def test_offsets_past_32_bits(B):
    """Rows whose elements lie beyond 2^32 of the tensor's first."""
    store = torch.zeros((1 << 32) + 4096, dtype=torch.float16, device="cuda")
    x = store.as_strided((2, 2, 64), ((1 << 32), 64, 1), 8)
    x.copy_(torch.randn(2, 2, 64, device="cuda"))
    y = torch.empty(2, 2, 64, dtype=torch.float16, device="cuda")
    positions = torch.tensor([5, 900], dtype=torch.int32, device="cuda")
    f = _frequencies(64)
    B.palquant_qk_norm_rope(x, None, y, None, B.qk_norm_rope(x, None, y, None, positions, B.rope_turns(f, "cuda")))
    _check(x, y, None, 1e-6, positions, f, False, "f16")


def test_captured_calls_read_their_positions_anew(B):
    x = torch.randn(5, 8, 128, device="cuda").to(torch.bfloat16)
    y = torch.empty_like(x)
    positions = torch.arange(5, dtype=torch.int32, device="cuda")
    f = _frequencies(128)
    d = B.qk_norm_rope(x, None, y, None, positions, B.rope_turns(f, "cuda"))
    B.palquant_qk_norm_rope(x, None, y, None, d)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.palquant_qk_norm_rope(x, None, y, None, d)
    for step in (3, 10000):
        positions += step
        graph.replay()
        _check(x, y, None, 1e-6, positions, f, False, "bf16")


@pytest.mark.parametrize("D", [24, 27])
@pytest.mark.parametrize("interleaved", [False, True])
def test_small_angles_keep_their_sine(B, interleaved, D):
    """Heads of (1, 0) pairs come out as cosines and sines: each right relative to itself, near whole and quarter turns too.

    Bound: frequencies are off by up to 2 units of 2^-64 turns a position (|p| 2^-60 in radians); the angle's remainder is rounded to fp32 (2^-24
    of it, and of its sine); sine and cosine have an error of 2 units at most (2^-22)."""
    from fractions import Fraction
    pi = Fraction(31415926535897932384626433832795028841971693993751058209749445923078164062862090, 10 ** 79)
    f = [1e-6, 1e-7, 3.3e-9, np.pi * (1 + 1e-6), np.pi / 2 * (1 - 1e-7), 2 * np.pi * (1 + 1e-8), -4e-7, 1e-3]
    positions = torch.tensor([1, 2, 3, -1, 77, -1000], dtype=torch.int32, device="cuda")
    x = torch.zeros(len(positions), 1, D, device="cuda")
    a, b = (slice(0, 16, 2), slice(1, 16, 2)) if interleaved else (slice(0, 8), slice(8, 16))
    x[..., a] = 1
    y = torch.empty_like(x)
    B.palquant_qk_norm_rope(x, None, y, None, B.qk_norm_rope(x, None, y, None, positions, B.rope_turns(f, "cuda"), norm=False, interleaved=interleaved))
    got = y.double().cpu().numpy()[:, 0]
    for t, p in enumerate(positions.tolist()):
        for j, freq in enumerate(f):
            angle = Fraction(freq) * p
            quarter = round(angle / (pi / 2))
            rest = float(angle - quarter * pi / 2)
            c, s = [(np.cos(rest), np.sin(rest)), (-np.sin(rest), np.cos(rest)), (-np.cos(rest), -np.sin(rest)), (np.sin(rest), -np.cos(rest))][quarter % 4]
            for value, want in ((got[t, a][j], c), (got[t, b][j], s)):
                assert abs(value - want) <= (2.0 ** -22 + 2.0 ** -24) * abs(want) + abs(p) * 2.0 ** -60, (p, freq, value, want)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("D,R,interleaved", [(64, 32, False), (64, 32, True), (64, 6, True), (128, 0, False), (128, 96, False), (37, 10, False), (37, 10, True), (80, 40, False)])
def test_elements_behind_the_rotated_part_stay_as_they_are(B, D, R, interleaved, kind):
    """Without a norm they are copied: infinities, NaN and zeros of either sign do not meet their neighbours."""
    x = torch.randn(9, 3, D, device="cuda").to(TYPES[kind])
    x[0, 0, R], x[1, 1, D - 1], x[2, 2, R + 3], x[3, 0, R::2] = float("inf"), float("-inf"), float("nan"), -0.0
    y = torch.empty_like(x)
    positions = torch.arange(9, dtype=torch.int32, device="cuda") * 1001
    turns = B.rope_turns(_frequencies(R), "cuda") if R else None
    B.palquant_qk_norm_rope(x, None, y, None, B.qk_norm_rope(x, None, y, None, positions, turns, norm=False, interleaved=interleaved))
    same = lambda t: torch.where(torch.isnan(t), 0, t.view(torch.int32 if kind == "f32" else torch.int16))  # noqa: E731  (bits, but for those of a NaN)
    assert torch.equal(torch.isnan(y[..., R:]), torch.isnan(x[..., R:]))
    assert torch.equal(same(y[..., R:].contiguous()), same(x[..., R:].contiguous()))
    assert torch.isfinite(y[..., :R]).all()


@pytest.mark.parametrize("D,R,interleaved", [(64, 32, False), (64, 32, True), (37, 10, False)])
def test_a_product_past_the_type_stays_its_own(B, D, R, interleaved):
    """A weight that takes one normed element behind the rotated part to infinity."""
    x = torch.randn(5, 2, D, device="cuda")
    x[:, :, R + 1] = x.abs().amax(2) + 2
    w = torch.ones(D, device="cuda")
    w[R + 1] = 3e38
    y = torch.empty_like(x)
    positions = torch.arange(5, dtype=torch.int32, device="cuda")
    B.palquant_qk_norm_rope(x, None, y, None, B.qk_norm_rope(x, None, y, None, positions, B.rope_turns(_frequencies(R), "cuda"), w, interleaved=interleaved))
    assert torch.isinf(y[:, :, R + 1]).all()
    keep = [d for d in range(D) if d != R + 1]
    want, size = ref.norm_rope(x.cpu().numpy(), w.cpu().numpy(), 1e-6, positions.cpu().numpy(), _frequencies(R), interleaved)
    assert np.all(np.abs(y.cpu().numpy().astype(np.float64) - want)[..., keep] <= ((2.0 ** -24 * np.abs(want) + 14 * 2.0 ** -23 * size))[..., keep])


@pytest.mark.parametrize("kind", list(TYPES))
def test_outputs_between_other_heads(B, kind):
    """In place where queries, keys and values of a head lie side by side; into the heads beside the inputs; heads first."""
    tokens, H, D = 11, 3, 64
    f = _frequencies(D)
    turns, positions = B.rope_turns(f, "cuda"), torch.arange(tokens, dtype=torch.int32, device="cuda") * 13

    def turn(q, k, q_out, k_out):
        q0, k0 = q.clone(), k.clone()
        B.palquant_qk_norm_rope(q, k, q_out, k_out, B.qk_norm_rope(q, k, q_out, k_out, positions, turns))
        _check(q0, q_out, None, 1e-6, positions, f, False, kind)
        _check(k0, k_out, None, 1e-6, positions, f, False, kind)

    x = torch.randn(tokens, H, 3, D, device="cuda").to(TYPES[kind])
    values = x[:, :, 2].clone()
    turn(x[:, :, 0], x[:, :, 1], x[:, :, 0], x[:, :, 1])
    assert torch.equal(x[:, :, 2], values)
    x = torch.randn(tokens, 12, D, device="cuda").to(TYPES[kind])
    before = x.clone()
    turn(x[:, 0::4], x[:, 1::4], x[:, 2::4], x[:, 3::4])
    assert torch.equal(x[:, 0::4], before[:, 0::4]) and torch.equal(x[:, 1::4], before[:, 1::4])
    x = torch.randn(5, tokens, D, device="cuda").to(TYPES[kind]).transpose(0, 1)
    turn(x[:, :3], x[:, 3:], x[:, :3], x[:, 3:])
