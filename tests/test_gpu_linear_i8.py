"""Dense layers on 8-bit tokens and weights: codes, scales and int32 sums equal the
oracle's bit for bit; the float outputs lie within their roundings of the value in
double (three fp32 roundings before the bias, one with it, one to the output type)."""
import numpy as np
import pytest

from oracle import tokens as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 0.0, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}  # relative, of normal numbers
F16_TINY = 2.0 ** -25  # half a step of the subnormal halves


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2208_01944_gb300 import binding
    yield binding
    assert binding.palquant_sync_check() == binding.PQ_OK


def _x(M, K, kind, seed):
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(M, K)) * np.exp(rng.normal(size=(1, K)) * 0.5)
    x[rng.integers(0, M), :] = 0 if M > 2 else 1  # a token of zeros
    return torch.from_numpy(x.astype(np.float32)).to(TYPES[kind]).cuda()


def _f32(t):
    return t.float().cpu().numpy()


def _weights(N, K, seed):
    rng = np.random.default_rng(seed + 1)
    return rng.integers(-128, 128, (N, K)).astype(np.int8), (rng.uniform(0.5, 2, N) / 127).astype(np.float32)


def _check_y(y, acc, s_x, s_w, bias, kind):
    want = ref.linear_value(acc, s_x, s_w)
    tol = np.abs(want) * 3 * 2.0 ** -24
    if bias is not None:
        want = want + bias.astype(np.float64)
        tol = tol + (np.abs(want) + tol) * 2.0 ** -24
    tol = tol + (np.abs(want) + tol) * HALF_ULP[kind] + (F16_TINY if kind == "f16" else 0) + 2.0 ** -140
    assert np.all(np.abs(_f32(y).astype(np.float64) - want) <= tol)


SIZES = [(1, 1, 1), (1, 16, 64), (2, 17, 15), (3, 40, 63), (8, 64, 128), (9, 33, 65), (16, 128, 1040), (17, 100, 777),
         (32, 257, 2048), (33, 130, 500), (70, 256, 4096), (129, 129, 129), (200, 384, 1088), (257, 1000, 320),
         (300, 520, 2500), (1, 64, 20000)]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_layer_matches_the_oracle(B, size, kind):
    M, N, K = size
    x = _x(M, K, kind, M * 7 + K)
    w, s_w = _weights(N, K, N + K)
    bias = np.random.default_rng(3).normal(size=N).astype(np.float32) if (M + N) % 2 else None
    q, s_x = ref.quantize_tokens(_f32(x))
    acc = ref.linear(q, w)
    wd, sd = torch.from_numpy(w).cuda(), torch.from_numpy(s_w).cuda()
    bd = None if bias is None else torch.from_numpy(bias).cuda()
    y = torch.full((M, N), 7.0, dtype=TYPES[kind], device="cuda")
    d = B.linear_desc(x, wd, y)
    scratch = torch.empty(B.palquant_linear_q8_scratch_bytes(d), dtype=torch.uint8, device="cuda")
    B.palquant_linear_q8(x, wd, sd, bd, y, d, scratch, scratch.numel())
    _check_y(y, acc, s_x, s_w, bias, kind)
    for fmt, dtype in ((B.PQ_CODES_INT8, torch.int8), (B.PQ_CODES_F16, torch.float16)):
        codes = torch.full((M, K), 5, dtype=dtype, device="cuda")
        scales = torch.empty(M, device="cuda")
        B.palquant_quantize_tokens(x, d.x_type, d.ldx, M, K, fmt, codes, K, scales)
        assert np.array_equal(codes.cpu().numpy().astype(np.int8), q)
        assert np.array_equal(scales.cpu().numpy(), s_x)
        sums = torch.full((M, N), -9, dtype=torch.int32, device="cuda")
        y2 = torch.full((M, N), 7.0, dtype=TYPES[kind], device="cuda")
        B.palquant_linear_i8(codes, fmt, K, scales, wd, sd, bd, sums, y2, d)
        assert np.array_equal(sums.cpu().numpy(), acc)
        assert torch.equal(y2, y)


@pytest.mark.parametrize("fmt", ["PQ_CODES_INT8", "PQ_CODES_F16"])
@pytest.mark.parametrize("M,N,K", [(1, 32, 131072), (40, 48, 16384), (300, 256, 8192)])
def test_sums_are_exact_at_the_ends_of_the_range(B, M, N, K, fmt):
    """All products of one sign and of the largest size: sums far above 2^24 stay exact."""
    rng = np.random.default_rng(K)
    q = np.where(rng.random((M, K)) < 0.001, 126, 127).astype(np.int8)
    q[M // 2] *= -1
    w = np.where(rng.random((N, K)) < 0.001, -127, -128).astype(np.int8)
    w[N // 2] = 127
    f = getattr(B, fmt)
    qd = torch.from_numpy(q).cuda().to(torch.float16 if f == B.PQ_CODES_F16 else torch.int8)
    wd = torch.from_numpy(w).cuda()
    sums = torch.empty((M, N), dtype=torch.int32, device="cuda")
    y = torch.empty((M, N), device="cuda")
    d = B.linear_desc(torch.empty((M, K), device="cuda"), wd, y)
    B.palquant_linear_i8(qd, f, K, None, wd, None, None, sums, None, d)
    assert np.array_equal(sums.cpu().numpy(), ref.linear(q, w))


@pytest.mark.parametrize("M,N,K", [(3, 40, 200), (150, 140, 333)])
def test_strides_and_alignments(B, M, N, K):
    """Rows inside larger matrices, at addresses that no wide access may use; what lies around the outputs stays."""
    rng = np.random.default_rng(5)
    big = torch.from_numpy(rng.normal(size=(M, K + 13)).astype(np.float32)).cuda().to(torch.bfloat16)
    x = big[:, 3:3 + K]
    w, s_w = _weights(N, K, 11)
    wbig = torch.zeros((N, K + 7), dtype=torch.int8, device="cuda")
    wbig[:, 5:5 + K] = torch.from_numpy(w).cuda()
    wd, sd = wbig[:, 5:5 + K], torch.from_numpy(s_w).cuda()
    ybig = torch.full((M, N + 9), 7.0, dtype=torch.float16, device="cuda")
    y = ybig[:, 1:1 + N]
    d = B.linear_desc(x, wd, y)
    scratch = torch.empty(B.palquant_linear_q8_scratch_bytes(d), dtype=torch.uint8, device="cuda")
    B.palquant_linear_q8(x, wd, sd, None, y, d, scratch, scratch.numel())
    q, s_x = ref.quantize_tokens(_f32(x))
    acc = ref.linear(q, w)
    _check_y(y, acc, s_x, s_w, None, "f16")
    assert bool((ybig[:, 0] == 7).all()) and bool((ybig[:, 1 + N:] == 7).all())
    for fmt, dtype in ((B.PQ_CODES_INT8, torch.int8), (B.PQ_CODES_F16, torch.float16)):
        qbig = torch.full((M, K + 5), 3, dtype=dtype, device="cuda")
        codes, scales = qbig[:, 1:1 + K], torch.empty(M, device="cuda")
        B.palquant_quantize_tokens(x, d.x_type, d.ldx, M, K, fmt, codes, K + 5, scales)
        assert np.array_equal(codes.cpu().numpy().astype(np.int8), q)
        assert bool((qbig[:, 0] == 3).all()) and bool((qbig[:, 1 + K:] == 3).all())
        sums = torch.empty((M, N), dtype=torch.int32, device="cuda")
        B.palquant_linear_i8(codes, fmt, K + 5, scales, wd, sd, None, sums, None, d)
        assert np.array_equal(sums.cpu().numpy(), acc)


@pytest.mark.parametrize("M,N,K,gap", [(17, 40, 131071, 0), (41, 2600, 2601, 0), (400, 700, 1001, 6), (300, 640, 1600, 3)])
def test_many_tokens_on_weight_rows_off_16_bytes(B, M, N, K, gap):
    """Weight rows at any address: columns of a wider matrix, `gap` bytes in, or of odd length."""
    x = _x(M, K, "bf16", K)
    w, s_w = _weights(N, K, N)
    wbig = torch.full((N, K + gap), 99, dtype=torch.int8, device="cuda")
    wd, sd = wbig[:, gap:], torch.from_numpy(s_w).cuda()
    wd.copy_(torch.from_numpy(w))
    y = torch.full((M, N), 7.0, device="cuda")
    d = B.linear_desc(x, wd, y)
    need = B.palquant_linear_q8_scratch_bytes(d)
    assert need >= N * K or M * N * K < 2 ** 28  # the copy of the weights
    scratch = torch.full((need + 64,), 171, dtype=torch.uint8, device="cuda")
    B.palquant_linear_q8(x, wd, sd, None, y, d, scratch, need)
    q, s_x = ref.quantize_tokens(_f32(x))
    _check_y(y, ref.linear(q, w), s_x, s_w, None, "f32")
    assert bool((scratch[need:] == 171).all())


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("M,N,K,shift", [(1, 33, 16, 0), (1, 100, 500, 1), (2, 65, 513, 0), (3, 129, 1024, 3), (4, 260, 1030, 0),
                                         (4, 64, 4096, 0), (1, 48, 16384, 0), (5, 48, 1100, 0), (2, 31, 8200, 1)])
def test_few_tokens_on_padded_weight_rows(B, M, N, K, shift, kind):
    """One to five tokens, weight rows padded to 16 bytes, token rows `shift` elements into a wider matrix."""
    x = _x(M, K, kind, K + M)
    xbig = torch.full((M, K + 8), 1e4, dtype=TYPES[kind], device="cuda")
    xbig[:, shift:shift + K] = x
    w, s_w = _weights(N, K, N + M)
    wbig = torch.full((N, -(-K // 16) * 16), 77, dtype=torch.int8, device="cuda")
    wbig[:, :K] = torch.from_numpy(w).cuda()
    xs, wd, sd = xbig[:, shift:shift + K], wbig[:, :K], torch.from_numpy(s_w).cuda()
    bias = np.random.default_rng(4).normal(size=N).astype(np.float32) if M % 2 else None
    y = torch.full((M, N + 3), 7.0, dtype=TYPES[kind], device="cuda")
    d = B.linear_desc(xs, wd, y[:, 1:1 + N])
    scratch = torch.empty(B.palquant_linear_q8_scratch_bytes(d), dtype=torch.uint8, device="cuda")
    B.palquant_linear_q8(xs, wd, sd, None if bias is None else torch.from_numpy(bias).cuda(), y[:, 1:1 + N], d, scratch,
                         scratch.numel())
    q, s_x = ref.quantize_tokens(_f32(x))
    _check_y(y[:, 1:1 + N], ref.linear(q, w), s_x, s_w, bias, kind)
    assert bool((y[:, 0] == 7).all()) and bool((y[:, 1 + N:] == 7).all())


@pytest.mark.parametrize("M", [4, 160])
def test_non_finite_tokens_poison_themselves_only(B, M):
    K, N = 256, 144
    x = _x(M, K, "f32", 1)
    x[1, 7], x[2, 255], x[3, 0] = float("nan"), float("inf"), -float("inf")
    x[0] *= 1e-30
    x[0, 0] = 2.0 ** -121  # amax / 127 below the smallest normal: codes 0
    x[0, 1:] = 0
    w, s_w = _weights(N, K, 2)
    wd, sd = torch.from_numpy(w).cuda(), torch.from_numpy(s_w).cuda()
    y = torch.empty((M, N), device="cuda")
    d = B.linear_desc(x, wd, y)
    scratch = torch.empty(B.palquant_linear_q8_scratch_bytes(d), dtype=torch.uint8, device="cuda")
    B.palquant_linear_q8(x, wd, sd, None, y, d, scratch, scratch.numel())
    out = _f32(y)
    assert np.isnan(out[1:4]).all() and (out[0] == 0).all()
    q, s_x = ref.quantize_tokens(_f32(x))
    assert np.isnan(s_x[1:4]).all() and s_x[0] == 0 and not q[:4].any()
    _check_y(y[4:], ref.linear(q[4:], w), s_x[4:], s_w, None, "f32") if M > 4 else None


def test_rounding_ties_are_to_even(B):
    """amax 127 makes the scale one rounding away from 1; halves around it follow the fp32 product."""
    x = np.zeros((2, 64), np.float32)
    x[0, :6] = [127, 0.5, 1.5, 2.5, -0.5, -1.5]
    x[1, :6] = [254, 127, 1, 3, -5, 63.5]
    xd = torch.from_numpy(x).cuda()
    codes, s = torch.empty((2, 64), dtype=torch.int8, device="cuda"), torch.empty(2, device="cuda")
    B.palquant_quantize_tokens(xd, B.PQ_F32, 64, 2, 64, B.PQ_CODES_INT8, codes, 64, s)
    q, sr = ref.quantize_tokens(x)
    assert np.array_equal(codes.cpu().numpy(), q) and np.array_equal(s.cpu().numpy(), sr)


def test_another_stream_and_a_graph(B):
    """The call runs on the stream it is given, and in a captured graph."""
    M, N, K = 64, 512, 1024
    x = _x(M, K, "bf16", 9)
    w, s_w = _weights(N, K, 4)
    wd, sd = torch.from_numpy(w).cuda(), torch.from_numpy(s_w).cuda()
    y, y2 = (torch.zeros((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    d = B.linear_desc(x, wd, y)
    scratch = torch.empty(B.palquant_linear_q8_scratch_bytes(d), dtype=torch.uint8, device="cuda")
    B.palquant_linear_q8(x, wd, sd, None, y, d, scratch, scratch.numel())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.palquant_linear_q8(x, wd, sd, None, y2, d, scratch, scratch.numel(), stream=side)
    side.synchronize()
    assert torch.equal(y, y2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.palquant_linear_q8(x, wd, sd, None, y2, d, scratch, scratch.numel())
    y2.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, y2)
