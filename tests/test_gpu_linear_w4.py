"""Dense layers with 4-bit weights and group scales, against the oracle in double.

Codes and scales are exact.  Bound of an output whose products' magnitudes sum to `size`: u |y| for the rounding to the
type (u its half step; half precision below its normal numbers 2^-25), and the sums.  Products are exact; a tensor-core sum may cut instead of
round, so each of the fp32 additions on the way of a product loses at most 2^-23 of its operands: 16 within a 16-wide step
counted as one cut of 2^-22 each for up to 24 such steps of a group (8 steps, three parts for fp32), one product with
the scale, and at most one addition for each 128 of K and 24 for joining: (2 * 24 + K / 128 + 26) 2^-23 size."""
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


def _pack(B, codes, scales, group):
    w = B.w4_weights(*codes.shape, group, scales.dtype)
    packed = torch.full((B.palquant_w4_packed_bytes(w),), 255, dtype=torch.uint8, device="cuda")
    B.palquant_w4_pack(codes, scales, w, packed, packed.numel())
    return w, packed


def _weights(N, K, group, s_kind, seed):
    rng = np.random.default_rng(seed)
    codes = torch.from_numpy(rng.integers(-8, 8, (N, K)).astype(np.int8)).cuda()
    scales = torch.from_numpy((np.exp(rng.normal(size=(N, -(-K // group)))) / 8).astype(np.float32)).to(TYPES[s_kind]).cuda()
    return codes, scales


def _run(B, w, packed, x, y, bias=None):
    d = B.linear_w4_desc(x, w, y)
    nbytes = B.palquant_linear_w4_scratch_bytes(w, d)
    scratch = torch.full((max(1, nbytes),), 255, dtype=torch.uint8, device="cuda")
    B.palquant_linear_w4(x, packed, bias, y, w, d, scratch, nbytes)
    return y


def _check(x, y, codes, scales, group, kind, bias=None):
    K = codes.shape[1]
    want, size = ref.linear_w4(x.float().cpu().numpy(), codes.cpu().numpy(), scales.float().cpu().numpy(), group,
                               None if bias is None else bias.cpu().numpy())
    got = y.float().cpu().numpy().astype(np.float64)
    tol = HALF_ULP[kind] * np.abs(want) + (74 + K / 128) * 2.0 ** -23 * size + (2.0 ** -25 if kind == "f16" else 0)
    assert np.all(np.abs(got - want) <= tol), np.max((np.abs(got - want) - tol) / size)


@pytest.mark.parametrize("s_kind", list(TYPES))
@pytest.mark.parametrize("N,K,group", [(16, 128, 128), (1, 1, 32), (17, 129, 64), (100, 1000, 32), (33, 777, 128), (48, 95, 64)])
def test_packed_weights_come_back(B, N, K, group, s_kind):
    codes, scales = _weights(N, K, group, s_kind, K)
    w, packed = _pack(B, codes, scales, group)
    back, s = torch.full((N, K + 5), 99, dtype=torch.int8, device="cuda"), torch.empty(scales.shape, device="cuda")
    B.palquant_w4_unpack(packed, w, back[:, :K], s)
    assert torch.equal(back[:, :K], codes) and torch.equal(s, scales.float()) and bool((back[:, K:] == 99).all())
    wide = torch.full((N, K + 3), 100, dtype=torch.int8, device="cuda")  # rows with a pitch; only the low 4 bits count
    wide[:, :K] = codes + 16 * (torch.arange(K, device="cuda", dtype=torch.int8) % 3)
    again = torch.full_like(packed, 255)
    B.palquant_w4_pack(wide[:, :K], scales, w, again, again.numel())
    assert torch.equal(again, packed)


@pytest.mark.parametrize("s_kind", list(TYPES))
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("N,K,group,pitch", [(5, 64, 32, 64), (33, 300, 128, 300), (40, 1001, 64, 1007), (20, 256, 32, 264)])
def test_quantised_weights(B, N, K, group, pitch, kind, s_kind):
    rng = np.random.default_rng(N)
    dtype, s_type = TYPES[kind], TYPES[s_kind]
    full = torch.from_numpy((rng.normal(size=(N, pitch)) * np.exp(3 * rng.normal(size=(N, 1)))).astype(np.float32)).to(dtype).cuda()
    full[1, :K] = 0
    full[2, 3], full[3, K - 1] = float("nan"), float("inf")
    if kind != "f16":
        full[4, :K] *= 2.0 ** -140 if kind == "f32" else 2.0 ** -130  # below the normal numbers
        full[0, :group] *= 2.0 ** 40  # (past half precision's scales)
    w = B.w4_weights(N, K, group, s_type)
    packed = torch.full((B.palquant_w4_packed_bytes(w),), 255, dtype=torch.uint8, device="cuda")
    number = {torch.float32: B.PQ_F32, torch.float16: B.PQ_F16, torch.bfloat16: B.PQ_BF16}[dtype]
    B.palquant_w4_quantize(full, number, pitch, w, packed, packed.numel())
    codes, scales = torch.empty((N, K), dtype=torch.int8, device="cuda"), torch.empty((N, -(-K // group)), device="cuda")
    B.palquant_w4_unpack(packed, w, codes, scales)
    want, s = ref.w4_quantize(full[:, :K].float().cpu().numpy(), group, lambda v: torch.from_numpy(v).to(s_type).float().numpy(),
                              np.float32(2.0 ** -14 if s_kind == "f16" else 2.0 ** -126))
    assert np.array_equal(scales.cpu().numpy(), s, equal_nan=True)
    assert np.array_equal(codes.cpu().numpy(), want)


SIZES = [  # M, N, K, group
    (1, 1, 1, 32), (1, 16, 128, 128), (2, 17, 31, 32), (3, 100, 129, 64), (5, 1001, 777, 32), (7, 48, 2048, 128), (8, 64, 4096, 64),
    (9, 33, 1000, 128), (16, 80, 512, 32), (17, 40, 640, 64), (31, 130, 1111, 128), (33, 65, 384, 32), (48, 256, 1024, 64), (64, 31, 900, 128),
    (65, 20, 260, 64), (200, 37, 300, 32), (1, 5000, 256, 64), (4, 12, 20000, 128), (1, 300, 8192, 32),
    # many stages and slots in a block, of every tile width and group; many tiles a block; parts of K in clusters
    (20, 130, 9000, 32), (20, 260, 9001, 64), (25, 140, 9100, 128), (40, 300, 9000, 32), (64, 129, 8960, 64), (57, 140, 9100, 128), (100, 300, 9000, 32),
    (128, 150, 8900, 64), (120, 140, 9100, 128), (300, 2600, 640, 64), (30, 21000, 512, 32), (260, 1300, 1536, 128), (24, 1024, 4096, 128),
    # pairs of strips, the last one alone; few tokens
    (1, 9760, 520, 128), (8, 9744, 300, 32), (16, 2064, 700, 64), (12, 2049, 513, 128), (3, 12000, 260, 64),
    # fewer columns than a load of the tensor cores takes; a last tile of one strip
    (20, 130007, 33, 32), (33, 66000, 70, 64),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("case", SIZES, ids=str)
def test_products(B, case, kind):
    M, N, K, group = case
    s_kind = ["f16", "bf16", "f32"][(M + N) % 3]
    codes, scales = _weights(N, K, group, s_kind, M + K)
    w, packed = _pack(B, codes, scales, group)
    rng = np.random.default_rng(M)
    x = torch.from_numpy((rng.normal(size=(M, K)) * np.exp(rng.normal(size=K))).astype(np.float32)).to(TYPES[kind]).cuda()
    bias = torch.from_numpy(rng.normal(size=N).astype(np.float32)).cuda() if N % 2 else None
    y = torch.full((M, N), 7.0, dtype=TYPES[kind], device="cuda")
    _run(B, w, packed, x, y, bias)
    _check(x, y, codes, scales, group, kind, bias)


@pytest.mark.parametrize("M", [1, 6, 20, 50])
@pytest.mark.parametrize("kind", list(TYPES))
def test_pitches_odd_addresses_and_other_output_types(B, kind, M):
    N, K, group = 50, 333, 64
    codes, scales = _weights(N, K, group, "f16", 3)
    w, packed = _pack(B, codes, scales, group)
    for pad, shift, out in ((5, 1, "f32"), (8 + 3, 8, "bf16"), (0, 0, "f16"), (K % 8 and 8 - K % 8, 0, "f32"), (2, 1, "f32"), (2, 8, "f32")):
        store = torch.full((M, K + pad + 9), float("nan"), dtype=TYPES[kind], device="cuda")  # what lies beside the rows is not read
        x = store[:, shift:shift + K]
        x.copy_(torch.randn(M, K, device="cuda"))
        y_all = torch.full((M, N + 4), 9.0, dtype=TYPES[out], device="cuda")
        y = y_all[:, 1:N + 1]
        _run(B, w, packed, x, y)
        _check(x, y, codes, scales, group, out)
        assert bool((y_all[:, 0] == 9).all()) and bool((y_all[:, N + 1:] == 9).all())


@pytest.mark.parametrize("M", [2, 40])
@pytest.mark.parametrize("kind", list(TYPES))
def test_extremes_stay_in_their_row_and_channel(B, kind, M):
    N, K, group = 40, 256, 64
    codes, scales = _weights(N, K, group, "f32", 5)
    codes[codes == 0] = 1
    scales[3, 1] = float("nan")
    w, packed = _pack(B, codes, scales, group)
    x = torch.randn(M, K, device="cuda").to(TYPES[kind])
    x[1, 7] = float("inf")
    x[0, 9] = 2.0 ** 15 if kind == "f16" else 2.0 ** 116  # (8 * 2^116 and the group's other products stay in fp32)
    scales_small = scales * 2.0 ** -40
    w2, packed2 = _pack(B, codes, scales_small, group)
    y = _run(B, w2, packed2, x, torch.empty(M, N, device="cuda"))
    assert torch.isnan(y[:, 3]).all()
    rest = [n for n in range(N) if n != 3]
    assert torch.isinf(y[1, rest]).all()
    rows = [m for m in range(M) if m != 1]
    _check(x[rows], y[rows][:, rest], codes[rest], scales_small[rest], group, "f32")


def test_bits_do_not_depend_on_the_batch_and_do_not_change(B):
    codes, scales = _weights(300, 4096, 128, "f16", 9)
    w, packed = _pack(B, codes, scales, 128)
    x = torch.randn(8, 4096, device="cuda").to(torch.bfloat16)
    y = [_run(B, w, packed, x, torch.empty(8, 300, dtype=torch.bfloat16, device="cuda")) for _ in range(3)]
    assert torch.equal(y[0], y[1]) and torch.equal(y[0], y[2])


def test_captured_on_two_streams(B):
    codes, scales = _weights(512, 2048, 128, "f16", 10)
    w, packed = _pack(B, codes, scales, 128)
    calls = []
    for M in (1, 24):
        x, y = torch.randn(M, 2048, device="cuda").half(), torch.empty(M, 512, dtype=torch.float16, device="cuda")
        d = B.linear_w4_desc(x, w, y)
        scratch = torch.empty(max(1, B.palquant_linear_w4_scratch_bytes(w, d)), dtype=torch.uint8, device="cuda")
        B.palquant_linear_w4(x, packed, None, y, w, d, scratch, scratch.numel())
        torch.cuda.synchronize()
        want = y.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.palquant_linear_w4(x, packed, None, y, w, d, scratch, scratch.numel())
        calls.append((x, y, want, graph, scratch, d, torch.cuda.Stream()))
    for _ in range(4):
        for x, y, want, graph, scratch, d, stream in calls:
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                y.zero_()
                graph.replay()
        torch.cuda.synchronize()
        for x, y, want, *_ in calls:
            assert torch.equal(y, want)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("M", [1, 5, 40, 300])
def test_outputs_beside_the_tokens(B, M, kind):
    """Columns of their own in the tokens' rows, before and behind them; the rest of the rows stays."""
    N, K, group = 96, 256, 64
    codes, scales = _weights(N, K, group, "f32", M)
    w, packed = _pack(B, codes, scales, group)
    rng = np.random.default_rng(M)
    rows = torch.from_numpy(rng.normal(size=(M, 100 + K + 100)).astype(np.float32)).to(TYPES[kind]).cuda()
    x = rows[:, 100:100 + K].clone()
    for at in (0, 100 + K):
        before = rows.clone()
        _run(B, w, packed, rows[:, 100:100 + K], rows[:, at:at + N])
        _check(x, rows[:, at:at + N], codes, scales, group, kind)
        before[:, at:at + N] = rows[:, at:at + N]
        assert torch.equal(rows, before)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(9, 150, 20000), (32, 40, 20001), (33, 20000, 1100), (64, 260, 9000)])
def test_three_parts_of_a_token_through_many_stages(B, M, N, K, group):
    """fp32 tokens on the tensor cores: rings of stages that go round many times, in one tile, in several and in parts of K."""
    codes, scales = _weights(N, K, group, "f32", M + group)
    w, packed = _pack(B, codes, scales, group)
    x = torch.randn(M, K, device="cuda", generator=torch.Generator(device="cuda").manual_seed(M))
    y = torch.full((M, N), 7.0, device="cuda")
    for _ in range(3):
        _check(x, _run(B, w, packed, x, y), codes, scales, group, "f32")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("N,K,M", [(300, 4096, 8), (9760, 520, 8), (2064, 700, 16)])
def test_a_token_has_the_same_bits_in_any_batch_of_one_kernel(B, N, K, M, kind):
    """Up to 8 tokens, and 16-bit ones from 9 to 16, are one kernel of tiles each; what else is in the batch, and where, does not count."""
    codes, scales = _weights(N, K, 128, "f16", 9)
    w, packed = _pack(B, codes, scales, 128)
    x = torch.randn(M, K, device="cuda").to(TYPES[kind])
    first = 1 if M <= 8 else 9
    if kind == "f32" and M > 8:
        first, M, x = 1, 8, x[:8]
    whole = _run(B, w, packed, x, torch.empty(M, N, dtype=x.dtype, device="cuda"))
    for rows in (list(range(first)), list(range(M - first, M)), list(range(M))[::-1], [M - 1] * first, list(range(M))[:first + 2]):
        part = x[rows].contiguous()
        assert torch.equal(_run(B, w, packed, part, torch.empty(len(rows), N, dtype=x.dtype, device="cuda")), whole[rows])
