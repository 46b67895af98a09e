"""The dense layer at the sizes where its tensor-core kernel works in pairs of blocks, and takes more than one tile a block.

On chips of 148 to 152 SMs the tiling rule gives 390 x 4880 (tokens x channels) pairs with 160 tokens a tile, 490 x 4880 pairs
with 192, 770 x 5540 and 970 x 5420 the same with a second tile for some pairs, and the last three single blocks of 32, 64 and
128 tokens with a second tile for some.  K = 300 is one exact stretch of sums, 2100 three."""
import numpy as np
import pytest

from oracle import tokens as ref
from test_gpu_linear_i8 import TYPES, _check_y, _f32, _weights, _x

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2208_01944_gb300 import binding
    yield binding
    assert binding.palquant_sync_check() == binding.PQ_OK


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("K", [300, 2100])
@pytest.mark.parametrize("M,N", [(390, 4880), (490, 4880), (770, 5540), (970, 5420), (20, 19460), (50, 19460), (200, 9740)])
def test_tiles(B, M, N, K, kind):
    x = _x(M, K, kind, M + K)
    w, s_w = _weights(N, K, N + K)
    pitch = -(-K // 16) * 16
    wbig = torch.full((N, pitch), 77, dtype=torch.int8, device="cuda")
    wd, sd = wbig[:, :K], torch.from_numpy(s_w).cuda()
    wd.copy_(torch.from_numpy(w))
    bias = np.random.default_rng(3).normal(size=N).astype(np.float32) if M % 4 else None
    bd = None if bias is None else torch.from_numpy(bias).cuda()
    q, s_x = ref.quantize_tokens(_f32(x))
    acc = q.astype(np.float64) @ w.astype(np.float64).T  # integers below 2^53: exact
    y = torch.full((M, N + 1), 7.0, dtype=TYPES[kind], device="cuda")
    d = B.linear_desc(x, wd, y[:, :N])
    assert B.palquant_linear_code_format(d) == B.PQ_CODES_F16
    scratch = torch.empty(B.palquant_linear_q8_scratch_bytes(d), dtype=torch.uint8, device="cuda")
    B.palquant_linear_q8(x, wd, sd, bd, y[:, :N], d, scratch, scratch.numel())
    _check_y(y[:, :N], acc, s_x, s_w, bias, kind)
    assert bool((y[:, N] == 7).all())
    codes, scales = torch.zeros((M, pitch), dtype=torch.float16, device="cuda"), torch.empty(M, device="cuda")
    B.palquant_quantize_tokens(x, d.x_type, d.ldx, M, K, B.PQ_CODES_F16, codes, pitch, scales)
    sums = torch.full((M, N), -9, dtype=torch.int32, device="cuda")
    B.palquant_linear_i8(codes, B.PQ_CODES_F16, pitch, scales, wd, sd, bd, sums, None, d)
    assert np.array_equal(sums.cpu().numpy(), acc.astype(np.int32))
