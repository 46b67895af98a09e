"""Weight rows read as aligned words up to their last bytes: rows of 16 j + 3 codes one after the other, so that the last
row starts on a word and ends three bytes into one."""
import numpy as np
import pytest

from oracle import tokens as ref
from test_gpu_linear_i8 import _check_y, _f32, _weights, _x

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2208_01944_gb300 import binding
    yield binding
    assert binding.palquant_sync_check() == binding.PQ_OK


@pytest.mark.parametrize("M", [1, 12, 40])
@pytest.mark.parametrize("N,K", [(41, 35), (41, 195), (33, 1027), (1021, 6595)])
def test_rows_that_end_inside_a_word(B, M, N, K):
    x = _x(M, K, "bf16", K)
    w, s_w = _weights(N, K, N)
    wd, sd = torch.from_numpy(w).cuda(), torch.from_numpy(s_w).cuda()
    y = torch.full((M, N), 7.0, device="cuda")
    d = B.linear_desc(x, wd, y)
    scratch = torch.empty(B.palquant_linear_q8_scratch_bytes(d), dtype=torch.uint8, device="cuda")
    B.palquant_linear_q8(x, wd, sd, None, y, d, scratch, scratch.numel())
    q, s_x = ref.quantize_tokens(_f32(x))
    _check_y(y, ref.linear(q, w), s_x, s_w, None, "f32")
    codes, scales = torch.empty((M, K), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    B.palquant_quantize_tokens(x, d.x_type, d.ldx, M, K, B.PQ_CODES_INT8, codes, K, scales)
    sums = torch.empty((M, N), dtype=torch.int32, device="cuda")
    B.palquant_linear_i8(codes, B.PQ_CODES_INT8, K, scales, wd, sd, None, sums, None, d)
    assert np.array_equal(sums.cpu().numpy(), ref.linear(q, w))
