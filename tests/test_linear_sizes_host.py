"""Sizes of the dense layer past 32 bits: refused with the status for it, and no scratch size is made from them (no GPU)."""
import pytest

B = pytest.importorskip("paper_2208_01944_gb300.binding", reason="libpalquant.so not built")


def _status(call, *args):
    with pytest.raises(B.PalquantError) as e:
        call(*args, stream=0)
    return e.value.status


@pytest.mark.parametrize("K", [0x7FFFFFF9, 0x7FFFFFFF])
def test_rows_whose_vectors_would_be_counted_past_32_bits(K):
    for fmt in (B.PQ_CODES_INT8, B.PQ_CODES_F16):
        assert _status(B.palquant_quantize_tokens, 64, B.PQ_F32, K, 1, K, fmt, 64, K, 64) == B.PQ_EUNSUPPORTED


@pytest.mark.parametrize("M", [1 << 31, 1 << 47, (1 << 63) - 1])
@pytest.mark.parametrize("ldw", [131072, 131073])
def test_tokens_past_32_bits(M, ldw):
    d = B.LinearDesc(M, 16, 131072, B.PQ_BF16, B.PQ_BF16, 131072, ldw, 16)
    assert B.palquant_linear_q8_scratch_bytes(d) == 0
    assert _status(B.palquant_linear_q8, 64, 64, 64, None, 64, d, 64, (1 << 64) - 1) == B.PQ_EUNSUPPORTED
