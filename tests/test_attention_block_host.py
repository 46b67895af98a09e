"""What the attention block refuses before it touches a GPU."""
import pytest

torch = pytest.importorskip("torch")
pytest.importorskip("paper_2208_01944_gb300.binding", reason="libpalquant.so not built")
from paper_2208_01944_gb300.attention_block import AttentionBlock8  # noqa: E402


@pytest.mark.parametrize("kw", [dict(b_qkv=torch.zeros(511)), dict(b_qkv=torch.zeros(513)), dict(b_qkv=torch.zeros(1)),
                                dict(page_tokens=48), dict(window=-1), dict(max_len=0),
                                dict(sequences=0), dict(heads=0), dict(kv_heads=0), dict(w_qkv=torch.zeros(512, 256).double()),
                                dict(w_qkv=torch.zeros(8 * 40, 256), w_out=torch.zeros(256, 4 * 40))],
                         ids=lambda kw: " ".join(f"{k}={getattr(v, 'shape', v)}" for k, v in kw.items()))
def test_arguments(kw):
    v = dict(w_qkv=torch.zeros(8 * 64, 256), w_out=torch.zeros(256, 4 * 64), heads=4, kv_heads=2, sequences=2, max_len=100)
    with pytest.raises(ValueError):
        AttentionBlock8(**(v | kw))
