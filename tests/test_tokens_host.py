"""What the 8-bit transformer calls refuse before anything is launched, and the oracle's
own statements of them (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import tokens as ref

B = pytest.importorskip("paper_2208_01944_gb300.binding", reason="libpalquant.so not built")


def _refused(call, *args, status=None):
    with pytest.raises(B.PalquantError) as e:
        call(*args, stream=0)
    assert e.value.status == (B.PQ_EINVAL if status is None else status)


def _linear(**kw):
    v = dict(M=4, N=32, K=64, x_type=0, y_type=0, ldx=64, ldw=64, ldy=32)
    v.update(kw)
    return B.LinearDesc(*[v[n] for n, _ in B.LinearDesc._fields_])


@pytest.mark.parametrize("kw", [dict(M=-1), dict(N=0), dict(K=0), dict(K=131073, ldx=131073, ldw=131073), dict(x_type=3),
                                dict(y_type=-1), dict(ldx=63), dict(ldw=63), dict(ldy=31)], ids=str)
def test_linear_descriptors_refused(kw):
    d = _linear(**kw)
    assert B.palquant_linear_q8_scratch_bytes(d) == 0
    _refused(B.palquant_linear_q8, 64, 64, 64, None, 64, d, 64, 1 << 30)
    if "x_type" not in kw and "ldx" not in kw:
        _refused(B.palquant_linear_i8, 64, 0, 131073, 64, 64, 64, None, None, 64, d)


@pytest.mark.parametrize("M,ldw,code,copy", [(1, 4096, 0, 0), (16, 4095, 0, 0), (17, 4096, 5, 0), (17, 4095, 0, 4000 * 4096),
                                             (600, 4095, 0, 4000 * 4096), (600, 4112, 5, 0)])
def test_linear_code_format_and_scratch(M, ldw, code, copy):
    d = _linear(M=M, N=4000, K=4095, ldx=4095, ldw=ldw, ldy=4000)
    assert B.palquant_linear_code_format(d) == code
    each = 2 if code == B.PQ_CODES_F16 or copy else 1
    need = B.palquant_linear_q8_scratch_bytes(d)
    assert M * 4096 * each + 4 * M + copy <= need <= M * 4096 * each + 4 * M + copy + 16


def test_linear_arguments_refused():
    d = _linear()
    need = B.palquant_linear_q8_scratch_bytes(d)
    assert need >= 4 * 64 + 4 * 4
    ok = [64, 64, 64, None, 64, d, 64, need]
    for i, bad in ((0, None), (1, None), (2, None), (4, None), (6, None), (0, 66), (2, 66), (3, 65), (4, 66), (6, 72), (7, need - 1)):
        args = list(ok)
        args[i] = bad
        _refused(B.palquant_linear_q8, *args)
    ok = [64, B.PQ_CODES_INT8, 64, 64, 64, 64, None, None, 64, d]
    for i, bad in ((0, None), (1, B.PQ_CODES_C16), (2, 63), (3, None), (4, None), (5, None), (8, None), (8, 66), (7, 66)):
        args = list(ok)
        args[i] = bad
        _refused(B.palquant_linear_i8, *args)
    ok = [64, B.PQ_F32, 64, 4, 64, B.PQ_CODES_INT8, 64, 64, 64]
    for i, bad in ((0, None), (0, 66), (1, 3), (2, 63), (3, -1), (4, 0), (5, B.PQ_CODES_C16), (6, None), (7, 63), (8, None), (8, 66)):
        args = list(ok)
        args[i] = bad
        _refused(B.palquant_quantize_tokens, *args)


def test_nothing_to_do_is_no_error():
    d = _linear(M=0)
    B.palquant_linear_q8(None, None, None, None, None, d, None, 0, stream=0)
    B.palquant_quantize_tokens(None, B.PQ_F32, 64, 0, 64, B.PQ_CODES_INT8, None, 64, None, stream=0)
    c = _cache()
    B.palquant_kv8_append(c, None, None, _tokens(B=0), stream=0)
    B.palquant_kv8_read(c, None, None, _tokens(max_n=0), stream=0)
    B.palquant_kv8_attention(c, None, None, _attn(B=0), None, 0, stream=0)
    B.palquant_kv8_attention(c, None, None, _attn(max_q=0), None, 0, stream=0)


def _cache(**kw):
    v = dict(num_pages=4, page_tokens=16, Hkv=2, D=64, k_dev=64, v_dev=64, k_scale_dev=64, v_scale_dev=64)
    v.update(kw)
    return B.KV8Cache(*[v[n] for n, _ in B.KV8Cache._fields_])


def _tokens(**kw):
    v = dict(type=0, B=2, max_n=3, table_pitch=2, k_token_stride=128, k_head_stride=64, v_token_stride=128, v_head_stride=64,
             cu_dev=64, start_dev=64, page_table_dev=64)
    v.update(kw)
    return B.KV8Tokens(*[v[n] for n, _ in B.KV8Tokens._fields_])


def _attn(**kw):
    v = dict(type=1, B=2, Hq=4, max_q=1, max_len=32, causal=1, window=0, table_pitch=2, scale=0.1, q_token_stride=256,
             q_head_stride=64, o_token_stride=256, o_head_stride=64, cu_q_dev=64, len_dev=64, page_table_dev=64)
    v.update(kw)
    return B.KV8Attn(*[v[n] for n, _ in B.KV8Attn._fields_])


BAD_CACHES = [dict(num_pages=0), dict(page_tokens=48), dict(page_tokens=8), dict(Hkv=0), dict(D=8), dict(D=72), dict(D=272),
              dict(k_dev=None), dict(v_dev=72), dict(k_scale_dev=66), dict(v_scale_dev=None)]


@pytest.mark.parametrize("kw", BAD_CACHES, ids=str)
def test_caches_refused(kw):
    c = _cache(**kw)
    _refused(B.palquant_kv8_append, c, 64, 64, _tokens())
    _refused(B.palquant_kv8_read, c, 64, 64, _tokens())
    _refused(B.palquant_kv8_attention, c, 64, 64, _attn(), 64, 1 << 30)
    assert B.palquant_kv8_attention_scratch_bytes(c, _attn()) == 0


@pytest.mark.parametrize("kw", [dict(type=3), dict(B=-1), dict(max_n=-1), dict(table_pitch=-1), dict(cu_dev=None),
                                dict(start_dev=66), dict(page_table_dev=None), dict(k_token_stride=-1), dict(v_head_stride=-64)],
                         ids=str)
def test_token_runs_refused(kw):
    _refused(B.palquant_kv8_append, _cache(), 64, 64, _tokens(**kw))
    _refused(B.palquant_kv8_read, _cache(), 64, 64, _tokens(**kw))


def test_missing_tensors_refused():
    _refused(B.palquant_kv8_append, _cache(), None, 64, _tokens())
    _refused(B.palquant_kv8_append, _cache(), 64, 66, _tokens())
    _refused(B.palquant_kv8_read, _cache(), None, None, _tokens())
    _refused(B.palquant_kv8_attention, _cache(), None, 64, _attn(), None, 0)
    _refused(B.palquant_kv8_attention, _cache(), 64, 65, _attn(), None, 0)
    big = _attn(max_len=100000)
    need = B.palquant_kv8_attention_scratch_bytes(_cache(), big)
    assert need > 0
    _refused(B.palquant_kv8_attention, _cache(), 64, 64, big, 64, need - 1)
    _refused(B.palquant_kv8_attention, _cache(), 64, 64, big, None, need)
    _refused(B.palquant_kv8_attention, _cache(), 64, 64, big, 72, need)


@pytest.mark.parametrize("kw", [dict(type=-1), dict(B=-1), dict(Hq=3), dict(Hq=0), dict(Hq=130), dict(max_q=-1), dict(max_len=-1),
                                dict(causal=2), dict(causal=0, window=5), dict(window=-1), dict(table_pitch=-1),
                                dict(scale=float("nan")), dict(q_token_stride=-1), dict(o_head_stride=-1), dict(cu_q_dev=None),
                                dict(len_dev=66), dict(page_table_dev=None)], ids=str)
def test_attention_refused(kw):
    _refused(B.palquant_kv8_attention, _cache(), 64, 64, _attn(**kw), 64, 1 << 30)


def test_descriptor_builders_check_their_tensors():
    x, w, y = torch.zeros(3, 8), torch.zeros(5, 8, dtype=torch.int8), torch.zeros(3, 5)
    d = B.linear_desc(x, w, y)
    assert (d.M, d.N, d.K, d.ldx, d.ldw, d.ldy, d.x_type) == (3, 5, 8, 8, 8, 5, B.PQ_F32)
    for bad in ((x, w.float(), y), (x, w, y.t()), (x[:, ::2], w[:, :4], y), (x, w[:, :7], y)):
        with pytest.raises(AssertionError):
            B.linear_desc(*bad)
    with pytest.raises(TypeError):
        B.linear_desc(x.double(), w, y)
    codes, scales = torch.zeros(4, 2, 16, 64, dtype=torch.int8), torch.zeros(4, 2)
    c = B.kv8_cache(codes, codes, scales, scales)
    assert (c.num_pages, c.page_tokens, c.Hkv, c.D) == (4, 16, 2, 64)
    with pytest.raises(AssertionError):
        B.kv8_cache(codes, codes[:3], scales, scales)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(AssertionError):
        B.kv8_tokens(torch.zeros(3, 2, 64), torch.zeros(3, 2, 64), i32(3), i32(3), i32(3, 2), 1)
    with pytest.raises(AssertionError):
        B.kv8_attn(torch.zeros(3, 4, 64), torch.zeros(3, 4, 64), i32(3).long(), i32(2), i32(2, 2), 1, 1, 0.1)
    assert ctypes.sizeof(B.LinearDesc) == 48


def test_oracle_scales_and_codes():
    x = np.array([[127.0, 1.0, -64.5], [0, 0, 0], [np.nan, 1, 2], [1, np.inf, 2], [2.0 ** -121, 0, 0]], np.float32)
    q, s = ref.quantize_tokens(x)
    assert list(q[0]) == [127, 1, -64] or list(q[0]) == [127, 1, -65]
    assert s[1] == 0 and np.isnan(s[2]) and np.isnan(s[3]) and s[4] == 0
    assert not q[1:].any()
    big = np.array([[3e38, -3e38, 1e38]], np.float32)
    q, s = ref.quantize_tokens(big)
    assert np.isfinite(s[0]) and list(q[0][:2]) == [127, -127]


def test_oracle_attention_matches_a_direct_softmax():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(5, 4, 8)), rng.normal(size=(9, 2, 8)), rng.normal(size=(9, 2, 8))
    o, spread, _ = ref.attention(q, k, v, 0.5, True, 4)
    for i in range(5):
        for h in range(4):
            lo, hi = max(0, 4 + i - 3), 5 + i
            s = 0.5 * k[lo:hi, h // 2] @ q[i, h]
            p = np.exp(s) / np.exp(s).sum()
            assert np.allclose(o[i, h], p @ v[lo:hi, h // 2]) and np.allclose(spread[i, h], p @ np.abs(v[lo:hi, h // 2]))
    o, _, _ = ref.attention(q, k[:2], v[:2], 0.5, True, 0)
    assert not o[:3].any() and o[3:].any()
