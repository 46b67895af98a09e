"""What the descriptor builders and calls of the 8-bit transformer layers refuse, before the library sees a pointer (no GPU)."""
import pytest
import torch

B = pytest.importorskip("paper_2208_01944_gb300.binding", reason="libpalquant.so not built")


def test_rows_that_overlap_are_refused():
    """A pitch below the row's length would otherwise be read as the row's length, past the end of what is there."""
    x, w, y = torch.zeros(4, 8), torch.zeros(5, 8, dtype=torch.int8), torch.zeros(4, 5)
    B.linear_desc(x, w, y)
    flat, codes, out = torch.zeros(64), torch.zeros(64, dtype=torch.int8), torch.zeros(64)
    for bad in ((x[:1].expand(4, 8), w, y), (flat.as_strided((4, 8), (3, 1)), w, y), (x, w[:1].expand(5, 8), y),
                (x, codes.as_strided((5, 8), (7, 1)), y), (x, w, y[:1].expand(4, 5)), (x, w, out.as_strided((4, 5), (4, 1)))):
        with pytest.raises(ValueError):
            B.linear_desc(*bad)
    d = B.linear_desc(x[:1].expand(1, 8), w, y[:1])  # the pitch of one row does not count
    assert (d.M, d.ldx, d.ldy) == (1, 8, 5)
    wide = torch.zeros(4, 11)
    assert B.linear_desc(wide[:, 2:10], w, y).ldx == 11


def _i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def _cache(H=2, D=64, pages=4, T=16):
    codes, scales = torch.zeros(pages, H, T, D, dtype=torch.int8), torch.zeros(pages, H)
    return B.kv8_cache(codes, codes.clone(), scales, scales.clone())


def _runs(k, v):
    return B.kv8_tokens(k, v, _i32(3), _i32(2), _i32(2, 2), 0)  # max_n = 0: a call that passes does nothing


def _queries(q, o):
    return B.kv8_attn(q, o, _i32(3), _i32(2), _i32(2, 2), 0, 32, 0.1)  # max_q = 0: the same


def test_runs_are_held_against_each_other_and_the_cache():
    k = torch.zeros(6, 2, 64)
    t = _runs(k, k.clone())
    B.palquant_kv8_append(_cache(), k, k, t, stream=0)
    B.palquant_kv8_read(_cache(), k, k, t, stream=0)
    B.palquant_kv8_read(_cache(), None, k, t, stream=0)
    for other in (torch.zeros(5, 2, 64), torch.zeros(6, 1, 64), torch.zeros(6, 2, 48), k.half()):
        with pytest.raises(ValueError):  # v unlike k
            _runs(k, other)
        with pytest.raises(ValueError):  # tensors unlike the descriptor's
            B.palquant_kv8_append(_cache(), k, other, t, stream=0)
        with pytest.raises(ValueError):
            B.palquant_kv8_read(_cache(), other, None, t, stream=0)
    sliced = torch.zeros(6, 4, 64)[:, :2]
    with pytest.raises(ValueError):  # strides unlike the descriptor's
        B.palquant_kv8_append(_cache(), sliced, k, t, stream=0)
    one = _runs(k[:1], k[:1])
    B.palquant_kv8_append(_cache(), sliced[:1], k[:1], one, stream=0)  # (the pitch of one row does not count)
    only_k = _runs(k, None)
    B.palquant_kv8_read(_cache(), k, None, only_k, stream=0)
    with pytest.raises(ValueError):
        B.palquant_kv8_read(_cache(), k, k, only_k, stream=0)
    for cache in (_cache(H=1), _cache(H=4), _cache(D=128)):
        for call in (B.palquant_kv8_append, B.palquant_kv8_read):
            with pytest.raises(ValueError):
                call(cache, k, k, t, stream=0)
    everywhere = torch.zeros(1, 2, 64).expand(6, 2, 64)  # one token, six times: may be appended, not read into
    B.palquant_kv8_append(_cache(), everywhere, everywhere, _runs(everywhere, everywhere), stream=0)
    with pytest.raises(ValueError):
        B.palquant_kv8_read(_cache(), everywhere, everywhere, _runs(everywhere, everywhere), stream=0)


def test_queries_are_held_against_the_cache():
    q, o = torch.zeros(6, 4, 64), torch.zeros(6, 4, 64)
    a = _queries(q, o)
    B.palquant_kv8_attention(_cache(), q, o, a, None, 0, stream=0)
    with pytest.raises(ValueError):
        B.palquant_kv8_attention(_cache(D=48), q, o, a, None, 0, stream=0)
    with pytest.raises(B.PalquantError):  # 4 query heads on 3 cache heads
        B.palquant_kv8_attention(_cache(H=3), q, o, a, None, 0, stream=0)
    for bad in (torch.zeros(6, 4, 48), torch.zeros(6, 3, 64), torch.zeros(5, 4, 64), q.half(), torch.zeros(4, 6, 64).transpose(0, 1)):
        with pytest.raises(ValueError):
            B.palquant_kv8_attention(_cache(), bad, o, a, None, 0, stream=0)
        with pytest.raises(ValueError):
            B.palquant_kv8_attention(_cache(), q, bad, a, None, 0, stream=0)
    with pytest.raises(ValueError):
        _queries(q, o[:1].expand(6, 4, 64))
    with pytest.raises(ValueError):
        _queries(q, o[:, :1].expand(6, 4, 64))
    shared = q[:, :1].expand(6, 4, 64)  # one query head for all: read only
    B.palquant_kv8_attention(_cache(), shared, o, _queries(shared, o), None, 0, stream=0)


@pytest.mark.parametrize("i", range(3))
def test_index_tensors_are_counted(i):
    k = torch.zeros(6, 2, 64)
    for change in (lambda t: t[:-1], lambda t: t.long(), lambda t: t.to("meta")):
        index = [_i32(3), _i32(2), _i32(2, 2)]
        index[i] = change(index[i])
        with pytest.raises(ValueError):
            B.kv8_tokens(k, k, *index, 1)
        with pytest.raises(ValueError):
            B.kv8_attn(k, k.clone(), *index, 1, 32, 0.1)


def test_scales_bias_and_codes_of_the_dense_layer_are_looked_at():
    """Tensors too short or of another type are refused before the library is called; what passes gets as far as its status."""
    x, w, y = torch.zeros(4, 64), torch.zeros(32, 64, dtype=torch.int8), torch.zeros(4, 32)
    s_w, bias, s_x = torch.zeros(32), torch.zeros(32), torch.zeros(4)
    d = B.linear_desc(x, w, y)
    with pytest.raises(ValueError):
        B.linear_desc(x, w, y.to("meta"))

    def q8(**kw):
        a = {"x": x, "w": w, "s_w": s_w, "bias": bias, "y": y} | kw
        B.palquant_linear_q8(*a.values(), d, None, 0, stream=0)

    def i8(**kw):
        a = {"q": w[:4], "format": B.PQ_CODES_INT8, "ldq": 64, "s_x": s_x, "w": w, "s_w": s_w, "bias": bias, "acc": None, "y": None} | kw
        B.palquant_linear_i8(*a.values(), d, stream=0)

    def tokens(**kw):
        a = {"x": x, "type": B.PQ_F32, "ldx": 64, "M": 4, "K": 64, "format": B.PQ_CODES_INT8, "q": w[:4], "ldq": 64, "s": s_x} | kw
        B.palquant_quantize_tokens(*a.values(), stream=0)

    for call in (q8, i8):  # (no scratch, no output)
        with pytest.raises(B.PalquantError):
            call()
    with pytest.raises(B.PalquantError):
        tokens(K=0)
    long = {"s_w": torch.zeros(40), "bias": torch.zeros(40)}  # longer than the layer is wide: taken
    with pytest.raises(B.PalquantError):
        q8(**long)
    for bad in ({"s_w": s_w[:31]}, {"s_w": s_w.half()}, {"bias": bias[:31]}, {"bias": bias.double()}, {"x": x[:3]}, {"x": x.half()},
                {"x": torch.zeros(64, 4).t()}, {"w": w[:31]}, {"w": torch.zeros(32, 80, dtype=torch.int8)[:, :64]}, {"y": y[:, :31]}):
        with pytest.raises(ValueError):
            q8(**bad)
    for bad in ({"q": w[:3]}, {"q": w[:4].half()}, {"format": B.PQ_CODES_F16}, {"ldq": 80}, {"s_x": s_x[:3]}, {"s_x": s_x.half()},
                {"w": w[:31]}, {"s_w": s_w[:31]}, {"bias": bias[:31]}, {"acc": torch.zeros(4, 31, dtype=torch.int32)},
                {"acc": torch.zeros(4, 32)}, {"y": y[:3]}):
        with pytest.raises(ValueError):
            i8(**bad)
    for bad in ({"x": x[:3]}, {"x": x.half()}, {"type": B.PQ_F16}, {"ldx": 65}, {"M": 5}, {"K": 65}, {"q": w[:3]}, {"q": x},
                {"format": B.PQ_CODES_F16}, {"ldq": 65}, {"s": s_x[:3]}, {"s": s_x.double()}):
        with pytest.raises(ValueError):
            tokens(**bad)
    padded = torch.zeros(4, 80)[:, :64]
    with pytest.raises(B.PalquantError):  # rows of a wider matrix: as far as its last element
        tokens(x=padded, ldx=80, format=7)
