"""What the decoder's calls around the 8-bit cache refuse before anything is launched, their sizes, and the oracle's statements of them
(no GPU)."""
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


# ------------------------------------------------------------------ sinks and trees
def _cache(**kw):
    v = dict(num_pages=10, page_tokens=64, Hkv=2, D=64, k_dev=64, v_dev=64, k_scale_dev=64, v_scale_dev=64)
    v.update(kw)
    return B.KV8Cache(*[v[n] for n, _ in B.KV8Cache._fields_])


def _attn(**kw):
    v = dict(type=1, B=2, Hq=8, max_q=4, max_len=3000, causal=1, window=1000, table_pitch=50, scale=0.1, q_token_stride=512,
             q_head_stride=64, o_token_stride=512, o_head_stride=64, cu_q_dev=64, len_dev=64, page_table_dev=64)
    v.update(kw)
    return B.KV8Attn(*[v[n] for n, _ in B.KV8Attn._fields_])


@pytest.mark.parametrize("kw,sinks", [({}, -1), (dict(causal=0, window=0), 4), (dict(window=-1), 4), (dict(Hq=7), 4), (dict(scale=float("nan")), 4)], ids=str)
def test_sinks_refused(kw, sinks):
    a = _attn(**kw)
    assert B.palquant_kv8_attention_sinks_scratch_bytes(_cache(), a, sinks) == 0
    _refused(B.palquant_kv8_attention_sinks, _cache(), 64, 64, a, sinks, 64, 1 << 30)


@pytest.mark.parametrize("kw,tree", [(dict(causal=0), {}), (dict(window=5), {}), ({}, dict(words=0)), ({}, dict(pitch=0)), (dict(max_q=33), {}),
                                     ({}, dict(bits_dev=None)), ({}, dict(bits_dev=66)), (dict(max_q=0x7FFFFFFF), dict(words=0x3FFFFFF, pitch=1 << 40))], ids=str)
def test_trees_refused(kw, tree):
    a = _attn(**{"window": 0, **kw})
    t = B.KV8Tree(**{"bits_dev": 64, "pitch": 1, "words": 1, **tree})
    _refused(B.palquant_kv8_attention_tree, _cache(), 64, 64, a, t, 64, 1 << 30)
    if "bits_dev" not in tree:
        assert B.palquant_kv8_attention_tree_scratch_bytes(_cache(), a, t) == 0


def test_no_tree_is_refused():
    args = (ctypes.byref(_cache()), 64, 64, ctypes.byref(_attn(window=0)), None, 64, 1 << 30, 0)
    assert B.lib.palquant_kv8_attention_tree(*args) == B.PQ_EINVAL


def test_views_check_their_scratch_and_pointers():
    t = B.KV8Tree(64, 1, 1)
    for call, size, a, extra in ((B.palquant_kv8_attention_sinks, B.palquant_kv8_attention_sinks_scratch_bytes, _attn(max_len=90000, window=30000), 4),
                                 (B.palquant_kv8_attention_tree, B.palquant_kv8_attention_tree_scratch_bytes, _attn(max_len=90000, window=0), t)):
        need = size(_cache(), a, extra)
        assert need > 0
        for q, o, scratch, n in ((None, 64, 64, need), (64, None, 64, need), (65, 64, 64, need), (64, 64, None, need), (64, 64, 72, need), (64, 64, 64, need - 1)):
            _refused(call, _cache(), q, o, a, extra, scratch, n)
        big = _attn(window=a.window, max_len=(1 << 30) + 1)
        assert size(_cache(), big, extra) == 0
        _refused(call, _cache(), 64, 64, big, extra, 64, 1 << 40, status=B.PQ_EUNSUPPORTED)
        nothing = _attn(window=a.window, B=0)
        assert size(_cache(), nothing, extra) == 0
        call(_cache(), None, None, nothing, extra, None, 0, stream=0)


@pytest.mark.parametrize("max_q", [1, 30])
def test_sinks_cut_the_visible_tokens_alone(max_q):
    """The scratch follows the window and the sinks, not the text; sinks without a window are plain attention."""
    small = B.palquant_kv8_attention_sinks_scratch_bytes(_cache(), _attn(max_q=max_q, max_len=100000, window=30000), 4)
    assert small == B.palquant_kv8_attention_sinks_scratch_bytes(_cache(), _attn(max_q=max_q, max_len=900000, window=30000), 4) > 0
    # a few rows over a few thousand tokens, or over a few hundred, are joined without it
    assert B.palquant_kv8_attention_sinks_scratch_bytes(_cache(), _attn(max_q=1, max_len=100000), 4) == 0
    assert B.palquant_kv8_attention_sinks_scratch_bytes(_cache(), _attn(max_q=1, max_len=100000, window=200), 4) == 0
    assert B.palquant_kv8_attention_sinks_scratch_bytes(_cache(), _attn(max_q=max_q, max_len=100000), 0x7FFFFFFF) == \
        B.palquant_kv8_attention_scratch_bytes(_cache(), _attn(max_q=max_q, max_len=100000, window=0))
    for a, sinks in ((_attn(window=0), 4), (_attn(window=3000), 4), (_attn(), 0)):
        plain = _attn(window=0 if a.window >= 3000 else a.window)
        assert B.palquant_kv8_attention_sinks_scratch_bytes(_cache(), a, sinks) == B.palquant_kv8_attention_scratch_bytes(_cache(), plain)


def _i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def test_tree_bits_are_held_against_the_queries():
    q = torch.zeros(6, 2, 64)
    a = B.kv8_attn(q, q.clone(), _i32(3), _i32(2), _i32(2, 2), 4, 32, 0.1)
    t = B.kv8_tree(_i32(6, 9)[:, :2], a)
    assert (t.pitch, t.words) == (9, 2)
    for bad in (_i32(5, 1), _i32(6, 1).long(), _i32(6), _i32(1, 1).expand(6, 1), _i32(6, 4)[:, ::2]):
        with pytest.raises(ValueError):
            B.kv8_tree(bad, a)
    other = B.kv8_attn(q[:5], q[:5].clone(), _i32(3), _i32(2), _i32(2, 2), 4, 32, 0.1)
    codes, scales = torch.zeros(4, 1, 16, 64, dtype=torch.int8), torch.zeros(4, 1)
    cache = B.kv8_cache(codes, codes.clone(), scales, scales.clone())
    with pytest.raises(ValueError):
        B.palquant_kv8_attention_tree(cache, 64, 64, other, t, None, 0, stream=0)


def test_tensors_off_the_current_device_are_refused():
    q = torch.zeros(6, 2, 64)
    a = B.kv8_attn(q, q.clone(), _i32(3), _i32(2), _i32(2, 2), 4, 32, 0.1)
    codes, scales = torch.zeros(4, 1, 16, 64, dtype=torch.int8), torch.zeros(4, 1)
    cache = B.kv8_cache(codes, codes.clone(), scales, scales.clone())
    with pytest.raises(ValueError):
        B.palquant_kv8_attention_sinks(cache, q, q, a, 4, None, 0, stream=0)
    with pytest.raises(ValueError):
        B.palquant_kv8_attention_tree(cache, q, q, a, B.kv8_tree(_i32(6, 1), a), None, 0, stream=0)
    with pytest.raises(ValueError):
        B.palquant_qk_norm_rope(q, None, q, None, B.qk_norm_rope(q, None, q, None), stream=0)
    w = B.w4_weights(16, 64, 32, torch.float16)
    with pytest.raises(ValueError):
        B.palquant_w4_quantize(torch.zeros(16, 64), B.PQ_F32, 64, w, torch.zeros(1 << 14, dtype=torch.uint8), 1 << 14, stream=0)


# ------------------------------------------------------------------ norm and rotation
def _rope(**kw):
    v = dict(type=2, w_type=2, tokens=5, Hq=4, Hkv=2, D=64, R=64, interleaved=0, norm=1, eps=1e-6, pos_dev=64, turns_dev=64, q_weight_dev=64,
             k_weight_dev=64)
    v.update({n: 512 if "token" in n else 64 for n, _ in B.QKRope._fields_ if n.endswith("stride")})
    v.update(kw)
    return B.QKRope(*[v[n] for n, _ in B.QKRope._fields_])


@pytest.mark.parametrize("kw", [dict(type=3), dict(w_type=-1), dict(tokens=-1), dict(Hq=-1), dict(Hq=0, Hkv=0), dict(D=0), dict(R=-2), dict(R=66), dict(R=63),
                                dict(interleaved=2), dict(norm=2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(q_token_stride=-1),
                                dict(k_out_head_stride=-1), dict(pos_dev=None), dict(turns_dev=None), dict(turns_dev=68), dict(pos_dev=66),
                                dict(q_weight_dev=65), dict(k_weight_dev=65)], ids=str)
def test_rope_descriptors_refused(kw):
    _refused(B.palquant_qk_norm_rope, 64, 64, 64, 64, _rope(**kw))


def test_rope_arguments_refused():
    for i in range(4):
        for bad in (None, 65):
            args = [64] * 4
            args[i] = bad
            _refused(B.palquant_qk_norm_rope, *args, _rope())
    for kw in (dict(D=1025), dict(tokens=1 << 31), dict(Hq=65535)):
        _refused(B.palquant_qk_norm_rope, 64, 64, 64, 64, _rope(**kw), status=B.PQ_EUNSUPPORTED)
    B.palquant_qk_norm_rope(None, None, None, None, _rope(tokens=0), stream=0)


def test_rope_tensors_are_held_against_each_other():
    q, k = torch.zeros(6, 4, 64), torch.zeros(6, 2, 64)
    turns, pos = B.rope_turns([1.0, 0.5], "cpu"), _i32(6)
    d = B.qk_norm_rope(q, k, q, k, pos, turns, torch.ones(64), torch.ones(64))
    assert (d.tokens, d.Hq, d.Hkv, d.D, d.R, d.norm) == (6, 4, 2, 64, 4, 1)
    ok = dict(q=q, k=k, q_out=q, k_out=k, positions=pos, turns=turns)
    one_row = torch.zeros(64)
    for bad in (dict(q=None, k=None, q_out=None, k_out=None), dict(k_out=None), dict(k=None), dict(k=k[:5], k_out=k[:5]), dict(k=k.half(), k_out=k.half()),
                dict(k=k[:, :, :32], k_out=k[:, :, :32]), dict(q_out=q.half()), dict(q_out=q[:, :2]), dict(q_out=one_row.expand(6, 4, 64)),
                dict(q_out=q.view(4, 6, 64).transpose(0, 1)),  # the input's place with other strides
                dict(positions=pos[:5]), dict(positions=pos.long()), dict(positions=None), dict(turns=turns.int()), dict(turns=B.rope_turns([0.1] * 33, "cpu")),
                dict(q_weight=torch.ones(63)), dict(q_weight=torch.ones(64), k_weight=torch.ones(64).half()), dict(q_weight=torch.ones(64), norm=False),
                dict(q=q.transpose(1, 2), q_out=q.transpose(1, 2))):
        with pytest.raises((ValueError, TypeError)):
            B.qk_norm_rope(**{**ok, **bad})
    assert B.qk_norm_rope(**{**ok, "positions": None, "turns": None}).R == 0


def test_rope_turns():
    from fractions import Fraction

    pi = Fraction(31415926535897932384626433832795028841971693993751058209749445923078164062862090, 10 ** 79)
    f = [1.0, 0.5, 1e-9, 6.283185307179586, -0.25, 123456.789, 0.0, -1e-30, 3.3e-5]
    got = B.rope_turns(f, "cpu").numpy().view(np.uint64)
    for x, t in zip(f, got.tolist()):
        off = (Fraction(t, 1 << 64) - Fraction(x) / (2 * pi)) % 1
        assert min(off, 1 - off) <= Fraction(1, 1 << 62) + abs(Fraction(x)) / (1 << 100)
    for bad in ([float("nan")], [float("inf")]):
        with pytest.raises(B.PalquantError):
            B.rope_turns(bad, "cpu")
    assert B.rope_turns([], "cpu").numel() == 0


# ------------------------------------------------------------------ 4-bit weights
@pytest.mark.parametrize("N,K,group,dtype,expect", [(16, 128, 128, torch.float16, 1024 + 32), (17, 129, 32, torch.float32, 4 * (1024 + 256)),
                                                    (1, 1, 64, torch.bfloat16, 1024 + 64), (4096, 4096, 128, torch.float16, 256 * 32 * 1056)])
def test_packed_bytes(N, K, group, dtype, expect):
    assert B.palquant_w4_packed_bytes(B.w4_weights(N, K, group, dtype)) == expect


def _w(**kw):
    v = dict(N=32, K=64, group=32, s_type=1)
    v.update(kw)
    return B.W4Weights(*[v[n] for n, _ in B.W4Weights._fields_])


def _linear(**kw):
    v = dict(M=4, N=32, K=64, x_type=0, y_type=0, ldx=64, ldw=0, ldy=32)
    v.update(kw)
    return B.LinearDesc(*[v[n] for n, _ in B.LinearDesc._fields_])


@pytest.mark.parametrize("kw", [dict(N=0), dict(N=0x7FFFFFFF), dict(K=0), dict(K=131073), dict(group=16), dict(group=48), dict(group=0), dict(group=256), dict(s_type=3)], ids=str)
def test_w4_descriptors_refused(kw):
    w = _w(**kw)
    d = _linear(N=w.N, K=w.K, ldx=1 << 20, ldy=1 << 40)
    assert B.palquant_w4_packed_bytes(w) == 0 and B.palquant_linear_w4_scratch_bytes(w, d) == 0
    _refused(B.palquant_w4_pack, 64, 64, w, 64, 1 << 40)
    _refused(B.palquant_w4_quantize, 64, 0, 1 << 20, w, 64, 1 << 40)
    _refused(B.palquant_w4_unpack, 64, w, 64, 64)
    _refused(B.palquant_linear_w4, 64, 64, None, 64, w, d, 64, 1 << 30)


@pytest.mark.parametrize("kw", [dict(M=-1), dict(N=31), dict(K=65), dict(x_type=3), dict(y_type=-1), dict(ldx=63), dict(ldy=31)], ids=str)
def test_w4_calls_refused(kw):
    d = _linear(**kw)
    assert B.palquant_linear_w4_scratch_bytes(_w(), d) == 0
    _refused(B.palquant_linear_w4, 64, 64, None, 64, _w(), d, 64, 1 << 30)


def test_w4_arguments_refused():
    w, d = _w(), _linear()
    need = B.palquant_w4_packed_bytes(w)
    for call, ok, bads in (
            (B.palquant_w4_pack, [64, 64, w, 64, need], ((0, None), (1, None), (1, 65), (3, None), (3, 72), (4, need - 1))),
            (B.palquant_w4_quantize, [64, 0, 64, w, 64, need], ((0, None), (0, 66), (1, 3), (2, 63), (4, None), (4, 72), (5, need - 1))),
            (B.palquant_w4_unpack, [64, w, 64, 64], ((0, None), (0, 72), (3, 66))),
            (B.palquant_linear_w4, [64, 64, None, 64, w, d, 64, 1 << 30], ((0, None), (0, 66), (1, None), (1, 72), (2, 66), (3, None), (3, 66)))):
        for i, bad in bads:
            args = list(ok)
            args[i] = bad
            _refused(call, *args)
    _refused(B.palquant_w4_unpack, 64, w, None, None)
    _refused(B.palquant_linear_w4, 64, 64, None, 64, w, _linear(M=32 * 65535 + 1), 64, 1 << 60, status=B.PQ_EUNSUPPORTED)
    B.palquant_linear_w4(None, None, None, None, w, _linear(M=0), None, 0, stream=0)


def test_w4_outputs_over_the_tokens_are_refused():
    """Where it is refused for nothing else: large scratch, aligned addresses."""
    w = _w(N=64)
    at = 1 << 20
    for y, kw in ((at, {}),                                            # in place
                  (at + 64, dict(M=1)), (at - 128, dict(M=1)),         # one row, over a part of it
                  (at + 256, dict(ldx=128, ldy=96)),                   # rows of different pitch, one between the others
                  (at + 128, dict(ldx=96, ldy=96)),                    # columns that reach into the other's
                  (at + 768 + 576, dict(ldx=192, ldy=192))):           # and so from a row's end into the next one's
        _refused(B.palquant_linear_w4, at, 64, None, y, w, _linear(**{**dict(N=64, ldy=64), **kw}), 64, 1 << 30)


def test_w4_tensors_are_held_against_the_descriptor():
    w = B.w4_weights(32, 64, 32, torch.float16)
    x, y = torch.zeros(4, 64), torch.zeros(4, 32)
    d = B.linear_w4_desc(x, w, y)
    assert (d.M, d.N, d.K, d.ldx, d.ldy) == (4, 32, 64, 64, 32)
    for bx, by in ((x[:, :63], y), (x, y[:, :31]), (x[:3], y), (x[:1].expand(4, 64), y), (x, y[:1].expand(4, 32)), (x.double(), y), (x.t(), y)):
        with pytest.raises((ValueError, TypeError)):
            B.linear_w4_desc(bx, w, by)
    with pytest.raises(ValueError):
        B.w4_weights(32, 64, 32, torch.int8)


# ------------------------------------------------------------------ the oracle
def test_what_queries_see():
    assert ref.sees_sinks(2, 6, 2, 1).astype(int).tolist() == [[1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]
    assert ref.sees_sinks(1, 3, 0, 0).all()
    assert ref.sees_tree(3, 4, np.array([[1], [3], [5]], np.uint32)).astype(int).tolist() == [[1, 1, 0, 0], [1, 1, 1, 0], [1, 1, 0, 1]]


def test_rotation_turns_by_its_angle_and_keeps_lengths():
    x = np.array([[[3.0, 0.0, 0.0, 4.0]]])
    y, _ = ref.norm_rope(x, None, 0.0, [2], [np.pi / 4, np.pi / 2], False, norm=False)
    assert np.allclose(y[0, 0], [0, 0, 3, -4], atol=1e-12)  # a quarter turn of (3, 0), half a turn of (0, 4)
    y, _ = ref.norm_rope(x, None, 0.0, [2], [np.pi / 4, np.pi / 2], True, norm=False)
    assert np.allclose(y[0, 0], [0, 3, 0, -4], atol=1e-12)
    y, _ = ref.norm_rope(x, np.full(4, 2.0), 0.0, [7], [0.3, 0.1], False)
    assert np.isclose((y ** 2).sum(), 16)  # 4 elements of mean square 1, twice


def test_w4_quantizer_by_hand():
    codes, s = ref.w4_quantize(np.array([[7.0, -3.5, 0.5, 1.49, 0, 0, 14, -13]]), 4)
    assert np.allclose(s, [[1.0, 2.0]])
    assert codes.tolist() == [[7, -4, 0, 1, 0, 0, 7, -6]]


# ------------------------------------------------------------------ the attention block
def test_block_options_refused():
    from paper_2208_01944_gb300.attention_block import AttentionBlock8

    v = dict(w_qkv=torch.zeros(8 * 64, 256), w_out=torch.zeros(256, 4 * 64), heads=4, kv_heads=2, sequences=2, max_len=100)
    one = torch.ones(64)
    for kw in (dict(sinks=-1, window=5), dict(sinks=4), dict(weight_bits=2), dict(weight_bits=4, weight_group=16), dict(rope=[1.0] * 33), dict(rope=[float("nan")]),
               dict(q_norm=one), dict(k_norm=one), dict(q_norm=one, k_norm=one.half()), dict(q_norm=one[:63], k_norm=one[:63]),
               dict(q_norm=one, k_norm=one, norm_eps=-1.0), dict(q_norm=one.double(), k_norm=one.double())):
        with pytest.raises(ValueError):
            AttentionBlock8(**(v | kw))


def test_bits_of_trees():
    from paper_2208_01944_gb300.attention_block import tree_bits

    assert tree_bits([[-1, 0, 0, 2], [], [-1, -1]]).tolist() == [[1], [3], [5], [13], [1], [2]]
    chain = tree_bits([list(range(-1, 40))])
    assert chain.shape == (41, 2) and chain[31].tolist() == [-1, 0] and chain[40].tolist() == [-1, 511]
    assert tree_bits([]).shape == (0, 1)
    for bad in ([[0]], [[-1, 1]], [[-2]]):
        with pytest.raises(ValueError):
            tree_bits(bad)


def test_weights_to_4_bits_refused():
    from paper_2208_01944_gb300.attention_block import weight_codes4

    for w, group in ((torch.zeros(4), 128), (torch.zeros(4, 8).double(), 128), (torch.zeros(4, 8).t(), 128), (torch.zeros(4, 8), 16)):
        with pytest.raises(ValueError):
            weight_codes4(w, group)


@pytest.mark.parametrize("M,K,ldx,x_type,nbytes", [(8, 4096, 4096, 0, 0), (9, 4095, 4095, 0, 9 * 4096 * 6), (9, 700, 700, 0, 0), (16, 4095, 4095, 1, 0),
                                                   (17, 4095, 4095, 1, 17 * 4096 * 2), (17, 4095, 4096, 2, 0), (64, 8000, 8001, 2, 64 * 8000 * 2)])
def test_w4_scratch_is_a_copy_of_the_tokens_that_need_one(M, K, ldx, x_type, nbytes):
    w, d = _w(N=1000, K=K), _linear(M=M, N=1000, K=K, ldx=ldx, ldy=1000, x_type=x_type)
    assert B.palquant_linear_w4_scratch_bytes(w, d) == nbytes
    if nbytes:
        for scratch, n in ((None, nbytes), (72, nbytes), (64, nbytes - 1)):
            _refused(B.palquant_linear_w4, 64, 64, None, 64, w, d, scratch, n)


def test_rope_outputs_over_other_heads_are_refused():
    """Where it is refused for nothing else: aligned addresses, every stride above the heads' length.  (q: 4 heads, k: 2 heads, 5 tokens, bfloat16.)"""
    at, far = 1 << 20, 1 << 30
    for q, k, q_out, k_out, kw in (
            (at, far, at + 128, far, {}),                     # a head further
            (at, far, at + 1024, far, {}),                    # a token further
            (at, far, at - 2, far, {}),                       # an element before
            (at, far, at, far, dict(q_out_head_stride=128)),  # the input's place with other strides
            (at, far, at, far, dict(q_out_token_stride=640)),
            (at, far, far, 2 * far, {}),                      # queries over keys, keys over queries, outputs over one another
            (at, far, 2 * far, at + 128, {}),
            (at, far, 2 * far, 2 * far + 256, {}),
            (at, at + 512, at, at + 384, {})):                # in place, but for the keys, which lie in the queries' last head
        _refused(B.palquant_qk_norm_rope, q, k, q_out, k_out, _rope(**kw))
    _refused(B.palquant_qk_norm_rope, at, None, at + 128, None, _rope(Hkv=0))


def test_rope_views_over_one_another_are_refused():
    qkv = torch.zeros(6, 8, 64)
    d = B.qk_norm_rope(qkv[:, :4], None, qkv[:, 1:5], None)
    d._device = None  # (these tensors are on the CPU: as if they were where they should be)
    with pytest.raises(B.PalquantError) as e:
        B.palquant_qk_norm_rope(qkv[:, :4], None, qkv[:, 1:5], None, d, stream=0)
    assert e.value.status == B.PQ_EINVAL


def test_block_scales_refused():
    from paper_2208_01944_gb300.attention_block import AttentionBlock8

    for scales in (torch.int8, torch.float64, None):
        with pytest.raises(ValueError):
            AttentionBlock8(torch.zeros(8 * 64, 256), torch.zeros(256, 4 * 64), 4, 2, 2, 100, weight_bits=4, weight_scales=scales)
