"""Attention over the 8-bit cache through a window with sinks, and for trees of drafted tokens.

The bounds are those of the other attention tests: with u the output type's half step and spread = sum p |v|, u |o| for
the rounding, 2^-11 (fp32 2^-21) spread for probabilities as one or two halves, 2^-20 (2 + max |score|) spread for fp32
scores, exponentials and sums, 2^-20 of the largest |v| for probabilities below the halves' normal range."""
import numpy as np
import pytest

from oracle import tokens as ref
from test_gpu_kv8 import HALF_ULP, TYPES, Cache, _cu, _i32

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2208_01944_gb300 import binding
    yield binding
    assert binding.palquant_sync_check() == binding.PQ_OK


def _queries(total, Hq, D, kind, seed):
    rng = np.random.default_rng(seed)
    q = torch.from_numpy(rng.normal(size=(total, Hq, D)).astype(np.float32)).to(TYPES[kind]).cuda()
    return q, torch.full_like(q, 7.0)


def _sinks(B, c, q, o, n, lens, window, sinks, stream=None):
    a = B.kv8_attn(q, o, _cu(n), _i32(lens), c.table_dev, max(n), max(lens), q.shape[2] ** -0.5, True, window)
    nbytes = B.palquant_kv8_attention_sinks_scratch_bytes(c.desc, a, sinks)
    scratch = torch.full((max(1, nbytes),), 255, dtype=torch.uint8, device="cuda")  # NaN wherever nothing is written
    B.palquant_kv8_attention_sinks(c.desc, q, o, a, sinks, scratch, nbytes, stream)
    return a, scratch


def _tree(B, c, q, o, n, lens, bits, stream=None):
    a = B.kv8_attn(q, o, _cu(n), _i32(lens), c.table_dev, max(n), max(lens), q.shape[2] ** -0.5)
    t = B.kv8_tree(bits, a)
    nbytes = B.palquant_kv8_attention_tree_scratch_bytes(c.desc, a, t)
    scratch = torch.full((max(1, nbytes),), 255, dtype=torch.uint8, device="cuda")
    B.palquant_kv8_attention_tree(c.desc, q, o, a, t, scratch, nbytes, stream)
    return a, t, scratch


def _check(c, q, o, n, lens, kind, seen):
    """seen(b): what sequence b's queries see, [n, length]."""
    at = np.concatenate([[0], np.cumsum(n)])
    q, o = q.float().cpu().numpy(), o.float().cpu().numpy().astype(np.float64)
    for b in range(len(n)):
        k = ref.read(c.k, c.ks, c.table[b], 0, lens[b])
        v = ref.read(c.v, c.vs, c.table[b], 0, lens[b])
        mask = seen(b)
        want, spread, top = ref.attention(q[at[b]:at[b + 1]], k, v, float(np.float32(q.shape[2] ** -0.5)), seen=mask)
        got = o[at[b]:at[b + 1]]
        big = np.abs(v[mask.any(0)]).max(initial=0)
        tol = HALF_ULP[kind] * np.abs(want) + ((2.0 ** -21 if kind == "f32" else 2.0 ** -11) + 2.0 ** -20 * (2 + top)) * spread
        tol = tol + 2.0 ** -20 * big * (0.01 if kind == "f32" else 1) + (2.0 ** -25 if kind == "f16" else 0)
        assert np.all(np.abs(got - want) <= tol), (b, np.max(np.abs(got - want) - tol))
        assert not got[~mask.any(1)].any()  # a query that sees nothing gives 0


SINKS = [  # queries, tokens, Hq, H, D, T, window, sinks
    ([1], [700], 8, 2, 64, 16, 256, 4),
    ([1, 1, 1, 1], [1, 0, 20, 1000], 4, 2, 16, 16, 16, 1),
    ([1, 1], [900, 33], 7, 1, 128, 64, 100, 200),       # more sinks than tokens in the window, than tokens
    ([1], [9000], 16, 2, 128, 128, 700, 130),           # parts that are joined
    ([1, 1], [3001, 2500], 12, 1, 96, 32, 701, 17),
    ([5, 33, 0], [260, 33, 80], 4, 2, 256, 64, 20, 3),
    ([4, 2, 1], [400, 130, 64], 6, 3, 80, 32, 1, 5),    # a window of the token itself
    ([70, 200, 1], [700, 333, 90], 8, 2, 128, 64, 60, 4),
    ([150], [2700], 4, 4, 64, 16, 100, 129),            # a second step of sinks on the tensor cores
    ([130, 20], [1300, 400], 5, 1, 32, 128, 33, 1),
    ([300, 10], [1000, 500], 4, 2, 128, 32, 300, 250),  # sinks that reach into some rows' windows
    ([20, 3], [9, 0], 4, 2, 64, 16, 4, 2),              # more queries than tokens: the first see nothing
    ([257], [2057], 10, 2, 112, 64, 1000, 64),
    ([60], [5000], 4, 1, 128, 16, 640, 128),            # parts on the tensor cores
]


# More work than finds room at one time, so that 16-bit queries go to the tensor cores: one tile of rows (two streams of softmax) and
# two, one half step and many, parts that are joined, odd sizes of heads, sequences of nothing.
SINKS += [
    ([21] * 20 + [1, 0, 9], [300, 77] * 10 + [500, 0, 9], 8, 4, 128, 64, 50, 4),
    ([12] * 30, [64, 90, 130] * 10, 16, 4, 64, 16, 33, 20),
    ([45] * 12, [45, 400, 200] * 4, 6, 3, 96, 32, 128, 130),
    ([90] * 12, [90, 500, 333] * 4, 6, 3, 112, 128, 100, 7),
    ([30], [9000], 4, 1, 128, 64, 5000, 100),
    ([30, 25], [9000, 8000], 8, 2, 32, 16, 5000, 16),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("case", SINKS, ids=str)
def test_sinks(B, case, kind):
    n, lens, Hq, H, D, T, window, sinks = case
    c = Cache(B, lens, H, D, T, seed=D + Hq)
    q, o = _queries(sum(n), Hq, D, kind, D)
    _sinks(B, c, q, o, n, lens, window, sinks)
    _check(c, q, o, n, lens, kind, lambda b: ref.sees_sinks(n[b], lens[b], window, sinks))


@pytest.mark.parametrize("n", [1, 90])
def test_sinks_that_hide_nothing_are_plain_attention(B, n):
    c = Cache(B, [700], 2, 64, 32, seed=3)
    q, o = _queries(n, 6, 64, "bf16", 1)
    plain = torch.empty_like(q)
    for window, sinks in ((0, 5), (700, 5), (0x7FFFFFFF, 0x7FFFFFFF), (90, 0)):
        a = B.kv8_attn(q, plain, _cu([n]), _i32([700]), c.table_dev, n, 700, 0.125, True, window)
        scratch = torch.empty(max(1, B.palquant_kv8_attention_scratch_bytes(c.desc, a)), dtype=torch.uint8, device="cuda")
        B.palquant_kv8_attention(c.desc, q, plain, a, scratch, scratch.numel())
        _sinks(B, c, q, o, [n], [700], window, sinks)
        assert torch.equal(o, plain)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,sequences", [(1, 1), (120, 1), (40, 14), (90, 9)])
def test_pages_between_sinks_and_window_are_not_read(B, n, sequences, kind):
    """Page ids out of range, NaN scales and scales of zero where no query looks."""
    T, window, sinks, length = 16, 100, 20, 2000
    c = Cache(B, [length], 2, 64, T, seed=5)
    table = c.table_dev.clone()
    lo = length - n + 1 - window
    hidden = [s for s in range(-(-length // T)) if s * T >= sinks and (s + 1) * T <= lo]
    assert len(hidden) > 60
    pages = c.table[0, hidden]
    c.ks[pages], c.vs[pages] = np.nan, np.inf
    for d, h in zip(c.dev, (c.k, c.v, c.ks, c.vs)):
        d.copy_(torch.from_numpy(h))
    table[0, hidden[::2]] = -5
    c.table_dev, c.table = table.expand(sequences, -1).contiguous(), np.repeat(c.table, sequences, 0)  # the same text for every sequence
    ns, lens = [n] * sequences, [length] * sequences
    q, o = _queries(n * sequences, 6, 64, kind, 2)
    _sinks(B, c, q, o, ns, lens, window, sinks)
    assert B.palquant_sync_check() == B.PQ_OK
    _check(c, q, o, ns, lens, kind, lambda b: ref.sees_sinks(n, length, window, sinks))


def _masks(kind, n, rng):
    """Bits of one sequence's drafts [n, words] as Python integers: a chain, a star, a random tree, or any bits at all."""
    rows = []
    for i in range(n):
        parent = {"chain": i - 1, "star": -1}.get(kind, int(rng.integers(-1, i)))
        rows.append(int.from_bytes(rng.bytes(n // 8 + 1), "little") & ((1 << n) - 1) if kind == "any" else
                    (rows[parent] if parent >= 0 else 0) | 1 << i)
    return rows


def _bits(masks, words, pitch=None):
    out = np.zeros((sum(map(len, masks)), pitch or words), np.uint32)
    out[:, words:] = 0xFFFFFFFF
    for r, m in enumerate(m for of in masks for m in of):
        out[r, :words] = [(m >> 32 * w) & 0xFFFFFFFF for w in range(words)]
    return out


TREES = [  # drafts, tokens with them, Hq, H, D, T, masks
    ([1], [1], 1, 1, 16, 16, "tree"),
    ([12], [300], 8, 2, 64, 16, "tree"),
    ([5, 1, 0, 7], [5, 33, 0, 1000], 4, 2, 96, 32, "tree"),
    ([9, 3], [5000, 77], 4, 4, 128, 128, "star"),       # parts that are joined
    ([31, 32], [100, 32], 3, 1, 80, 64, "any"),
    ([33, 2], [260, 200], 2, 2, 256, 64, "tree"),
    ([24, 24, 1, 17], [24, 700, 90, 2000], 8, 2, 128, 64, "tree"),
    ([64], [1064], 4, 1, 64, 16, "chain"),
    ([65, 40], [129, 999], 5, 1, 32, 128, "any"),
    ([130, 128], [500, 128], 4, 2, 128, 32, "tree"),
    ([200], [3000], 2, 1, 112, 64, "any"),
    ([20, 3], [9, 0], 4, 2, 64, 16, "any"),             # more drafts than tokens: the first ones are not in the cache
    ([90], [60], 4, 2, 128, 16, "any"),
    ([48], [6000], 4, 1, 128, 16, "tree"),              # parts on the tensor cores
]


TREES += [  # (as with the sinks above)
    ([21] * 20 + [1, 0, 9], [300, 77] * 10 + [500, 0, 9], 8, 4, 128, 64, "tree"),
    ([12] * 30, [12, 64, 130] * 10, 16, 4, 64, 16, "any"),
    ([33] * 12, [33, 400, 200] * 4, 9, 3, 96, 32, "any"),
    ([70] * 12, [70, 500, 333] * 4, 6, 3, 112, 128, "tree"),
    ([30], [7000], 4, 1, 128, 64, "tree"),
    ([30, 25], [7000, 6001], 8, 2, 32, 16, "any"),
    ([130], [5000], 2, 1, 128, 32, "any"),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("case", TREES, ids=str)
def test_tree(B, case, kind):
    n, lens, Hq, H, D, T, masks = case
    c = Cache(B, lens, H, D, T, seed=D + Hq)
    rng = np.random.default_rng(sum(n))
    bits = _bits([_masks(masks, m, rng) for m in n], -(-max(n) // 32), 9)
    q, o = _queries(sum(n), Hq, D, kind, D)
    wide = torch.from_numpy(bits.view(np.int32)).cuda()
    _tree(B, c, q, o, n, lens, wide[:, : -(-max(n) // 32)])
    at = np.concatenate([[0], np.cumsum(n)])
    _check(c, q, o, n, lens, kind, lambda b: ref.sees_tree(n[b], lens[b], bits[at[b]:at[b + 1]]))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("n", [7, 70])
def test_chain_is_causal_attention_and_bits_past_the_drafts_do_not_count(B, n, kind):
    c = Cache(B, [900], 2, 128, 64, seed=7)
    q, o = _queries(n, 8, 128, kind, 3)
    bits = np.full((n, 4), 0xFFFFFFFF, np.uint32)
    for i in range(n):
        for j in range(i + 1, n):
            bits[i, j // 32] &= ~np.uint32(1 << (j % 32))
    _tree(B, c, q, o, [n], [900], torch.from_numpy(bits.view(np.int32)).cuda())
    _check(c, q, o, [n], [900], kind, lambda b: ref.sees_sinks(n, 900, 0, 0))


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n,sequences", [(6, 1), (80, 1), (24, 40), (72, 20)])
def test_drafts_that_see_nothing(B, n, sequences, kind):
    """No text before the drafts, and rows of bits that are empty: zeros, beside rows that see only themselves."""
    ns = [n] * sequences
    c = Cache(B, ns, 2, 64, 16, seed=n)
    bits = _bits([[(1 << i) if i % 3 else 0 for i in range(n)]] * sequences, -(-n // 32))
    q, o = _queries(n * sequences, 4, 64, kind, 4)
    _tree(B, c, q, o, ns, ns, torch.from_numpy(bits.view(np.int32)).cuda())
    _check(c, q, o, ns, ns, kind, lambda b: ref.sees_tree(n, n, bits[:n]))
    assert not o.view(sequences, n, 4, 64)[:, ::3].any()


@pytest.mark.parametrize("n,sequences", [(6, 1), (80, 1), (24, 40), (72, 20)])
def test_drafts_that_a_draft_does_not_see_do_not_touch_it(B, n, sequences):
    """Siblings on a page with NaN scales: only the drafts that see it become NaN."""
    T = 16
    ns, lens = [n] * sequences, [64 + n] * sequences
    c = Cache(B, lens, 2, 64, T, seed=9)
    c.ks[c.table[:, 64 // T]] = np.nan  # drafts 0 to T - 1
    c.dev[2].copy_(torch.from_numpy(c.ks))
    bits = _bits([[1 if i % 2 else 0 for i in range(n)]] * sequences, -(-n // 32))
    q, o = _queries(n * sequences, 8, 64, "f16", 5)
    _tree(B, c, q, o, ns, lens, torch.from_numpy(bits.view(np.int32)).cuda())
    assert torch.isnan(o[1::2]).all() and torch.isfinite(o[::2]).all()  # (n is even)


@pytest.mark.parametrize("view", ["sinks", "tree"])
def test_graphs_and_streams_with_a_workspace_each(B, view):
    """Two captured calls, replayed on two streams, give what the calls gave; rows that belong to no sequence keep theirs."""
    n, lens = [3, 2], [4000, 1500]
    c = Cache(B, lens, 2, 128, 64, seed=11)
    bits = torch.from_numpy(_bits([_masks("tree", m, np.random.default_rng(1)) for m in n], 1).view(np.int32)).cuda()
    sets = [_queries(8, 8, 128, "bf16", s) for s in (1, 2)]
    want, graphs, keep = [], [], []
    for q, o in sets:
        a = B.kv8_attn(q, o, _cu(n), _i32(lens), c.table_dev, 3, 4000, 0.1, True, 3500 if view == "sinks" else 0)
        t = B.kv8_tree(torch.cat([bits, bits[:3]]), a)
        nbytes = max(1, B.palquant_kv8_attention_sinks_scratch_bytes(c.desc, a, 4) if view == "sinks" else
                     B.palquant_kv8_attention_tree_scratch_bytes(c.desc, a, t))
        scratch = torch.empty(nbytes, dtype=torch.uint8, device="cuda")

        def call(q=q, o=o, a=a, t=t, scratch=scratch):
            if view == "sinks":
                B.palquant_kv8_attention_sinks(c.desc, q, o, a, 4, scratch, scratch.numel())
            else:
                B.palquant_kv8_attention_tree(c.desc, q, o, a, t, scratch, scratch.numel())

        call()
        torch.cuda.synchronize()
        assert bool((o[5:] == 7).all())
        want.append(o.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
        keep.append((a, t, scratch))
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for (q, o), graph, stream in zip(sets, graphs, streams):
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                o.zero_()
                graph.replay()
        torch.cuda.synchronize()
        for (q, o), w in zip(sets, want):
            assert torch.equal(o[:5], w[:5]) and not o[5:].any()


@pytest.mark.parametrize("n", [1, 60])
def test_sinks_of_a_long_cache_past_32_bits(B, n):
    """Pages whose codes lie beyond 2^32 bytes, at both ends of the walk."""
    H, D, T = 16, 128, 128
    pages = (1 << 32) // (H * T * D) + 6
    g = torch.Generator(device="cuda").manual_seed(2)
    k = torch.zeros((pages, H, T, D), dtype=torch.int8, device="cuda")
    v = torch.zeros_like(k)
    ids = [pages - 1, pages - 3, pages - 2, 0, pages - 4]
    for side in (k, v):
        side[ids] = torch.randint(-127, 128, (5, H, T, D), generator=g, device="cuda", dtype=torch.int8)
    ks, vs = torch.full((pages, H), 0.02, device="cuda"), torch.full((pages, H), 0.02, device="cuda")
    cache = B.kv8_cache(k, v, ks, vs)
    length = 5 * T - 3
    q = torch.randn(n, H, D, generator=g, device="cuda").half()
    o = torch.empty_like(q)
    a = B.kv8_attn(q, o, _cu([n]), _i32([length]), _i32([ids]), n, length, D ** -0.5, True, 150)
    scratch = torch.empty(max(1, B.palquant_kv8_attention_sinks_scratch_bytes(cache, a, 9)), dtype=torch.uint8, device="cuda")
    B.palquant_kv8_attention_sinks(cache, q, o, a, 9, scratch, scratch.numel())
    kf, vf = (x[ids].permute(0, 2, 1, 3).reshape(-1, H, D)[:length].float().cpu().numpy() * np.float32(0.02) for x in (k, v))
    want, spread, top = ref.attention(q.float().cpu().numpy(), kf, vf, float(np.float32(D ** -0.5)), seen=ref.sees_sinks(n, length, 150, 9))
    tol = 2.0 ** -11 * np.abs(want) + (2.0 ** -11 + 2.0 ** -20 * (2 + top)) * spread + 2.0 ** -18
    assert np.all(np.abs(o.float().cpu().numpy() - want) <= tol)


@pytest.mark.parametrize("view", ["sinks", "tree"])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("n,lens,Hq,H,D,T", [([30, 30], [9000, 0], 4, 1, 128, 64), ([25, 30, 12], [0, 8000, 0], 8, 2, 64, 16)])
def test_queries_without_tokens_beside_long_texts(B, n, lens, Hq, H, D, T, kind, view):
    """One tile of rows cut into parts: the empty texts' rows are joined from a part without a step.  They give 0, whatever their
    queries hold (a NaN in one, the largest numbers in another)."""
    c = Cache(B, [max(1, v) for v in lens], H, D, T, seed=13)
    q, o = _queries(sum(n), Hq, D, kind, 6)
    at = np.concatenate([[0], np.cumsum(n)])
    for b in range(len(n)):
        if lens[b] == 0:
            q[at[b]:at[b] + 2], q[at[b] + 3] = float("nan"), 60000.0
    bits = np.full((sum(n), 1), 0xFFFFFFFF, np.uint32)
    for _ in range(10):
        if view == "sinks":
            _, scratch = _sinks(B, c, q, o, n, lens, 5000, 100)
        else:
            scratch = _tree(B, c, q, o, n, lens, torch.from_numpy(bits.view(np.int32)).cuda())[2]
        assert scratch.numel() > 1
        for b in range(len(n)):
            if lens[b] == 0:
                assert not o[at[b]:at[b + 1]].any()  # (a NaN counts as something)
    full = [b for b in range(len(n)) if lens[b]]
    rows = np.concatenate([np.arange(at[b], at[b + 1]) for b in full])
    c.table = c.table[full]
    _check(c, q[rows], o[rows], [n[b] for b in full], [lens[b] for b in full], kind,
           lambda i: ref.sees_sinks(n[full[i]], lens[full[i]], 5000, 100) if view == "sinks" else ref.sees_tree(n[full[i]], lens[full[i]], bits))


@pytest.mark.parametrize("n,sequences,Hq,H,D", [(1, 1, 32, 8, 128), (40, 1, 8, 2, 64), (12, 20, 8, 2, 64), (70, 9, 8, 2, 64), (9, 2, 16, 4, 256)])
@pytest.mark.parametrize("window", [20, 43, 44, 1000, "tree"])
def test_half_precision_outputs_are_off_by_their_rounding(B, window, n, sequences, Hq, H, D):
    """Of all outputs together, in the norm: with 11-bit weights the error is about sqrt(2) of the rounding's, whether a window hides something of
    the text (44 tokens, or as many as the queries) or only could.

    Bound: the exact outputs' own rounding, 1/16 more for other elements being rounded than those (thousands of them, each error
    spread evenly over a step), and 2^-20 (2 + max |score|) spread for fp32 scores, exponentials and sums, as everywhere."""
    length = max(44, n)
    ns, lens = [n] * sequences, [length] * sequences
    c = Cache(B, lens, H, D, 16, seed=21)
    q, o = _queries(n * sequences, Hq, D, "f16", 8)
    q *= 0.25  # (the weight of a token that outweighs the others is a power of two: no rounding would show)
    if window == "tree":
        bits = np.zeros((n * sequences, -(-n // 32)), np.uint32)
        for i in range(n):
            bits[i::n, i // 32] = 1 << (i % 32)
        _tree(B, c, q, o, ns, lens, torch.from_numpy(bits.view(np.int32)).cuda())
        seen = ref.sees_tree(n, length, bits[:n])
    else:
        _sinks(B, c, q, o, ns, lens, window, 4)
        seen = ref.sees_sinks(n, length, window, 4)
    off = allowed = bound = 0.0
    qf, of = q.float().cpu().numpy(), o.double().cpu().numpy()
    for b in range(sequences):
        k, v = ref.read(c.k, c.ks, c.table[b], 0, length), ref.read(c.v, c.vs, c.table[b], 0, length)
        want, spread, top = ref.attention(qf[b * n:(b + 1) * n], k, v, float(np.float32(D ** -0.5)), seen=seen)
        off += ((of[b * n:(b + 1) * n] - want) ** 2).sum()
        allowed += ((want.astype(np.float16).astype(np.float64) - want) ** 2).sum()
        bound += ((2.0 ** -20 * (2 + top) * spread) ** 2).sum()
    assert off ** 0.5 <= 17 / 16 * allowed ** 0.5 + bound ** 0.5, (off ** 0.5 / allowed ** 0.5, bound ** 0.5 / allowed ** 0.5)
