"""The paged 8-bit cache and attention over it, against the oracle in double.

Append and read are bit-exact.  Attention's bound: with u the output type's half ulp and
spread = sum p |v|, an output may be off by
  u |o|                      the rounding to the type,
+ 2^-11 spread (16-bit), 2^-21 spread (fp32)   the probabilities as one or two halves,
+ 2^-20 (2 + max |score|) spread   scores, exponentials and sums in fp32,
+ 2^-20 of the largest |v|   probabilities below the halves' normal range."""
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


def _i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def _cu(counts):
    return _i32(np.concatenate([[0], np.cumsum(counts)]))


class Cache:
    """A pool on the GPU and its copy on the host, pages handed out in no order, the last one to nobody."""

    def __init__(self, B, tokens, H, D, T, seed=0, filled=False):
        rng = np.random.default_rng(seed)
        need = [max(1, -(-n // T)) for n in tokens]
        pages = sum(need) + 1
        order = rng.permutation(pages - 1)
        self.table = np.zeros((len(tokens), max(need)), np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            self.table[b, n:] = 1 << 30  # never to be looked at
            at += n
        self.k = rng.integers(-127, 128, (pages, H, T, D)).astype(np.int8)
        self.v = rng.integers(-127, 128, (pages, H, T, D)).astype(np.int8)
        self.ks = (np.exp(rng.normal(size=(pages, H)) * 0.5) / 60).astype(np.float32)
        self.vs = (np.exp(rng.normal(size=(pages, H)) * 2.0) / 60).astype(np.float32)
        self.dev = [torch.from_numpy(a.copy()).cuda() for a in (self.k, self.v, self.ks, self.vs)]
        self.desc = B.kv8_cache(*self.dev)
        self.table_dev = _i32(self.table)

    def same(self):
        return all(np.array_equal(d.cpu().numpy(), h, equal_nan=h.dtype == np.float32) for d, h in zip(self.dev, (self.k, self.v, self.ks, self.vs)))


APPENDS = [  # new tokens, tokens before, H, D, T
    ([1], [0], 1, 16, 16), ([1, 1, 1], [5, 15, 16], 2, 64, 16), ([3, 0, 40], [0, 7, 31], 3, 80, 32),
    ([100, 1, 64, 65], [64, 63, 0, 1], 2, 128, 64), ([300], [127], 1, 256, 128), ([257, 130], [3, 90], 4, 96, 128),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("case", APPENDS, ids=str)
def test_append_and_read(B, case, kind):
    n, start, H, D, T = case
    rng = np.random.default_rng(T + D)
    c = Cache(B, [a + b for a, b in zip(n, start)], H, D, T, seed=D)
    total = sum(n)
    # strides of a fused projection's output: k and v are slices of one tensor
    fused = torch.from_numpy((rng.normal(size=(total, 2 * H, D + 3)) * 3).astype(np.float32)).to(TYPES[kind]).cuda()
    wide = D % 2 == 0 and kind != "f32"
    k, v = (fused[:, :H, :D], fused[:, H:, 3:]) if wide else (fused[:, :H, :D].contiguous(), fused[:, H:, 3:].contiguous())
    t = B.kv8_tokens(k, v, _cu(n), _i32(start), c.table_dev, max(n))
    at = np.concatenate([[0], np.cumsum(n)])
    for _ in range(2):  # the second time the scales have grown already
        B.palquant_kv8_append(c.desc, k, v, t)
        for b in range(len(n)):
            ref.append(c.k, c.ks, c.table[b], start[b], k[at[b]:at[b + 1]].float().cpu().numpy())
            ref.append(c.v, c.vs, c.table[b], start[b], v[at[b]:at[b + 1]].float().cpu().numpy())
        assert c.same()
    ko, vo = torch.empty_like(k), torch.empty(v.shape, dtype=v.dtype, device="cuda")
    back = B.kv8_tokens(ko, vo, _cu(n), _i32(start), c.table_dev, max(n))
    B.palquant_kv8_read(c.desc, ko, vo, back)
    for got, codes, scales in ((ko, c.k, c.ks), (vo, c.v, c.vs)):
        want = np.concatenate([ref.read(codes, scales, c.table[b], start[b], n[b]) for b in range(len(n))])
        assert torch.equal(got.cpu(), torch.from_numpy(want).to(TYPES[kind]))


def test_append_token_by_token_keeps_the_largest_scale(B):
    H, D, T = 2, 64, 16
    rng = np.random.default_rng(1)
    c = Cache(B, [40], H, D, T)
    x = rng.normal(size=(40, H, D)).astype(np.float32) * rng.uniform(0, 4, (40, 1, 1)).astype(np.float32)
    x[3] = 0
    x[20, 1, 5] = np.inf  # poisons page 1 of head 1
    xd = torch.from_numpy(x).cuda()
    for i in range(40):
        t = B.kv8_tokens(xd[i:i + 1], xd[i:i + 1], _cu([1]), _i32([i]), c.table_dev, 1)
        B.palquant_kv8_append(c.desc, xd[i:i + 1], xd[i:i + 1], t)
        ref.append(c.k, c.ks, c.table[0], i, x[i:i + 1])
        ref.append(c.v, c.vs, c.table[0], i, x[i:i + 1])
    assert c.same()
    assert np.isnan(c.ks[c.table[0, 1], 1]) and np.isfinite(c.ks[c.table[0, 1], 0])


def _attend(B, c, q_counts, lens, Hq, kind, causal, window, seed=0, loud=1.0, strided=False, scale=None):
    H, D = c.k.shape[1], c.k.shape[3]
    rng = np.random.default_rng(seed)
    total = sum(q_counts)
    q = torch.from_numpy((rng.normal(size=(total, Hq, D)) * loud).astype(np.float32)).to(TYPES[kind]).cuda()
    o = torch.full((total, Hq, D), 7.0, dtype=TYPES[kind], device="cuda")
    if strided:  # heads first, and an odd element before the first
        qb = torch.zeros((Hq, total, D + 1), dtype=TYPES[kind], device="cuda")
        qb[:, :, 1:] = q.transpose(0, 1)
        q = qb[:, :, 1:].transpose(0, 1)
        o = torch.full((total, Hq, D + 1), 7.0, dtype=TYPES[kind], device="cuda")[:, :, 1:]
    scale = D ** -0.5 if scale is None else scale
    a = B.kv8_attn(q, o, _cu(q_counts), _i32(lens), c.table_dev, max(q_counts), max(lens), scale, causal, window)
    scratch = torch.empty(max(1, B.palquant_kv8_attention_scratch_bytes(c.desc, a)), dtype=torch.uint8, device="cuda")
    B.palquant_kv8_attention(c.desc, q, o, a, scratch, scratch.numel())
    return q.float().cpu().numpy(), o.float().cpu().numpy().astype(np.float64), float(np.float32(scale))


def _check(c, q, o, q_counts, lens, kind, causal, window, scale):
    at = np.concatenate([[0], np.cumsum(q_counts)])
    for b, n in enumerate(q_counts):
        k = ref.read(c.k, c.ks, c.table[b], 0, lens[b])
        v = ref.read(c.v, c.vs, c.table[b], 0, lens[b])
        want, spread, top = ref.attention(q[at[b]:at[b + 1]], k, v, scale, causal, window)
        got = o[at[b]:at[b + 1]]
        # probabilities carry the value scales: small ones are small beside the largest |v| seen
        big = np.abs(v).max(initial=0)
        tol = HALF_ULP[kind] * np.abs(want) + ((2.0 ** -21 if kind == "f32" else 2.0 ** -11) + 2.0 ** -20 * (2 + top)) * spread
        tol = tol + 2.0 ** -20 * big * (0.01 if kind == "f32" else 1) + (2.0 ** -25 if kind == "f16" else 0)
        assert np.all(np.abs(got - want) <= tol), (b, np.max(np.abs(got - want) - tol))


ATTENTIONS = [  # queries, tokens, Hq, H, D, T, causal, window
    ([1], [1], 1, 1, 16, 16, True, 0),
    ([1, 1, 1], [17, 0, 300], 8, 2, 64, 16, True, 0),
    ([1, 1], [1000, 129], 7, 1, 128, 64, True, 0),
    ([1], [5000], 16, 2, 128, 128, True, 0),
    ([1, 1], [3001, 2500], 12, 1, 96, 32, True, 700),
    ([4, 2, 1], [4, 130, 64], 6, 3, 80, 32, True, 0),
    ([5, 33], [260, 33], 4, 2, 256, 64, True, 0),
    ([70, 200, 1], [70, 333, 90], 8, 2, 128, 64, True, 0),
    ([150], [700], 4, 4, 64, 16, True, 100),
    ([130, 20], [130, 400], 5, 1, 32, 128, True, 33),
    ([300, 10], [40, 500], 4, 2, 128, 32, False, 0),
    ([20, 3], [9, 0], 4, 2, 64, 16, True, 0),  # more queries than tokens: the first see nothing
    ([260, 100], [600, 1000], 8, 1, 128, 128, True, 0),
    ([257], [257], 10, 2, 112, 64, True, 0),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("case", ATTENTIONS, ids=str)
def test_attention(B, case, kind):
    n, lens, Hq, H, D, T, causal, window = case
    c = Cache(B, lens, H, D, T, seed=D + Hq)
    q, o, scale = _attend(B, c, n, lens, Hq, kind, causal, window, seed=D)
    _check(c, q, o, n, lens, kind, causal, window, scale)
    at = np.concatenate([[0], np.cumsum(n)])
    for b in range(len(n)):  # queries that see no token
        blind = n[b] if lens[b] == 0 else max(0, n[b] - lens[b]) if causal else 0
        assert not o[at[b]:at[b] + blind].any()


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("n", [1, 40, 200])
def test_attention_strides_and_loud_scores(B, n, kind):
    """Heads-first queries at odd addresses; scores of several hundred (one token takes all)."""
    c = Cache(B, [500], 2, 64, 32, seed=4)
    q, o, scale = _attend(B, c, [n], [500], 6, kind, True, 0, loud=60.0, strided=True)
    _check(c, q, o, [n], [500], kind, True, 0, scale)


@pytest.mark.parametrize("n", [1, 150])
def test_attention_edges_of_the_scales(B, n):
    """Pages of zeros, poisoned pages that no query may see, and one that only the last queries see."""
    T, H, D, length = 32, 2, 64, 320
    c = Cache(B, [length + 64], H, D, T, seed=6)
    for side, s in ((0, 2), (1, 3)):
        page = c.table[0, 2]
        (c.k, c.v)[side][page, 0] = 0
        (c.ks, c.vs)[side][page, 0] = 0.0
    for block in (length // T, length // T + 1):  # past the end
        c.ks[c.table[0, block]] = np.nan
        c.vs[c.table[0, block]] = np.inf
    for d, h in zip(c.dev, (c.k, c.v, c.ks, c.vs)):
        d.copy_(torch.from_numpy(h))
    q, o, scale = _attend(B, c, [n], [length], 4, "f16", True, 0)
    _check(c, q, o, [n], [length], "f16", True, 0, scale)
    last = c.table[0, length // T - 1]  # the last page of the sequence
    c.dev[3][last] = float("nan")
    _, o, _ = _attend(B, c, [n], [length], 4, "f16", True, 0)
    sees = np.arange(length - n, length) >= length - T
    assert np.isnan(o[sees]).all() and np.isfinite(o[~sees]).all()


@pytest.mark.parametrize("n", [1, 140])
def test_attention_non_finite_queries_stay_in_their_row(B, n):
    c = Cache(B, [200], 1, 64, 16, seed=8)
    q = torch.randn(n, 4, 64, device="cuda").to(torch.bfloat16)
    clean = q.clone()
    q[0, 1, 3], q[0, 2, 0] = float("nan"), float("inf")
    outs = []
    for x in (q, clean):
        o = torch.empty_like(x)
        a = B.kv8_attn(x, o, _cu([n]), _i32([200]), c.table_dev, n, 200, 0.125)
        scratch = torch.empty(max(1, B.palquant_kv8_attention_scratch_bytes(c.desc, a)), dtype=torch.uint8, device="cuda")
        B.palquant_kv8_attention(c.desc, x, o, a, scratch, scratch.numel())
        outs.append(o.float().cpu())
    assert torch.isnan(outs[0][0, 1:3]).all()
    outs[0][0, 1:3] = outs[1][0, 1:3] = 0
    assert torch.equal(outs[0], outs[1])


def test_pages_out_of_range_are_reported_and_skipped(B):
    c = Cache(B, [100], 1, 64, 16, seed=9)
    table = c.table_dev.clone()
    table[0, 3], table[0, 4] = -1, c.k.shape[0]
    x = torch.randn(40, 1, 64, device="cuda")
    t = B.kv8_tokens(x, x, _cu([40]), _i32([40]), table, 40)
    before = [d.clone() for d in c.dev]
    B.palquant_kv8_append(c.desc, x, x, t)
    assert B.palquant_sync_check() == B.PQ_EINVAL
    assert B.palquant_sync_check() == B.PQ_OK  # reported once
    touched = c.table[0, 2]
    keep = np.arange(c.k.shape[0]) != touched
    for d, was in zip(c.dev, before):
        assert torch.equal(d[torch.from_numpy(keep).cuda()], was[torch.from_numpy(keep).cuda()])
    for n in (1, 64):
        q, o = torch.randn(n, 2, 64, device="cuda"), torch.empty(n, 2, 64, device="cuda")
        for kind in (torch.float32, torch.float16):
            a = B.kv8_attn(q.to(kind), o.to(kind), _cu([n]), _i32([100]), table, n, 100, 0.1)
            out = o.to(kind)
            scratch = torch.empty(max(1, B.palquant_kv8_attention_scratch_bytes(c.desc, a)), dtype=torch.uint8, device="cuda")
            B.palquant_kv8_attention(c.desc, q.to(kind), out, a, scratch, scratch.numel())
            assert B.palquant_sync_check() == B.PQ_EINVAL
            assert torch.isfinite(out.float()).all()


def test_offsets_past_32_bits(B):
    """Pages whose codes lie beyond 2^32 bytes of the pool."""
    H, D, T = 16, 256, 128
    pages = (1 << 32) // (H * T * D) + 6
    k = torch.zeros((pages, H, T, D), dtype=torch.int8, device="cuda")
    v = torch.zeros_like(k)
    ks, vs = torch.ones((pages, H), device="cuda"), torch.ones((pages, H), device="cuda")
    cache = B.kv8_cache(k, v, ks, vs)
    table = _i32([[pages - 1, pages - 3]])
    g = torch.Generator(device="cuda").manual_seed(1)
    x, y = (torch.randn(200, H, D, generator=g, device="cuda") for _ in range(2))
    t = B.kv8_tokens(x, y, _cu([200]), _i32([0]), table, 200)
    B.palquant_kv8_append(cache, x, y, t)
    assert not k[: pages - 3].any() and not v[: pages - 3].any() and not k[pages - 2].any()
    xo, yo = torch.empty_like(x), torch.empty_like(y)
    B.palquant_kv8_read(cache, xo, yo, B.kv8_tokens(xo, yo, _cu([200]), _i32([0]), table, 200))
    for got, want in ((xo, x), (yo, y)):
        for i in range(0, 200, T):
            part = want[i:i + T]
            step = part.abs().amax((0, 2)) / 127
            assert bool(((got[i:i + T] - part).abs() <= 0.501 * step[None, :, None]).all())
    for n in (1, 150):
        q, o = torch.randn(n, H, D, device="cuda").half(), torch.empty(n, H, D, device="cuda").half()
        a = B.kv8_attn(q, o, _cu([n]), _i32([200]), table, n, 200, 1 / 16)
        scratch = torch.empty(max(1, B.palquant_kv8_attention_scratch_bytes(cache, a)), dtype=torch.uint8, device="cuda")
        B.palquant_kv8_attention(cache, q, o, a, scratch, scratch.numel())
        want, spread, top = ref.attention(q.float().cpu().numpy(), xo.cpu().numpy(), yo.cpu().numpy(), 1 / 16)
        tol = 2.0 ** -11 * np.abs(want) + (2.0 ** -11 + 2.0 ** -20 * (2 + top)) * spread + 2.0 ** -18
        assert np.all(np.abs(o.float().cpu().numpy() - want) <= tol)


def test_results_do_not_change_from_call_to_call(B):
    c = Cache(B, [3000, 700], 2, 128, 64, seed=12)
    outs = [_attend(B, c, [1, 1], [3000, 700], 8, "bf16", True, 0)[1] for _ in range(4)]
    assert all(np.array_equal(outs[0], o) for o in outs[1:])
