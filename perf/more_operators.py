"""Cases, plain forms and definitions of a decoder's operators around the 8-bit cache.

  project  tokens times 4-bit weights with a scale for each output channel and group of input channels, plus an
           optional bias
  rotate   root-mean-square norm of every query and key head with a weight for each element, and the rotation
           by the token's position, in one pass
  sinks    attention over the 8-bit cache through a sliding window and a few first tokens that stay visible
  tree     attention over the 8-bit cache for a tree of drafted tokens: each sees the text and its ancestors

``run`` computes a case in elementary torch operations in 32 bits (angles in 64), or, where ``own`` is set, through
the package's entry points.  ``exact`` states the same in 64 bits.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ cases
def listed():
    def project(name, M, N, K, group, dtype, scales="f16", bias=False):
        return {"name": name, "op": "project", "M": M, "N": N, "K": K, "group": group, "dtype": dtype, "scales": scales,
                "bias": bias}

    def rotate(name, B, n, start, Hq, Hkv, D, R, dtype, interleaved=False, theta=500000.0):
        return {"name": name, "op": "rotate", "B": B, "n": n, "start": start, "Hq": Hq, "Hkv": Hkv, "D": D, "R": R,
                "dtype": dtype, "interleaved": interleaved, "theta": theta}

    def attention(name, op, B, q, length, Hq, Hkv, D, T, dtype, window=0, sinks=0, empty=False):
        return {"name": name, "op": op, "B": B, "q": q, "len": length, "Hq": Hq, "Hkv": Hkv, "D": D, "T": T, "dtype": dtype,
                "window": window, "sinks": sinks, "empty": empty}

    return [
        # One token through one projection: a single user's step, bound by latency and the weights' bytes.
        project("project one token", 1, 4096, 4096, 128, "bf16"),
        # A few tokens, odd sizes, 32-bit activations and scales, the last group not full.
        project("project odd", 5, 1001, 777, 32, "f32", scales="f32", bias=True),
        # A few users' tokens through the widest layer: bound by the weights' bytes.
        project("project wide", 8, 16384, 8192, 128, "f16"),
        # A batch of users, small groups: as many products as the weights' bytes allow.
        project("project batch", 48, 8192, 4096, 64, "bf16"),
        # One token far into a text: latency.
        rotate("rotate one token", 1, 1, 100000, 32, 8, 128, 128, "bf16"),
        # Odd head counts and sizes, half of each head rotated, neighbours as pairs, 32 bits.
        rotate("rotate odd", 3, 111, 77, 6, 3, 80, 40, "f32", interleaved=True, theta=10000.0),
        # Prompts of a batch: bound by the bytes.
        rotate("rotate prompts", 8, 2048, 4096, 32, 8, 128, 128, "bf16"),
        # One user's single token through a narrow window: latency.
        attention("sinks short", "sinks", 1, 1, 700, 8, 2, 64, 16, "f16", window=256, sinks=4),
        # A batch's single tokens, texts far longer than the window: bound by the visible codes' bytes.
        attention("sinks tokens", "sinks", 64, 1, 24000, 32, 8, 128, 64, "bf16", window=4096, sinks=4),
        # Prompts' later parts through a window.
        attention("sinks prompt", "sinks", 2, 4096, 10000, 32, 8, 128, 64, "bf16", window=2048, sinks=16),
        # One user's dozen drafts over a short text: latency.
        attention("tree one", "tree", 1, 12, 2000, 8, 2, 64, 16, "f16"),
        # A batch of users, two dozen drafts each over ragged texts, one with nothing yet.
        attention("tree batch", "tree", 32, 24, 6000, 32, 8, 128, 64, "bf16", empty=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["project", "project", "rotate", "sinks", "tree"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "project":
        while True:
            M, N, K = _log(rng, 1, 64), _log(rng, 64, 16384), _log(rng, 64, 16384)
            if rng.random() < 0.6:  # layers' widths are mostly round
                N, K = max(64, N // 64 * 64), max(64, K // 64 * 64)
            if N * K <= 16384 * 8192 and M * N * K <= 48 * 8192 * 4096:
                break
        return {"op": op, "M": M, "N": N, "K": K, "group": rng.choice([32, 64, 128]), "dtype": dtype,
                "scales": rng.choice(["f16", "f16", "bf16", "f32"]), "bias": rng.random() < 0.3}
    if op == "rotate":
        while True:
            B, n = _log(rng, 1, 64), 1 if rng.random() < 0.4 else _log(rng, 2, 8192)
            Hkv, D = rng.choice([1, 2, 3, 4, 8]), rng.choice([32, 64, 80, 96, 128, 128, 256])
            Hq = Hkv * rng.choice([1, 2, 4, 5, 8])
            if B * n * (Hq + Hkv) * D * BYTES[dtype] <= 8 * 2048 * 40 * 128 * 2:
                break
        return {"op": op, "B": B, "n": n, "start": 0 if rng.random() < 0.2 else _log(rng, 1, 1000000), "Hq": Hq, "Hkv": Hkv,
                "D": D, "R": D if rng.random() < 0.7 else D // 2, "dtype": dtype, "interleaved": rng.random() < 0.3,
                "theta": rng.choice([10000.0, 500000.0, 1000000.0])}
    while True:
        B, Hkv, group = _log(rng, 1, 64), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8])
        D = rng.choice([32, 64, 80, 96, 128, 128, 256])
        if op == "tree":
            q, length, window, sinks = _log(rng, 2, 128), _log(rng, 1, 20000), 0, 0
        else:
            q = 1 if rng.random() < 0.5 else _log(rng, 2, 4096)
            length, window, sinks = _log(rng, 1, 40000), _log(rng, 16, 6000), rng.choice([1, 4, 4, 16, 100])
        length = max(q, length)
        seen = min(length, window + q + sinks) if window else length
        pairs = B * q * seen * Hkv * group
        if (pairs * D * (4 if dtype == "f32" or D == 256 else 1) <= 2 * 4096 * 6160 * 32 * 128 and pairs <= 2 * 4096 * 6160 * 32
                and B * length * Hkv * D <= 64 * 15000 * 8 * 128 and B * seen * Hkv * D <= 64 * 6000 * 8 * 128):
            break
    return {"op": op, "B": B, "q": q, "len": length, "Hq": Hkv * group, "Hkv": Hkv, "D": D, "T": rng.choice([16, 32, 64, 128]),
            "dtype": dtype, "window": window, "sinks": sinks, "empty": B > 1 and rng.random() < 0.3}


def _ragged(most, least, B):
    """B numbers from least to most, the first the largest, spread evenly and in no order."""
    return [most - int((most - least) * math.modf(b * 0.6180339887)[0]) for b in range(B)]


def _rotate_counts(case):
    """(tokens, first position) of every sequence."""
    B = case["B"]
    return _ragged(case["n"], max(1, case["n"] // 2), B), _ragged(case["start"], case["start"] // 2, B)


def _attention_counts(case):
    """(queries, cached tokens with theirs) of every sequence."""
    B = case["B"]
    q = _ragged(case["q"], max(1, case["q"] // 3), B)
    lens = [max(n, v) for n, v in zip(q, _ragged(case["len"], max(1, case["len"] // 4), B))]
    if case["empty"]:
        q[-1] = lens[-1] = 0
    return q, lens


# ------------------------------------------------------------------------------------------------ inputs
def _pages(case, g, tokens):
    """A page table [B, pages of the longest sequence] over a pool in no order, and the pool's size."""
    need = [-(-n // case["T"]) for n in tokens]
    most, total = max(max(need), 1), max(sum(need), 1)
    ids = torch.randperm(total, generator=g, device=DEVICE).to(torch.int32)
    table = torch.zeros(len(need), most, dtype=torch.int32, device=DEVICE)
    inside = torch.arange(most, device=DEVICE)[None, :] < torch.tensor(need, device=DEVICE)[:, None]
    table[inside] = ids[: sum(need)]
    return table, total


def _codes(shape, g, spread=32.0, lo=-127, hi=127):
    """Codes as a quantiser leaves them: a bell, its widest at the ends."""
    out = torch.empty(shape, dtype=torch.int8, device=DEVICE)
    flat = out.view(-1)
    step = 1 << 27
    for at in range(0, flat.numel(), step):
        part = flat[at:at + step]
        part.copy_((torch.randn(part.numel(), generator=g, device=DEVICE) * spread).round_().clamp_(lo, hi))
    return out


def _scales(shape, g):
    return torch.exp(torch.randn(shape, generator=g, device=DEVICE) * 0.3) / 32


def _int32(values):
    return torch.tensor(values, dtype=torch.int32).to(DEVICE)


def _cumulative(counts):
    return _int32([0] + counts).cumsum(0).to(torch.int32)


def _parents(case, seed):
    """Every sequence's drafts: the parent of each among those before it (-1: it follows the text)."""
    rng = random.Random(seed)
    out = []
    for n in _attention_counts(case)[0]:
        # mostly a chain or a sibling of the newest drafts, now and then a new branch
        out.append([i - 1 - min(i, int(rng.expovariate(0.5))) for i in range(n)])
    return out


def _ancestor_bits(parents, words):
    """A row of 32-bit words for each draft: bit j is set where draft j is the draft itself or one of its ancestors."""
    rows = []
    for of_sequence in parents:
        masks = []
        for i, parent in enumerate(of_sequence):
            masks.append((masks[parent] if parent >= 0 else 0) | 1 << i)
        rows += [[(m >> 32 * w) & 0xFFFFFFFF for w in range(words)] for m in masks]
    return torch.tensor(rows, dtype=torch.int64).view(-1, words).to(torch.int32).to(DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    rand = lambda *shape: torch.randn(shape, generator=g, device=DEVICE)  # noqa: E731
    if case["op"] == "project":
        M, N, K = case["M"], case["N"], case["K"]
        x = rand(M, K) * torch.exp(rand(K) * 0.5) * torch.exp(rand(M, 1) * 0.3)  # some channels are louder than others
        scales = torch.exp(rand(N, -(-K // case["group"])) * 0.3) / (3 * math.sqrt(K))
        s = {"case": case, "x": x.to(dtype), "codes": _codes((N, K), g, 3.0, -8, 7), "scales": scales.to(DTYPES[case["scales"]]),
             "bias": rand(N) if case["bias"] else None, "y": torch.empty(M, N, dtype=dtype, device=DEVICE)}
    elif case["op"] == "rotate":
        n, start = _rotate_counts(case)
        Hq, Hkv, D, R = case["Hq"], case["Hkv"], case["D"], case["R"]
        # queries, keys and values side by side, as one projection writes them
        qkv = (rand(sum(n), Hq + 2 * Hkv, D) * torch.exp(rand(Hq + 2 * Hkv, 1) * 0.5)).to(dtype)
        positions = torch.cat([torch.arange(a, a + m, dtype=torch.int32) for a, m in zip(start, n)]).to(DEVICE)
        s = {"case": case, "q": qkv[:, :Hq], "k": qkv[:, Hq:Hq + Hkv], "positions": positions,
             "q_weight": (1 + 0.2 * rand(D)).to(dtype), "k_weight": (1 + 0.2 * rand(D)).to(dtype),
             "frequencies": [case["theta"] ** (-2.0 * i / R) for i in range(R // 2)],
             "q_out": torch.empty(sum(n), Hq, D, dtype=dtype, device=DEVICE),
             "k_out": torch.empty(sum(n), Hkv, D, dtype=dtype, device=DEVICE)}
        s["frequencies_dev"] = torch.tensor(s["frequencies"], dtype=torch.float64).to(DEVICE)
    else:
        q, lens = _attention_counts(case)
        H, D, T = case["Hkv"], case["D"], case["T"]
        table, pages = _pages(case, g, lens)
        s = {"case": case, "q": rand(sum(q), case["Hq"], D).to(dtype), "o": torch.empty(sum(q), case["Hq"], D, dtype=dtype, device=DEVICE),
             "cache": (_codes((pages, H, T, D), g), _codes((pages, H, T, D), g), _scales((pages, H), g), _scales((pages, H), g)),
             "table": table, "cu": _cumulative(q), "lens": _int32(lens), "max_q": max(q), "max_len": max(lens), "total_q": sum(q)}
        if case["op"] == "tree":
            s["bits"] = _ancestor_bits(_parents(case, seed), -(-max(q) // 32))
    if own:
        s["plan"] = _plan(s)
    return s


# ------------------------------------------------------------------------------------------------ the package's calls
def _plan(s):
    """The descriptors, packed weights and workspaces that a program makes once and keeps."""
    from paper_2208_01944_gb300 import binding as B

    case = s["case"]
    scratch = lambda n: torch.empty(max(1, n), dtype=torch.uint8, device=DEVICE)  # noqa: E731
    if case["op"] == "project":
        w = B.w4_weights(case["N"], case["K"], case["group"], s["scales"].dtype)
        packed = scratch(B.palquant_w4_packed_bytes(w))
        B.palquant_w4_pack(s["codes"], s["scales"], w, packed, packed.numel())
        d = B.linear_w4_desc(s["x"], w, s["y"])
        return w, packed, d, scratch(B.palquant_linear_w4_scratch_bytes(w, d))
    if case["op"] == "rotate":
        turns = B.rope_turns(s["frequencies"], DEVICE)
        return B.qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["positions"], turns, s["q_weight"], s["k_weight"],
                              eps=EPS, interleaved=case["interleaved"])
    cache = B.kv8_cache(*s["cache"])
    a = B.kv8_attn(s["q"], s["o"], s["cu"], s["lens"], s["table"], s["max_q"], s["max_len"], scale=case["D"] ** -0.5,
                   causal=True, window=case["window"])
    if case["op"] == "sinks":
        return cache, a, scratch(B.palquant_kv8_attention_sinks_scratch_bytes(cache, a, case["sinks"]))
    tree = B.kv8_tree(s["bits"], a)
    return cache, a, tree, scratch(B.palquant_kv8_attention_tree_scratch_bytes(cache, a, tree))


def _run_own(s):
    from paper_2208_01944_gb300 import binding as B

    op = s["case"]["op"]
    if op == "project":
        w, packed, d, scratch = s["plan"]
        B.palquant_linear_w4(s["x"], packed, s["bias"], s["y"], w, d, scratch, scratch.numel())
        return s["y"]
    if op == "rotate":
        B.palquant_qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], s["plan"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "sinks":
        cache, a, scratch = s["plan"]
        B.palquant_kv8_attention_sinks(cache, s["q"], s["o"], a, s["case"]["sinks"], scratch, scratch.numel())
        return s["o"]
    cache, a, tree, scratch = s["plan"]
    B.palquant_kv8_attention_tree(cache, s["q"], s["o"], a, tree, scratch, scratch.numel())
    return s["o"]


# ------------------------------------------------------------------------------------------------ plain forms
def _project_plain(s):
    case = s["case"]
    scales = s["scales"].float().repeat_interleave(case["group"], 1)[:, : case["K"]]
    y = s["x"].float() @ (s["codes"].float() * scales).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["x"].dtype)


def _rotate_plain(s):
    R = s["case"]["R"]
    angle = s["positions"].double()[:, None] * s["frequencies_dev"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def one(x, weight):
        x32 = x.float()
        x32 = x32 * torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + EPS) * weight.float()
        out = x32.clone()
        first, second = (slice(0, R, 2), slice(1, R, 2)) if s["case"]["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
        a, b = x32[..., first], x32[..., second]
        out[..., first] = a * cos - b * sin
        out[..., second] = b * cos + a * sin
        return out.to(x.dtype)

    return {"q": one(s["q"], s["q_weight"]), "k": one(s["k"], s["k_weight"])}


def _attention_plain(s):
    case, table = s["case"], s["table"].long()
    B, H, D, T, Q = case["B"], case["Hkv"], case["D"], case["T"], s["max_q"]
    group, window, sinks = case["Hq"] // H, case["window"], case["sinks"]
    k_codes, v_codes, k_scales, v_scales = s["cache"]
    cu, lens = s["cu"].long(), s["lens"].long()
    count = cu[1:] - cu[:-1]
    # the tokens that some query of a sequence sees: the first ones, and the last ones
    last = min(s["max_len"], window + Q - 1) if window else s["max_len"]
    first = min(sinks, s["max_len"])
    tail = (lens[:, None] - last).clamp(min=0) + torch.arange(last, device=DEVICE)
    head = torch.arange(first, device=DEVICE).expand(B, first)
    at = torch.cat([head, tail], 1)  # [B, L]
    there = (at < lens[:, None])
    if first:
        there[:, :first] &= head < tail[:, :1]  # (a first token that is among the last ones counts once)
    L = at.shape[1]
    page, slot = table.gather(1, (at // T).clamp(max=table.shape[1] - 1)), at % T

    def values(codes, scales):
        v = codes[page, :, slot].float() * scales[page][..., None]  # [B, L, H, D]
        return torch.where(there[..., None, None], v, 0.0).transpose(1, 2)

    i = torch.arange(Q, device=DEVICE)
    row = (cu[:-1, None] + i).clamp(max=s["total_q"] - 1)
    q = s["q"].float()[row].view(B, Q, H, group, D).permute(0, 2, 3, 1, 4).reshape(B, H, group * Q, D)
    score = (q @ values(k_codes, k_scales).transpose(2, 3)).view(B, H, group, Q, L) * D ** -0.5
    place = (lens - count)[:, None] + i  # [B, Q]
    at = at[:, None]
    if case["op"] == "tree":
        draft = at - (lens - count)[:, None, None]  # [B, 1, L]: the draft's number, below 0 in the text
        word = s["bits"].long()[row].gather(2, (draft // 32).clamp(0, s["bits"].shape[1] - 1).expand(B, Q, L))
        seen = (draft < 0) | ((word >> (draft % 32)) & 1).bool()
    else:
        seen = at <= place[..., None]
        if window:
            seen = seen & ((at > place[..., None] - window) | (at < sinks))
    seen = (seen & there[:, None])[:, None, None]
    score = score.masked_fill_(~seen, float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, H, group * Q, L) @ values(v_codes, v_scales)).view(B, H, group, Q, D) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(B * Q, case["Hq"], D)
    b = torch.repeat_interleave(torch.arange(B, device=DEVICE), count, output_size=s["total_q"])
    return o[b * Q + torch.arange(s["total_q"], device=DEVICE) - cu[:-1][b]].to(s["q"].dtype)


def run(state):
    if own:
        return _run_own(state)
    return {"project": _project_plain, "rotate": _rotate_plain, "sinks": _attention_plain, "tree": _attention_plain}[
        state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_project(s):
    group, K = s["case"]["group"], s["case"]["K"]
    x, scales = s["x"].double(), s["scales"].double()
    out = torch.zeros(s["y"].shape, dtype=torch.float64, device=DEVICE)
    for j in range(scales.shape[1]):
        part = slice(j * group, min(K, (j + 1) * group))
        out += torch.mm(x[:, part], s["codes"][:, part].double().t()) * scales[:, j]
    return out if s["bias"] is None else out + s["bias"].double()


def _exact_rotate(s):
    R, interleaved = s["case"]["R"], s["case"]["interleaved"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE),
                       torch.outer(s["positions"].double(), s["frequencies_dev"]))  # [tokens, R / 2]
    found = {}
    for name in ("q", "k"):
        x = s[name].double()
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * s[name + "_weight"].double()
        rotated = x[..., :R]
        pairs = rotated.unflatten(-1, (R // 2, 2)) if interleaved else rotated.unflatten(-1, (2, R // 2)).transpose(-1, -2)
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
        rotated = pairs.flatten(-2) if interleaved else pairs.transpose(-1, -2).flatten(-2)
        found[name] = torch.cat([rotated, x[..., R:]], -1)
    return found


def _sees(case, parents, length, n, lo, m, keys):
    """Which of `keys` (positions) the queries lo to lo + m of a sequence see, [m, keys]."""
    if case["op"] == "sinks":
        place = length - n + lo + torch.arange(m, device=DEVICE)[:, None]
        near = (keys <= place) & (keys > place - case["window"])
        return near | ((keys < case["sinks"]) & (keys <= place))
    seen = torch.zeros(m, length, dtype=torch.bool)
    seen[:, : length - n] = True
    for i in range(m):
        j = lo + i
        while j >= 0:
            seen[i, length - n + j] = True
            j = parents[j]
    return seen.to(DEVICE)[:, keys]


def _exact_attention(s, seed):
    case, table = s["case"], s["table"].long()
    H, D, T, group = case["Hkv"], case["D"], case["T"], case["Hq"] // case["Hkv"]
    cu, lens = s["cu"].cpu().tolist(), s["lens"].cpu().tolist()
    parents = _parents(case, seed) if case["op"] == "tree" else [None] * case["B"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    for b, length in enumerate(lens):
        n = cu[b + 1] - cu[b]
        for lo in range(0, n, 512):
            m = min(512, n - lo)
            keys = torch.arange(length, device=DEVICE)
            if case["op"] == "sinks":
                keys = keys[(keys > length - n + lo - case["window"]) & (keys < length - n + lo + m) | (keys < case["sinks"])]
            seen = _sees(case, parents[b], length, n, lo, m, keys).repeat_interleave(group, 0)
            page, slot = table[b][keys // T], keys % T
            rows = slice(cu[b] + lo, cu[b] + lo + m)
            for h in range(H):
                k = s["cache"][0][page, h, slot].double() * s["cache"][2][page, h].double()[:, None]
                v = s["cache"][1][page, h, slot].double() * s["cache"][3][page, h].double()[:, None]
                q = s["q"][rows, h * group:(h + 1) * group].double().reshape(m * group, D)
                score = (q @ k.t() / math.sqrt(D)).masked_fill(~seen, -math.inf)
                out[rows, h * group:(h + 1) * group] = (torch.softmax(score, 1) @ v).view(m, group, D)
    return out


def exact(case, seed):
    """The definition in 64 bits.  Every query here sees its own token."""
    s = prepare(case, seed)
    if case["op"] == "project":
        return _exact_project(s)
    if case["op"] == "rotate":
        return _exact_rotate(s)
    return _exact_attention(s, seed) if work(case)["flops"] < 2e12 else None


# ------------------------------------------------------------------------------------------------ work
def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "project":
        M, N, K = case["M"], case["N"], case["K"]
        groups = -(-K // case["group"])
        return {"bytes": M * K * e + N * K // 2 + N * groups * BYTES[case["scales"]] + (4 * N if case["bias"] else 0) + M * N * e,
                "flops": 2 * M * N * K}
    if case["op"] == "rotate":
        tokens, heads = sum(_rotate_counts(case)[0]), case["Hq"] + case["Hkv"]
        return {"bytes": 2 * tokens * heads * case["D"] * e + 4 * tokens + 2 * case["D"] * e,
                "flops": tokens * heads * (4 * case["D"] + 3 * case["R"])}
    H, D, T = case["Hkv"], case["D"], case["T"]
    q, lens = _attention_counts(case)
    pairs = read = 0
    for n, length in zip(q, lens):
        if case["op"] == "tree":
            # every draft's ancestors are at least itself
            pairs, read = pairs + n * (length - n) + n, read + length
            continue
        window, sinks = case["window"], case["sinks"]
        for i in range(n):
            p = length - n + i
            near = min(window, p + 1)
            pairs += near + min(sinks, p + 1 - near)
        near = min(length, window + n - 1)
        read += (near + min(sinks, length - near)) if n else 0
    mask = 4 * sum(q) * -(-max(q) // 32) if case["op"] == "tree" else 0
    return {"bytes": 2 * sum(q) * case["Hq"] * D * e + 2 * read * H * D + 8 * -(-read // T) * H + mask,
            "flops": 4 * pairs * case["Hq"] * D}
