"""Cases, plain forms and definitions of the 8-bit transformer operators.

  linear     tokens quantised to 8 bits with a scale each, times 8-bit weights with a scale for each
             output channel (exact integer sums), plus an optional bias
  append     new keys and values quantised into the pages of a cache that has one scale for each page and
             head, and the values the touched pages then stand for
  attention  attention over that cache: single tokens, chunks of a prompt, whole prompts

``run`` computes a case in elementary torch operations in 32 bits, or, where ``own`` is set, through the
package's entry points.  ``exact`` states the same in 64 bits.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
INV127 = 0.007874015718698502  # 1 / 127 rounded to 32 bits


# ------------------------------------------------------------------------------------------------ cases
def listed():
    def linear(name, M, N, K, dtype, bias=False):
        return {"name": name, "op": "linear", "M": M, "N": N, "K": K, "dtype": dtype, "bias": bias}

    def append(name, B, n, start, Hkv, D, T, dtype):
        return {"name": name, "op": "append", "B": B, "n": n, "start": start, "Hkv": Hkv, "D": D, "T": T, "dtype": dtype}

    def attention(name, B, q, length, Hq, Hkv, D, T, dtype, causal=True, window=0, empty=False):
        return {"name": name, "op": "attention", "B": B, "q": q, "len": length, "Hq": Hq, "Hkv": Hkv, "D": D, "T": T,
                "dtype": dtype, "causal": causal, "window": window, "empty": empty}

    return [
        # One token through one projection: a single user's step, bound by latency and the weights' bytes.
        linear("linear one token", 1, 4096, 4096, "bf16"),
        # A few tokens, odd sizes, 32-bit activations: a small classifier head over a narrow network.
        linear("linear odd", 13, 1001, 777, "f32", bias=True),
        # A batch of single tokens through a wide projection: serving.
        linear("linear batch", 48, 8192, 4096, "bf16"),
        # A prompt's tokens through a square projection.
        linear("linear prompt", 2048, 4096, 4096, "bf16"),
        # The largest: many prompts' tokens through a wide layer.
        linear("linear large", 8192, 8192, 8192, "f16", bias=True),
        # Every user of a batch adds one token in the middle of a page.
        append("append tokens", 128, 1, 1500, 8, 128, 32, "bf16"),
        # Odd head size and short prompts that begin inside a page, 32-bit inputs.
        append("append odd", 5, 333, 77, 3, 80, 16, "f32"),
        # Prompts of a batch.
        append("append prompts", 16, 4096, 0, 8, 128, 64, "bf16"),
        # One user's single token over a short text: latency.
        attention("attention short", 1, 1, 300, 8, 2, 64, 16, "f16"),
        # A batch's single tokens over ragged texts: bound by the cache's bytes.
        attention("attention tokens", 64, 1, 8192, 32, 8, 128, 64, "bf16"),
        # One token over one very long text: the work has to be split along it.
        attention("attention long", 1, 1, 130001, 28, 4, 128, 128, "bf16"),
        # Prompts, the second half of which follows a cached first half.
        attention("attention prompt", 4, 2048, 4096, 32, 8, 128, 64, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "append", "attention", "attention"])
    if op == "linear":
        while True:
            M, N, K = _log(rng, 1, 8192), _log(rng, 64, 12000), _log(rng, 64, 12000)
            if rng.random() < 0.5:  # layers' widths are mostly round, tokens' numbers are not
                N, K = max(64, N // 64 * 64), max(64, K // 64 * 64)
            if 3072 not in (M, N, K) and M * N * K <= 8192 ** 3:
                break
        return {"op": op, "M": M, "N": N, "K": K, "dtype": rng.choice(["bf16", "f16", "f32"]), "bias": rng.random() < 0.3}
    if op == "append":
        while True:
            B, Hkv, D = _log(rng, 1, 256), rng.choice([1, 2, 3, 8, 16]), rng.choice([32, 64, 80, 96, 128, 256])
            n = 1 if rng.random() < 0.4 else _log(rng, 2, 6000)
            start = 0 if rng.random() < 0.3 else _log(rng, 1, 4000)
            if 3072 not in (n, start) and B * n * Hkv * D <= 16 * 4096 * 8 * 128 and B * (n + start + 256) * Hkv * D <= 1 << 30:
                break
        return {"op": op, "B": B, "n": n, "start": start, "Hkv": Hkv, "D": D, "T": rng.choice([16, 32, 64, 128]),
                "dtype": rng.choice(["bf16", "f16", "f32"])}
    while True:
        B, Hkv, group = _log(rng, 1, 96), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 5, 8])
        D = rng.choice([32, 64, 80, 96, 128, 128, 256])
        q = 1 if rng.random() < 0.5 else _log(rng, 2, 2500)
        length = max(q, _log(rng, 1, 60000))
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        causal = rng.random() < 0.8
        window = _log(rng, 16, 4000) if causal and rng.random() < 0.25 else 0
        pairs = B * q * length * Hkv * group * D
        if (3072 not in (q, length, window) and pairs <= 4 * 2048 * 4096 * 32 * 128 // (4 if dtype == "f32" else 1)
                and B * length * Hkv * D <= 56 * 8192 * 8 * 128 and B * q * length * Hkv * group <= 4 * 2048 * 4096 * 32):
            break
    return {"op": op, "B": B, "q": q, "len": length, "Hq": Hkv * group, "Hkv": Hkv, "D": D, "T": rng.choice([16, 32, 64, 128]),
            "dtype": dtype, "causal": causal, "window": window, "empty": B > 1 and rng.random() < 0.3}


def _ragged(most, least, B):
    """B numbers from least to most, the first the largest, spread evenly and in no order."""
    return [most - int((most - least) * math.modf(b * 0.6180339887)[0]) for b in range(B)]


def _append_counts(case):
    """(new tokens, tokens before) of every sequence."""
    B = case["B"]
    return _ragged(case["n"], max(1, case["n"] // 3), B), _ragged(case["start"], case["start"] // 2, B)


def _attention_counts(case):
    """(queries, cached tokens with theirs) of every sequence."""
    B = case["B"]
    q = _ragged(case["q"], max(1, case["q"] // 3), B)
    lens = [max(n, v) for n, v in zip(q, _ragged(case["len"], max(1, case["len"] // 4), B))]
    if case["empty"]:
        lens[-1] = 0
    return q, lens


# ------------------------------------------------------------------------------------------------ inputs
def _cumulative(counts):
    return torch.tensor([0] + counts).cumsum(0).to(torch.int32).to(DEVICE)


def _pages(case, g, tokens, spare):
    """A page table [B, pages of the longest sequence] over a pool in no order, and the pool's size with `spare` unused pages at its end."""
    T = case["T"]
    need = [-(-n // T) for n in tokens]
    most, total = max(max(need), 1), max(sum(need), 1)
    ids = torch.randperm(total, generator=g, device=DEVICE).to(torch.int32)
    table = torch.zeros(len(need), most, dtype=torch.int32, device=DEVICE)
    counts = torch.tensor(need, device=DEVICE)
    inside = torch.arange(most, device=DEVICE)[None, :] < counts[:, None]
    table[inside] = ids[: sum(need)]
    return table, total + spare


def _codes(shape, g):
    """8-bit codes as a quantiser leaves them: a bell, its widest at the ends."""
    out = torch.empty(shape, dtype=torch.int8, device=DEVICE)
    flat = out.view(-1)
    step = 1 << 27
    for at in range(0, flat.numel(), step):
        part = flat[at:at + step]
        part.copy_((torch.randn(part.numel(), generator=g, device=DEVICE) * 32).round_().clamp_(-127, 127))
    return out


def _scales(shape, g):
    return torch.exp(torch.randn(shape, generator=g, device=DEVICE) * 0.3) / 32


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    rand = lambda *shape: torch.randn(shape, generator=g, device=DEVICE)  # noqa: E731
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        x = rand(M, K) * torch.exp(rand(K) * 0.5) * torch.exp(rand(M, 1) * 0.3)  # some channels are louder than others
        s = {"case": case, "x": x.to(dtype), "w": _codes((N, K), g), "s_w": _scales((N,), g) / math.sqrt(K),
             "bias": rand(N) if case["bias"] else None, "y": torch.empty(M, N, dtype=dtype, device=DEVICE)}
    elif case["op"] == "append":
        n, start = _append_counts(case)
        H, D, T = case["Hkv"], case["D"], case["T"]
        table, pages = _pages(case, g, [a + b for a, b in zip(n, start)], 1)
        loud = torch.exp(rand(H, D) * 0.5)
        first = [v // T * T for v in start]
        back = [a + b - f for a, b, f in zip(n, start, first)]  # tokens of the touched pages
        s = {"case": case, "k": (rand(sum(n), H, D) * loud).to(dtype), "v": rand(sum(n), H, D).to(dtype),
             "cache": (_codes((pages, H, T, D), g), _codes((pages, H, T, D), g), _scales((pages, H), g), _scales((pages, H), g)),
             "table": table, "cu": _cumulative(n), "start": torch.tensor(start, dtype=torch.int32, device=DEVICE),
             "back_cu": _cumulative(back), "back_start": torch.tensor(first, dtype=torch.int32, device=DEVICE),
             "back_most": max(back), "back_total": sum(back),
             "k_back": torch.empty(sum(back), H, D, dtype=dtype, device=DEVICE),
             "v_back": torch.empty(sum(back), H, D, dtype=dtype, device=DEVICE)}
    else:
        q, lens = _attention_counts(case)
        H, D, T = case["Hkv"], case["D"], case["T"]
        table, pages = _pages(case, g, lens, 0)
        s = {"case": case, "q": rand(sum(q), case["Hq"], D).to(dtype), "o": torch.empty(sum(q), case["Hq"], D, dtype=dtype, device=DEVICE),
             "cache": (_codes((pages, H, T, D), g), _codes((pages, H, T, D), g), _scales((pages, H), g), _scales((pages, H), g)),
             "table": table, "cu": _cumulative(q), "lens": torch.tensor(lens, dtype=torch.int32, device=DEVICE),
             "max_q": max(q), "max_len": max(lens), "total_q": sum(q)}
    if own:
        s["plan"] = _plan(s)
    return s


# ------------------------------------------------------------------------------------------------ the package's calls
def _plan(s):
    """The descriptors and workspaces that a program makes once and keeps."""
    from paper_2208_01944_gb300 import binding as B

    case = s["case"]
    scratch = lambda n: torch.empty(max(1, n), dtype=torch.uint8, device=DEVICE)  # noqa: E731
    if case["op"] == "linear":
        d = B.linear_desc(s["x"], s["w"], s["y"])
        return d, scratch(B.palquant_linear_q8_scratch_bytes(d))
    cache = B.kv8_cache(*s["cache"])
    if case["op"] == "append":
        return (cache, B.kv8_tokens(s["k"], s["v"], s["cu"], s["start"], s["table"], case["n"]),
                B.kv8_tokens(s["k_back"], s["v_back"], s["back_cu"], s["back_start"], s["table"], s["back_most"]))
    a = B.kv8_attn(s["q"], s["o"], s["cu"], s["lens"], s["table"], s["max_q"], s["max_len"], scale=case["D"] ** -0.5,
                   causal=case["causal"], window=case["window"])
    return cache, a, scratch(B.palquant_kv8_attention_scratch_bytes(cache, a))


def _run_own(s):
    from paper_2208_01944_gb300 import binding as B

    op = s["case"]["op"]
    if op == "linear":
        d, scratch = s["plan"]
        B.palquant_linear_q8(s["x"], s["w"], s["s_w"], s["bias"], s["y"], d, scratch, scratch.numel())
        return s["y"]
    if op == "append":
        cache, new, back = s["plan"]
        B.palquant_kv8_append(cache, s["k"], s["v"], new)
        B.palquant_kv8_read(cache, s["k_back"], s["v_back"], back)
        return {"k": s["k_back"], "v": s["v_back"], "k_scales": s["cache"][2], "v_scales": s["cache"][3]}
    cache, a, scratch = s["plan"]
    B.palquant_kv8_attention(cache, s["q"], s["o"], a, scratch, scratch.numel())
    return s["o"]


# ------------------------------------------------------------------------------------------------ plain forms
def _inverse(scale):
    return torch.where(scale > 0, 1.0 / scale, torch.zeros_like(scale))


def _linear_plain(s):
    x = s["x"].float()
    s_x = x.abs().amax(1, keepdim=True) * INV127
    q = (x * _inverse(s_x)).round().clamp(-127, 127)
    y = (q @ s["w"].float().t()) * s_x * s["s_w"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(s["x"].dtype)


def _append_side(s, x, codes, scales, page, new, old, row):
    """One side (keys or values): the touched pages [B, pages, H, T, D] quantised anew and written back."""
    new, old = new[:, :, None, :, None], old[:, :, None, :, None]
    fresh = torch.where(new, x.float()[row].permute(0, 1, 3, 2, 4), 0.0)
    was = torch.where(old.any(3), scales[page][..., None], 0.0)
    scale = torch.maximum(was, fresh.abs().amax((3, 4))[..., None] * INV127)
    inverse = _inverse(scale)
    kept = codes[page]
    again = (kept.float() * (was * inverse)[..., None]).round().clamp(-127, 127)
    fresh = (fresh * inverse[..., None]).round().clamp(-127, 127)
    codes[page] = torch.where(new, fresh, torch.where(old, again, kept.float())).to(torch.int8)
    scales[page] = scale[..., 0]


def _append_plain(s):
    case, table = s["case"], s["table"].long()
    T, B = case["T"], case["B"]
    k_codes, v_codes, k_scales, v_scales = s["cache"]
    start, cu = s["start"].long(), s["cu"].long()
    count = cu[1:] - cu[:-1]
    most = (case["n"] + T - 2) // T + 1
    block = start[:, None] // T + torch.arange(most, device=DEVICE)
    at = block[..., None] * T + torch.arange(T, device=DEVICE)
    i = at - start[:, None, None]
    new, old = (i >= 0) & (i < count[:, None, None]), i < 0
    row = (cu[:-1, None, None] + i).clamp(0, s["k"].shape[0] - 1)
    # pages that a shorter sequence does not touch stand for the spare one at the pool's end
    page = torch.where(new.any(2), table.gather(1, block.clamp(max=table.shape[1] - 1)), k_scales.shape[0] - 1)
    spare = [t[-1].clone() for t in s["cache"]]
    _append_side(s, s["k"], k_codes, k_scales, page, new, old, row)
    _append_side(s, s["v"], v_codes, v_scales, page, new, old, row)
    for t, was in zip(s["cache"], spare):
        t[-1] = was
    back = s["back_cu"].long()
    b = torch.repeat_interleave(torch.arange(B, device=DEVICE), back[1:] - back[:-1], output_size=s["back_total"])
    pos = torch.arange(s["back_total"], device=DEVICE) - back[:-1][b] + s["back_start"].long()[b]
    page, slot = table[b, pos // T], pos % T
    value = lambda codes, scales: (codes[page, :, slot].float() * scales[page][..., None]).to(s["k"].dtype)  # noqa: E731
    return {"k": value(k_codes, k_scales), "v": value(v_codes, v_scales), "k_scales": k_scales, "v_scales": v_scales}


def _attention_plain(s):
    case, table = s["case"], s["table"].long()
    B, H, D, T = case["B"], case["Hkv"], case["D"], case["T"]
    group, Q = case["Hq"] // H, s["max_q"]
    k_codes, v_codes, k_scales, v_scales = s["cache"]
    L = table.shape[1] * T
    value = lambda codes, scales: (codes[table].float() * scales[table][..., None, None]).transpose(1, 2).reshape(B, H, L, D)  # noqa: E731
    cu, lens = s["cu"].long(), s["lens"].long()
    count = cu[1:] - cu[:-1]
    i = torch.arange(Q, device=DEVICE)
    row = (cu[:-1, None] + i).clamp(max=s["total_q"] - 1)
    q = s["q"].float()[row].view(B, Q, H, group, D).permute(0, 2, 3, 1, 4).reshape(B, H, group * Q, D)
    score = (q @ value(k_codes, k_scales).transpose(2, 3)).view(B, H, group, Q, L) * D ** -0.5
    j = torch.arange(L, device=DEVICE)
    seen = (j < lens[:, None, None]).expand(B, Q, L)
    if case["causal"]:
        at = (lens - count)[:, None] + i
        seen = seen & (j <= at[..., None])
        if case["window"]:
            seen = seen & (j > at[..., None] - case["window"])
    seen = seen[:, None, None]
    score = score.masked_fill(~seen, float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == float("-inf"), 0.0, top))
    del score
    total = p.sum(-1, keepdim=True)
    v = value(v_codes, v_scales)
    v = torch.where((j < lens[:, None])[:, None, :, None], v, 0.0)
    o = (p.view(B, H, group * Q, L) @ v).view(B, H, group, Q, D) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(B * Q, case["Hq"], D)
    b = torch.repeat_interleave(torch.arange(B, device=DEVICE), count, output_size=s["total_q"])
    return o[b * Q + torch.arange(s["total_q"], device=DEVICE) - cu[:-1][b]].to(s["q"].dtype)


def run(state):
    if own:
        return _run_own(state)
    return {"linear": _linear_plain, "append": _append_plain, "attention": _attention_plain}[state["case"]["op"]](state)


# ------------------------------------------------------------------------------------------------ 64 bits
def _rounded(v):
    """What the definition keeps in 32 bits (scales, their inverses, the product that is rounded to a code)."""
    return v.float().double()


def _exact_codes(v, scale):
    """Codes of `v`: the 32-bit product with the scale's 32-bit inverse, to the nearest whole number, half to even."""
    inverse = torch.where(scale > 0, _rounded(1.0 / scale), 0.0)
    return torch.round(_rounded(v * inverse)).clamp(-127, 127)


def _exact_linear(s):
    x = s["x"].double()
    out = torch.empty(x.shape[0], s["w"].shape[0], dtype=torch.float64, device=DEVICE)
    w = s["w"].double().t().contiguous()
    for at in range(0, x.shape[0], 1024):
        rows = x[at:at + 1024]
        scale = _rounded(rows.abs().max(1).values * INV127)[:, None]
        out[at:at + 1024] = torch.mm(_exact_codes(rows, scale), w) * scale * s["s_w"].double()[None]
    return out if s["bias"] is None else out + s["bias"].double()


def _exact_append(s):
    T, table = s["case"]["T"], s["table"].cpu().tolist()
    cu, starts = s["cu"].cpu().tolist(), s["start"].cpu().tolist()
    found = {}
    for side, x, codes, scales in (("k", s["k"], s["cache"][0], s["cache"][2]), ("v", s["v"], s["cache"][1], s["cache"][3])):
        scales, values = scales.double(), []
        for b, start in enumerate(starts):
            end = start + cu[b + 1] - cu[b]
            for block in range(start // T, -(-end // T)):
                lo, hi = max(start, block * T), min(end, block * T + T)
                page, n_old = table[b][block], lo - block * T
                new = x[cu[b] + lo - start:cu[b] + hi - start].double().transpose(0, 1)  # [H, tokens, D]
                scale = _rounded(new.abs().amax((1, 2)) * INV127)
                was = scales[page].clone()
                if n_old:
                    scale = torch.maximum(scale, was)
                parts = []
                if n_old:
                    inverse = torch.where(scale > 0, _rounded(1.0 / scale), 0.0)
                    ratio = _rounded(was * inverse)[:, None, None]
                    parts.append(torch.round(_rounded(codes[page, :, :n_old].double() * ratio)).clamp(-127, 127))
                parts.append(_exact_codes(new, scale[:, None, None]))
                scales[page] = scale
                values.append((torch.cat(parts, 1) * scale[:, None, None]).transpose(0, 1))
        found[side], found[side + "_scales"] = torch.cat(values), scales
    return {name: found[name] for name in ("k", "v", "k_scales", "v_scales")}


def _exact_attention(s):
    case, table = s["case"], s["table"].long()
    H, D, T, group = case["Hkv"], case["D"], case["T"], case["Hq"] // case["Hkv"]
    cu, lens = s["cu"].cpu().tolist(), s["lens"].cpu().tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    for b, length in enumerate(lens):
        n = cu[b + 1] - cu[b]
        if not length:
            continue
        pages = table[b, : -(-length // T)]
        for h in range(H):
            k = (s["cache"][0][pages, h].double() * s["cache"][2][pages, h].double()[:, None, None]).reshape(-1, D)[:length]
            v = (s["cache"][1][pages, h].double() * s["cache"][3][pages, h].double()[:, None, None]).reshape(-1, D)[:length]
            for at in range(0, n, 256):
                m = min(256, n - at)
                rows = slice(cu[b] + at, cu[b] + at + m)
                q = s["q"][rows, h * group:(h + 1) * group].double().reshape(m * group, D)
                score = q @ k.t() / math.sqrt(D)
                if case["causal"]:
                    place = length - n + at + torch.arange(m, device=DEVICE).repeat_interleave(group)[:, None]
                    key = torch.arange(length, device=DEVICE)[None]
                    score[(key > place) | ((key <= place - case["window"]) if case["window"] else torch.zeros_like(key > place))] = -math.inf
                out[rows, h * group:(h + 1) * group] = (torch.softmax(score, 1) @ v).view(m, group, D)
    return out


def exact(case, seed):
    """The definition in 64 bits.  A causal query always sees its own token here, so no row of a sequence that has tokens is empty."""
    if case["op"] == "attention" and work(case)["flops"] > 4e12:
        return None
    s = prepare(case, seed)
    return {"linear": _exact_linear, "append": _exact_append, "attention": _exact_attention}[case["op"]](s)


# ------------------------------------------------------------------------------------------------ work
def work(case):
    e = BYTES[case["dtype"]]
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K * e + N * K + 4 * N * (2 if case["bias"] else 1) + M * N * e, "flops": 2 * M * N * K}
    H, D, T = case["Hkv"], case["D"], case["T"]
    if case["op"] == "append":
        n, start = _append_counts(case)
        new = sum(n) * H * D
        old = sum(v % T for v in start) * H * D
        back = new + old  # values read back; codes written and read; new tokens read
        pages = sum(-(-(a + b) // T) - b // T for a, b in zip(n, start)) * H
        return {"bytes": 2 * (new * e + (new + old) + back * (1 + e)) + 4 * 2 * pages, "flops": 2 * 3 * back}
    q, lens = _attention_counts(case)
    pairs = read = 0
    for n, length in zip(q, lens):
        if not length:
            continue
        if not case["causal"]:
            pairs, read = pairs + n * length, read + length
            continue
        window = case["window"] or length
        whole = [min(window, length - n + i + 1) for i in (0, n - 1)]
        grow = max(0, min(n, window - (length - n)))  # queries that the window does not cut
        pairs += grow * whole[0] + grow * (grow - 1) // 2 + (n - grow) * window if grow else n * window
        read += min(length, window + n - 1)
    return {"bytes": 2 * sum(q) * case["Hq"] * D * e + 2 * read * H * D + 8 * -(-read // T) * H,
            "flops": 4 * pairs * case["Hq"] * D}
