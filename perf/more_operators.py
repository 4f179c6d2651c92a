"""Cases of a drafter's attention: queries and keys on their way into it, a cache held in 4 bits, and
attention over that cache and over whole prompts.

Four calls of a drafting or serving step, each measured by itself:
  rope    norms of queries and keys for each head, and the rotation by their positions, in one pass
  append  keys and values into the 4-bit cache, and read back from it as the values it then holds
  cached  attention over the 4-bit cache: single tokens, the nodes of a draft tree, many sequences
  prompt  causal attention over whole prompts of different lengths, packed one behind the other

The cache holds a token's keys and values of a head as 4-bit floats (sign, two exponent bits, one
mantissa bit) with a power of two for every 32 of them, in pages of tokens.

Where `own` is false the operators are computed in their plain form, in 32 bits with elementary torch
operations (angles of far positions in 64); where it is true by the package's kernels.  `exact` gives
the results in 64 bits.
"""
import math
import random

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]
_LARGEST_SCALE = {"bf16": 125, "f16": 13, "f32": 125}          # 6 * 2^e stays finite in the type
_EPS = 1e-6


def _rope(name, dtype, T, heads, kv_heads, D, rot, norm, interleaved, start):
    return {"name": name, "op": "rope", "dtype": dtype, "T": T, "heads": heads, "kv_heads": kv_heads, "D": D, "rot": rot,
            "norm": norm, "interleaved": interleaved, "start": start}


def _append(name, dtype, T, kv_heads, D, page, pages):
    return {"name": name, "op": "append", "dtype": dtype, "T": T, "kv_heads": kv_heads, "D": D, "page": page, "pages": pages}


def _cached(name, dtype, S, rows, tree, heads, kv_heads, D, page, length, ragged):
    return {"name": name, "op": "cached", "dtype": dtype, "S": S, "rows": rows, "tree": tree, "heads": heads,
            "kv_heads": kv_heads, "D": D, "page": page, "length": length, "ragged": ragged}


def _prompt(name, dtype, S, T, before, heads, kv_heads, D):
    return {"name": name, "op": "prompt", "dtype": dtype, "S": S, "T": T, "before": before, "heads": heads,
            "kv_heads": kv_heads, "D": D}


def listed():
    return [
        # One token of chain drafting at the Llama3-8B head layout, with norms of the heads: latency.
        _rope("rope_m1", "bf16", 1, 32, 8, 128, 128, True, False, 2000),
        # A prompt of 8192 tokens far behind in a long context, no norms: bandwidth.
        _rope("rope_prompt", "bf16", 8192, 32, 8, 128, 128, False, False, 120000),
        # Odd sizes, full precision, a part of the head rotated, neighbours as pairs.
        _rope("rope_ragged_f32", "f32", 777, 14, 2, 64, 32, True, True, 0),
        # A serving batch's newest tokens, small pages.
        _append("append_m64", "bf16", 64, 8, 128, 16, 4096),
        # A prompt at the Qwen2.5-7B head layout, fp16.
        _append("append_prompt", "f16", 8192, 4, 128, 64, 256),
        # Chain drafting: one token, 2 K of context.
        _cached("cached_m1", "bf16", 1, 1, False, 32, 8, 128, 64, 2000, False),
        # Every node of a draft tree at once at the Qwen2.5-7B layout (seven heads share one of keys), fp16, small pages.
        _cached("cached_tree", "f16", 1, 60, True, 28, 4, 128, 16, 4111, False),
        # 64 sequences of up to 8192 tokens, one token each: the common serving step.
        _cached("cached_serve", "bf16", 64, 1, False, 32, 8, 128, 64, 8192, True),
        # A tree level of eight nodes over a very long context.
        _cached("cached_long", "bf16", 1, 8, True, 32, 8, 128, 128, 131072, False),
        # A short prompt: latency.
        _prompt("prompt_short", "bf16", 1, 300, 0, 32, 8, 128),
        # Twelve prompts of odd lengths in one call, fp16.
        _prompt("prompt_packed", "f16", 12, 8191, 0, 28, 4, 128),
        # One long prompt, every head its own keys (the Llama2-7B layout): the most work.
        _prompt("prompt_long", "bf16", 1, 8192, 0, 32, 32, 128),
    ]


_LAYOUTS = [(32, 8, 128), (32, 8, 128), (32, 32, 128), (28, 4, 128), (14, 2, 64), (12, 12, 64), (9, 3, 64), (8, 1, 256), (8, 4, 256)]


def _log_between(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    """1 to 16384 tokens to rotate or to append, 1 to 128 sequences with 1 to 64 rows each and up to 131072
    cached tokens, prompts of up to 8192 tokens in all; heads of 64 to 256 values; no more work than
    the largest listed case."""
    most = {n: max(work(c)[n] for c in listed()) for n in ("bytes", "flops")}
    while True:
        op = rng.choice(["rope", "append", "cached", "cached", "prompt", "prompt"])
        heads, kv_heads, D = rng.choice(_LAYOUTS)
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if op == "rope":
            case = _rope("", dtype, _log_between(rng, 1, 16384), heads, kv_heads, D, rng.choice([D, D, D // 2, 2 * (D // 6)]),
                         rng.random() < 0.5, rng.random() < 0.3, rng.choice([0, 5000, 1000000]))
        elif op == "append":
            page, T = rng.choice([16, 32, 64, 128, 256]), _log_between(rng, 1, 16384)
            case = _append("", dtype, T, kv_heads, D, page, -(-T * rng.choice([1, 2, 5]) // page) + rng.choice([0, 7]))
        elif op == "cached":
            S, length = _log_between(rng, 1, 128), _log_between(rng, 1, 131072)
            rows = rng.choice([1, 1, 1, _log_between(rng, 1, 64)])
            case = _cached("", dtype, S, rows, rng.random() < 0.5, heads, kv_heads, D, rng.choice([16, 32, 64, 128, 256]),
                           max(length, rows), rng.random() < 0.6)
            if S * length > 64 * 8192 or S * rows * heads * length > 1 << 28:
                continue                                         # what the plain form can hold
        else:
            T = _log_between(rng, 1, 8192)
            case = _prompt("", dtype, min(T, _log_between(rng, 1, 40)), T, rng.choice([0, 0, _log_between(rng, 1, 1000)]), heads, kv_heads, D)
        del case["name"]
        w = work(case)
        if all(w[n] <= most[n] for n in most):
            return case


# ---------------------------------------------------------------- lengths that follow from a case alone
def _parts(total, n, salt):
    """n whole numbers of at least one that sum to total, of very different sizes."""
    rng = random.Random(total * 1009 + n * 31 + salt)
    cuts = sorted(rng.sample(range(1, total), n - 1)) if n > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def _cached_lengths(case):
    """(cached tokens, rows) of each sequence; the rows are the newest of its tokens."""
    rng = random.Random(case["S"] * 7919 + case["length"])
    rows = [rng.randint(1, case["rows"]) if case["ragged"] else case["rows"] for _ in range(case["S"])]
    return [(max(r, rng.randint(1, case["length"])) if case["ragged"] and s else case["length"], r) for s, r in enumerate(rows)]


def _prompt_lengths(case):
    """(rows, keys) of each sequence: `before` keys and more where a prompt goes on behind what is there."""
    rows = _parts(case["T"], case["S"], 5)
    return [(n, n + case["before"] * (1 + s) // case["S"]) for s, n in enumerate(rows)]


# ---------------------------------------------------------------- the 4-bit floats
def _quantise(x, dtype):
    """(codes, exponents) of x [..., D] in 32 bits: codes 0..15 [..., D], one exponent for every 32 values."""
    u = x.float().reshape(*x.shape[:-1], -1, 32)
    m, e = torch.frexp(u.abs().amax(dim=-1))
    e = torch.where(m > 0.875, e - 2, e - 3).clamp(-126, _LARGEST_SCALE[dtype])      # the largest is 3.5 to 7 of them
    e = torch.where(m > 0, e, torch.full_like(e, -126))
    u = u * torch.exp2(-e.float())[..., None]
    a = u.abs()
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)    # ties to even codes
    return (code + 8 * (u < 0)).reshape(x.shape), e


def _held(codes, exponents):
    """The values of codes [..., D/2] bytes with scales [..., D/32] bytes, in 32 bits."""
    code = torch.stack([codes & 15, codes >> 4], dim=-1).reshape(*codes.shape[:-1], -1)
    value = torch.tensor(_E2M1, device="cuda")[code.int()]
    scale = torch.exp2(exponents.float() - 127.0)
    return (value.reshape(*exponents.shape, 32) * scale[..., None]).reshape(code.shape)


def _packed(code):
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)


# ---------------------------------------------------------------- inputs
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda")


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _running(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _rope_inputs(case, gen):
    T, heads, kv_heads, D, dt = case["T"], case["heads"], case["kv_heads"], case["D"], _TORCH[case["dtype"]]
    qkv = _normal(gen, T, heads + 2 * kv_heads, D).to(dt)                            # what one projection leaves
    s = {"q": qkv[:, :heads], "k": qkv[:, heads:heads + kv_heads], "q_weight": None, "k_weight": None,
         "positions": case["start"] + torch.arange(T, device="cuda", dtype=torch.int32),
         "inv_freq": torch.pow(500000.0, -torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"]).float()}
    if case["norm"]:
        s["q_weight"], s["k_weight"] = ((1.0 + 0.3 * _normal(gen, D)).to(dt) for _ in range(2))
    return s


def _append_inputs(case, gen):
    T, kv_heads, D, page, pages, dt = (case[n] for n in ("T", "kv_heads", "D", "page", "pages", "dtype"))
    spread = torch.exp(_normal(gen, 1, kv_heads, D) * 0.5)                           # some channels of keys are large
    qkv = _normal(gen, T, 2 * kv_heads, D)
    qkv[:, :kv_heads] *= spread
    qkv = qkv.to(_TORCH[dt])
    made = [torch.randint(0, 256, (pages, kv_heads, page, n), generator=gen, device="cuda", dtype=torch.uint8) for n in (D // 2, D // 32) * 2]
    order = torch.randperm(pages * page // 16, generator=gen, device="cuda")[:-(-T // 16)]        # runs of 16 places
    slots = (order[:, None] * 16 + torch.arange(16, device="cuda")).reshape(-1)[:T].int()
    return {"k": qkv[:, :kv_heads], "v": qkv[:, kv_heads:], "cache": tuple(made), "slots": slots}


def _cached_inputs(case, gen):
    heads, kv_heads, D, page, dt = (case[n] for n in ("heads", "kv_heads", "D", "page", "dtype"))
    lengths = _cached_lengths(case)
    held = [-(-n // page) for n, _ in lengths]
    pages, rows = sum(held), [r for _, r in lengths]
    cache = []
    for _ in range(2):
        code, e = _quantise(_normal(gen, pages, kv_heads, page, D), "bf16")
        cache += [_packed(code), (e + 127).to(torch.uint8)]
        del code, e
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.full((len(lengths), max(held)), -1, dtype=torch.int32, device="cuda")
    at = _running(held)
    for s, n in enumerate(held):
        table[s, :n] = order[at[s]:at[s + 1]]
    s = {"q": (_normal(gen, sum(rows), heads, D) * 1.5).to(_TORCH[dt]), "cache": tuple(cache), "page_table": table,
         "lengths": _int32([n for n, _ in lengths]), "offsets": _int32(_running(rows)), "max_rows": max(rows),
         "max_length": max(n for n, _ in lengths), "history": None, "tree": None}
    if case["tree"]:                                             # every node sees its ancestors and itself
        rng, words = random.Random(int(torch.randint(0, 1 << 30, (1,), generator=gen, device="cuda"))), []
        for r in rows:
            seen = []
            for i in range(r):
                seen.append((1 << i) | (seen[rng.randrange(max(0, i - 12), i)] if i else 0))
            words += [w - (1 << 64) if w >> 63 else w for w in seen]
        s["tree"] = torch.tensor(words, dtype=torch.int64, device="cuda")
        s["history"] = _int32([n - r for n, r in lengths])
    return s


def _prompt_inputs(case, gen):
    heads, kv_heads, D, dt = case["heads"], case["kv_heads"], case["D"], _TORCH[case["dtype"]]
    lengths = _prompt_lengths(case)
    keys = sum(n for _, n in lengths)
    kv = _normal(gen, keys, 2 * kv_heads, D).to(dt)
    return {"q": (_normal(gen, case["T"], heads, D) * 1.5).to(dt), "k": kv[:, :kv_heads].contiguous(), "v": kv[:, kv_heads:],
            "offsets": _int32(_running([n for n, _ in lengths])),
            "k_offsets": _int32(_running([n for _, n in lengths])) if case["before"] else None}


_INPUTS = {"rope": _rope_inputs, "append": _append_inputs, "cached": _cached_inputs, "prompt": _prompt_inputs}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = _INPUTS[case["op"]](case, gen)
    s["case"] = case
    if case["op"] == "cached":
        s["workspace"] = torch.zeros(256 << 20, dtype=torch.uint8, device="cuda")   # a serving loop's scratch
    return s


# ---------------------------------------------------------------- plain forms
def _plain_rope_of(s, x, weight):
    case, y = s["case"], x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + _EPS) * weight.float()
    rot = case["rot"]
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if case["interleaved"] else (y[..., :rot // 2], y[..., rot // 2:rot])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], dim=-1).reshape(*y.shape[:-1], rot) if case["interleaved"] else torch.cat([a, b], dim=-1)
    return torch.cat([turned, y[..., rot:]], dim=-1).to(x.dtype)


def _plain_append(s):
    case, (k_codes, k_scales, v_codes, v_scales) = s["case"], s["cache"]
    slot = s["slots"].long()
    page, at = slot // case["page"], slot % case["page"]
    for x, codes, scales in ((s["k"], k_codes, k_scales), (s["v"], v_codes, v_scales)):
        code, e = _quantise(x, case["dtype"])
        codes[page, :, at] = _packed(code)
        scales[page, :, at] = (e + 127).to(torch.uint8)
    return tuple(_held(codes[page, :, at], scales[page, :, at]).to(s["k"].dtype)
                 for codes, scales in ((k_codes, k_scales), (v_codes, v_scales)))


def _softmax_product(score, seen, v):
    """softmax over the last axis of score where `seen`, times v; zero for a row that sees nothing."""
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(dim=-1, keepdim=True)
    p = torch.exp(score.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)))
    total = p.sum(dim=-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))


def _plain_cached(s):
    case, q, (k_codes, k_scales, v_codes, v_scales) = s["case"], s["q"], s["cache"]
    T, heads, D = q.shape
    S, kv_heads, page, R = s["page_table"].shape[0], case["kv_heads"], case["page"], s["max_rows"]
    table = s["page_table"].long().clamp(min=0)
    n_keys = table.shape[1] * page
    k, v = (_held(c[table], e[table]).transpose(1, 2).reshape(S, kv_heads, n_keys, D)
            for c, e in ((k_codes, k_scales), (v_codes, v_scales)))
    first, counts = s["offsets"][:-1].long(), (s["offsets"][1:] - s["offsets"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(S, device="cuda"), counts, output_size=T)
    row = torch.arange(T, device="cuda") - first[seq]
    padded = torch.zeros((S, R, heads, D), device="cuda")
    padded[seq, row] = q.float() / math.sqrt(D)
    padded = padded.reshape(S, R, kv_heads, -1, D).permute(0, 2, 3, 1, 4).reshape(S, kv_heads, -1, D)
    score = torch.matmul(padded, k.transpose(2, 3)).reshape(S, heads, R, n_keys)
    key, length = torch.arange(n_keys, device="cuda"), s["lengths"].long()
    if s["tree"] is None:
        seen_rows = key[None, :] <= (length[seq] - counts[seq] + row)[:, None]
    else:
        bit = key[None, :] - s["history"].long()[seq][:, None]
        seen_rows = (bit < 0) | ((bit < 64) & (((s["tree"][:, None] >> bit.clamp(0, 63)) & 1) == 1))
    seen = torch.zeros((S, R, n_keys), dtype=torch.bool, device="cuda")
    seen[seq, row] = seen_rows & (key[None, :] < length[seq][:, None])
    out = _softmax_product(score.reshape(S, kv_heads, -1, R, n_keys), seen[:, None, None], v[:, :, None]).reshape(S, heads, R, D)
    return out.transpose(1, 2)[seq, row].to(q.dtype)


def _plain_prompt(s):
    q, k, v = (s[n].float().transpose(0, 1) for n in ("q", "k", "v"))               # [heads, tokens, D]
    kv_heads, T, D, keys = k.shape[0], q.shape[1], q.shape[2], k.shape[1]
    offsets = s["offsets"].long()
    k_offsets = offsets if s["k_offsets"] is None else s["k_offsets"].long()
    S = offsets.numel() - 1
    at = torch.arange(S, device="cuda")
    seq = torch.repeat_interleave(at, offsets[1:] - offsets[:-1], output_size=T)
    key_seq = torch.repeat_interleave(at, k_offsets[1:] - k_offsets[:-1], output_size=keys)
    last = k_offsets[seq + 1] - offsets[seq + 1] + torch.arange(T, device="cuda")    # the newest key that a row sees
    seen = (seq[:, None] == key_seq) & (torch.arange(keys, device="cuda") <= last[:, None])
    q = (q / math.sqrt(D)).reshape(kv_heads, -1, D)
    score = torch.matmul(q, k.transpose(1, 2)).reshape(kv_heads, -1, T, keys)
    out = _softmax_product(score, seen, v[:, None])
    return out.reshape(-1, T, D).transpose(0, 1).to(s["q"].dtype).contiguous()


def run(s):
    case = s["case"]
    if own:
        import paper_2502_16880_amd as coral
        if case["op"] == "rope":
            return coral.coral_qk_norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], q_weight=s["q_weight"],
                                            k_weight=s["k_weight"], eps=_EPS, interleaved=case["interleaved"])
        if case["op"] == "append":
            coral.coral_kv4_append(s["cache"], s["k"], s["v"], s["slots"])
            return coral.coral_kv4_read(s["cache"], s["slots"], s["k"].dtype)
        if case["op"] == "cached":
            return coral.coral_attention_kv4(s["q"], s["cache"], s["page_table"], s["lengths"], s["offsets"], s["max_rows"],
                                             max_length=s["max_length"], history=s["history"], tree=s["tree"],
                                             workspace=s["workspace"])
        return coral.coral_attention_prompt(s["q"], s["k"], s["v"], s["offsets"], k_offsets=s["k_offsets"])
    if case["op"] == "rope":
        return _plain_rope_of(s, s["q"], s["q_weight"]), _plain_rope_of(s, s["k"], s["k_weight"])
    if case["op"] == "append":
        return _plain_append(s)
    return _plain_cached(s) if case["op"] == "cached" else _plain_prompt(s)


# ---------------------------------------------------------------- what is measured against
def work(case):
    """Every input and output once: heads before and after, codes with their scales, queries, keys,
    values and results; two products for every key that a row sees."""
    w, D = _BYTES[case["dtype"]], case["D"]
    if case["op"] == "rope":
        n = case["T"] * (case["heads"] + case["kv_heads"]) * D
        return {"bytes": 2 * n * w + case["T"] * 4 + (2 * D * w if case["norm"] else 0), "flops": 8.0 * n}
    if case["op"] == "append":
        n = 2 * case["T"] * case["kv_heads"] * D
        return {"bytes": 2 * n * w + 2 * n * (1 / 2 + 1 / 32) + case["T"] * 4, "flops": 4.0 * n}
    pairs = rows = keys = 0
    for n, m in (_prompt_lengths(case) if case["op"] == "prompt" else _cached_lengths(case)):
        if case["op"] == "cached":
            n, m = m, n
        pairs += n * m - n * (n - 1) // 2
        rows, keys = rows + n, keys + m
    b = 2 * rows * case["heads"] * D * w
    b += 2 * keys * case["kv_heads"] * D * (w if case["op"] == "prompt" else 1 / 2 + 1 / 32)
    return {"bytes": b, "flops": 4.0 * pairs * case["heads"] * D}


def _exact_rope(case, s):
    out = []
    for x, weight in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = x.double()
        if weight is not None:
            y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + _EPS) * weight.double()
        half = case["rot"] // 2
        index = torch.arange(half, device="cuda")
        first, second = (2 * index, 2 * index + 1) if case["interleaved"] else (index, index + half)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["inv_freq"].double())
        z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        out.append(y)
    return tuple(out)


def _exact_append(case, s):
    """The nearest 4-bit value for each number, the scale's exponent by the block's largest."""
    table = torch.tensor(sorted(set(_E2M1)), dtype=torch.float64, device="cuda")
    order = torch.tensor([0, 1, 2, 3, 4, 5, 6, 7], device="cuda")[(torch.arange(15, device="cuda") - 7).abs()]
    out = []
    for x in (s["k"], s["v"]):
        u = x.double().reshape(*x.shape[:-1], -1, 32)
        largest = u.abs().amax(-1, keepdim=True)
        low = torch.full_like(largest, 2.0 ** -126)
        scale = torch.maximum(torch.exp2(torch.floor(torch.log2(torch.maximum(largest, low))) - 2), low)
        scale = torch.where(largest > 7 * scale, 2 * scale, scale).clamp(max=2.0 ** _LARGEST_SCALE[case["dtype"]])
        parts = []
        for some in (u / scale).split(1024):
            off = (some[..., None] - table).abs()
            best = off.amin(-1, keepdim=True)
            parts.append(table[torch.where(off == best, order % 2 * 16 + torch.arange(15, device="cuda"), 99).argmin(-1)])
        out.append((torch.cat(parts) * scale).reshape(x.shape))
    return tuple(out)


def _exact_attention(q, k, v, last, seen=None):
    """One sequence's attention in 64 bits: q [n, heads, D], k and v [m, kv_heads, D]; row i sees keys up to last[i]."""
    group = q.shape[1] // k.shape[1]
    if seen is None:
        seen = torch.arange(k.shape[0], device="cuda") <= last[:, None]
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    for h in range(q.shape[1]):
        score = (q[:, h].double() @ k[:, h // group].double().t()) * q.shape[2] ** -0.5
        weight = torch.softmax(torch.where(seen, score, torch.full_like(score, -math.inf)), dim=-1)
        out[:, h] = weight @ v[:, h // group].double()
    return out


def _exact_cached(case, s):
    out, at = [], 0
    table = torch.tensor(_E2M1, dtype=torch.float64, device="cuda")
    for i, (n, r) in enumerate(_cached_lengths(case)):
        pages = s["page_table"][i, :-(-n // case["page"])].long()
        kv = []
        for codes, scales in (s["cache"][:2], s["cache"][2:]):
            c = codes[pages].transpose(1, 2).flatten(0, 1)[:n].int()
            e = scales[pages].transpose(1, 2).flatten(0, 1)[:n].double() - 127
            value = torch.empty((*c.shape[:-1], case["D"]), dtype=torch.float64, device="cuda")
            value[..., 0::2], value[..., 1::2] = table[c % 16], table[c // 16]
            kv.append(value * torch.pow(2.0, e).repeat_interleave(32, dim=-1))
        seen = torch.ones((r, n), dtype=torch.bool, device="cuda")
        newest = torch.tril(seen[:, :r])
        if s["tree"] is not None:
            words = s["tree"][at:at + r].tolist()
            newest = torch.tensor([[(w >> b) & 1 == 1 for b in range(r)] for w in words], device="cuda")
        seen[:, n - r:] = newest
        out.append(_exact_attention(s["q"][at:at + r], kv[0], kv[1], None, seen))
        at += r
    return torch.cat(out)


def _exact_prompt(case, s):
    out, at, k_at = [], 0, 0
    for n, m in _prompt_lengths(case):
        last = m - n + torch.arange(n, device="cuda")
        out.append(_exact_attention(s["q"][at:at + n], s["k"][k_at:k_at + m], s["v"][k_at:k_at + m], last))
        at, k_at = at + n, k_at + m
    return torch.cat(out)


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "append": _exact_append, "cached": _exact_cached, "prompt": _exact_prompt}[case["op"]](case, s)
