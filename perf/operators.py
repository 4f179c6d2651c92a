"""Cases of the operators around the LM head: products with 4-bit weights, and rules on logits.

Three calls of a drafting or serving step, each measured by itself:
  matvec  y = act(x W^T + bias) + residual, W in 4 bits with a scale (and a zero point) per group of
          columns: an LM head, the router's pre-mix and a drafter's projections, 1 to 64 tokens
  adjust  penalties for repeated tokens, biases and a grammar mask on a step's logits
  topk    the same rules, and each row's k best tokens with their log-probabilities, as tree
          expansion and sampling take them

Where `own` is false the operators are computed in their plain form, in 32 bits with elementary torch
operations; where it is true by the package's kernels.  `exact` gives the results in 64 bits.
"""
import math

import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]
_ROWS = 16384                       # weight rows multiplied in 64 bits at a time


def _matvec(name, dtype, M, N, K, group, codes, zeros, out, act="identity", bias=False, residual=False):
    return {"name": name, "op": "matvec", "dtype": dtype, "M": M, "N": N, "K": K, "group": group, "codes": codes,
            "zeros": zeros, "out": out, "act": act, "bias": bias, "residual": residual}


def _logits(name, op, dtype, M, V, k, prompt, output, shared, biases, allowed):
    return {"name": name, "op": op, "dtype": dtype, "M": M, "V": V, "k": k, "prompt": prompt, "output": output,
            "shared": shared, "biases": biases, "allowed": allowed}


def listed():
    return [
        # The router's pre-mix of a 4096-wide drafter, one token: a small square matrix, latency.
        _matvec("premix_m1", "bf16", 1, 4096, 4096, 128, "int", True, "bf16", act="silu", residual=True),
        # The LM head at the Llama3-8B shape in chain drafting: the commonest large product.
        _matvec("head_llama3_m1", "bf16", 1, 128256, 4096, 128, "int", False, "f32"),
        # The Qwen2.5-7B shape, a tree level of 16 nodes, fp16 and zero points.
        _matvec("head_qwen_f16_m16", "f16", 16, 152064, 3584, 64, "int", True, "f32"),
        # A wide tree or several sequences at once, 4-bit floats with fine groups: the most work.
        _matvec("head_e2m1_m64", "bf16", 64, 128256, 4096, 32, "e2m1", False, "f32"),
        # Odd sizes, activations in full precision, a bias.
        _matvec("ragged_f32_m7", "f32", 7, 50257, 2568, 32, "int", True, "f32", bias=True),
        # One sequence in chain drafting: 2 K tokens so far, a few biases, no grammar.
        _logits("adjust_m1", "adjust", "f32", 1, 128256, 0, 1500, 500, False, 16, 1.0),
        # A serving batch of 64 sequences with grammars, long prompts and odd rows.
        _logits("adjust_m64", "adjust", "bf16", 64, 151665, 0, 8000, 1000, False, 100, 0.3),
        # Chain drafting without any rule: the k best and their log-probabilities.
        _logits("topk_m1", "topk", "f32", 1, 128256, 10, 0, 0, False, 0, 1.0),
        # A tree level of eight nodes over one shared prompt, where a grammar leaves few tokens.
        _logits("topk_tree_m8", "topk", "f32", 8, 128256, 10, 4000, 300, True, 16, 0.002),
        # A serving batch with every rule, many candidates.
        _logits("topk_m64", "topk", "f32", 64, 152064, 64, 2000, 2000, False, 32, 0.5),
        # An odd vocabulary in 16 bits (equal values are common), 24 nodes, long shared context.
        _logits("topk_ragged_m24", "topk", "f16", 24, 50257, 20, 60000, 700, True, 0, 1.0),
    ]


def _log_between(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """Products of 256 to 14336 columns and 64 to 152 K rows, logits of 1000 to 152 K tokens, 1 to 64
    tokens a step; no more work than the largest listed case."""
    most = {n: max(work(c)[n] for c in listed()) for n in ("bytes", "flops")}
    while True:
        M = max(1, min(64, int(_log_between(rng, 1, 65))))
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        if rng.random() < 0.5:
            step = rng.choice([128, 128, 32, 8])
            K = max(256, int(_log_between(rng, 256, 14336) / step + 0.5) * step)
            N = int(_log_between(rng, 64, 152064))
            codes = rng.choice(["int", "int", "e2m1"])
            case = _matvec("", dtype, M, N, K, rng.choice([32, 64, 128, 128]), codes,
                           codes == "int" and rng.random() < 0.5, rng.choice(["f32", dtype]),
                           rng.choice(["identity", "identity", "silu", "relu"]), rng.random() < 0.3, rng.random() < 0.3)
        else:
            op = rng.choice(["adjust", "topk"])
            V = int(_log_between(rng, 1000, 152064))
            case = _logits("", op, dtype, M, V, rng.choice([1, 4, 10, 10, 20, 64]) if op == "topk" else 0,
                           int(_log_between(rng, 1, 40000)) - 1, int(_log_between(rng, 1, 4000)) - 1, rng.random() < 0.4,
                           rng.choice([0, 0, 3, 30, 300]), rng.choice([1.0, 1.0, 0.6, 0.05, 0.002]))
        del case["name"]
        w = work(case)
        if all(w[n] <= most[n] for n in most):
            return case


# ---------------------------------------------------------------- inputs
def _matvec_inputs(case, gen):
    M, N, K, dt = case["M"], case["N"], case["K"], _TORCH[case["dtype"]]
    groups = -(-K // case["group"])
    x = torch.randn((M, K), generator=gen, device="cuda")
    s = {"x": (x / x.square().mean(dim=1, keepdim=True).sqrt()).to(dt),          # what a norm leaves
         "codes": torch.randint(0, 256, (N, K // 2), generator=gen, device="cuda", dtype=torch.uint8),
         "zeros": None, "bias": None, "residual": None}
    # weights of about 0.02, as this repository's heads have them
    s["scales"] = ((0.5 + torch.rand((N, groups), generator=gen, device="cuda")) * 0.005).to(dt)
    if case["zeros"]:
        s["zeros"] = torch.randint(4, 12, (N, groups), generator=gen, device="cuda", dtype=torch.uint8)
    if case["bias"]:
        s["bias"] = torch.randn(N, generator=gen, device="cuda")
    if case["residual"]:
        s["residual"] = torch.randn((M, N), generator=gen, device="cuda").to(dt)
    return s


def _logits_inputs(case, gen):
    M, V, P, L, B = (case[n] for n in ("M", "V", "prompt", "output", "biases"))
    s = {"logits": (torch.randn((M, V), generator=gen, device="cuda") * 2.5).to(_TORCH[case["dtype"]]),
         "history": None, "ranges": None, "penalties": None, "bias_ids": None, "bias_values": None,
         "bias_ranges": None, "mask": None}
    row = torch.arange(M, device="cuda", dtype=torch.int32)
    if P + L > 0:
        prompts = 1 if case["shared"] else M                  # the nodes of one sequence share its prompt
        n = prompts * P + M * L
        # frequent tokens come again and again, as in text
        s["history"] = (torch.rand(n, generator=gen, device="cuda").pow(4) * V).int().clamp_(max=V - 1)
        at = row * 0 if case["shared"] else row * P
        s["ranges"] = torch.stack([at, at + P, prompts * P + row * L, prompts * P + row * L + L], dim=1).contiguous()
        s["penalties"] = torch.rand((M, 3), generator=gen, device="cuda") * 0.3 + torch.tensor([1.0, 0.0, 0.0], device="cuda")
    if B:
        first = torch.randint(0, V, (M, 1), generator=gen, device="cuda")
        s["bias_ids"] = ((first + torch.arange(B, device="cuda") * 3) % V).int().reshape(-1)      # each id once a row
        s["bias_values"] = torch.randn(M * B, generator=gen, device="cuda") * 4.0
        s["bias_ranges"] = torch.stack([row * B, row * B + B], dim=1).contiguous()
    if case["allowed"] < 1.0:
        words = -(-V // 32)
        keep = torch.rand((M, words, 32), generator=gen, device="cuda") < case["allowed"]
        s["mask"] = (keep.long() << torch.arange(32, device="cuda")).sum(dim=2).int()             # bit j of word w: id 32 w + j
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = _matvec_inputs(case, gen) if case["op"] == "matvec" else _logits_inputs(case, gen)
    s["case"] = case
    if case["op"] == "topk":
        s["workspace"] = torch.zeros(8 << 20, dtype=torch.uint8, device="cuda")                   # a serving loop's scratch
    return s


# ---------------------------------------------------------------- plain forms
def _plain_matvec(s):
    case, codes = s["case"], s["codes"]
    K, group = case["K"], case["group"]
    w = torch.stack([codes & 15, codes >> 4], dim=2).reshape(case["N"], K)       # column 2 j in the low half of byte j
    scale = s["scales"].float().repeat_interleave(group, dim=1)[:, :K]
    if case["codes"] == "e2m1":
        w = torch.tensor(_E2M1, device="cuda")[w.int()]
    elif s["zeros"] is not None:
        w = w.float() - s["zeros"].float().repeat_interleave(group, dim=1)[:, :K]
    else:
        w = w.float() - 8.0
    y = s["x"].float() @ (w * scale).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    if case["act"] == "silu":
        y = y / (1.0 + torch.exp(-y))
    elif case["act"] == "relu":
        y = torch.where(y > 0, y, torch.zeros_like(y))
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(_TORCH[case["out"]])


def _flat(begin, length, total):
    """Row, and place in the flat array, of the entries [begin, begin + length) of every row."""
    row = torch.repeat_interleave(torch.arange(begin.numel(), device="cuda"), length, output_size=total)
    first = torch.cumsum(length, 0) - length
    return row, begin[row] + torch.arange(total, device="cuda") - first[row]


def _plain_rules(s):
    """The logits under their rules, in 32 bits: repetition, frequency, presence, bias, mask."""
    case, z = s["case"], s["logits"].to(torch.float32, copy=True)
    M, V = z.shape
    if s["history"] is not None:
        r = s["ranges"].long()
        counts = torch.zeros((2, M, V), dtype=torch.int32, device="cuda")
        for which, n in ((0, case["prompt"]), (1, case["output"])):
            row, at = _flat(r[:, 2 * which], r[:, 2 * which + 1] - r[:, 2 * which], M * n)
            ones = torch.ones_like(row, dtype=torch.int32)
            counts[which].index_put_((row, s["history"][at].long()), ones, accumulate=True)
        rep, freq, pres = (s["penalties"][:, j:j + 1] for j in range(3))
        z = torch.where(counts.sum(dim=0) > 0, torch.where(z > 0, z / rep, z * rep), z)
        z = z - counts[1].float() * freq
        z = z - (counts[1] > 0).float() * pres
    if s["bias_ids"] is not None:
        r = s["bias_ranges"].long()
        row, at = _flat(r[:, 0], r[:, 1] - r[:, 0], M * case["biases"])
        ids = s["bias_ids"][at].long()
        z.index_put_((row, ids), z[row, ids] + s["bias_values"][at])
    if s["mask"] is not None:
        bits = (s["mask"][:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
        z = torch.where(bits.reshape(M, -1)[:, :V] == 1, z, torch.full_like(z, -math.inf))
    return z


def _plain_topk(s):
    z, k = _plain_rules(s), s["case"]["k"]
    top = z.max(dim=1, keepdim=True).values
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)              # a row that its mask leaves empty
    lse = torch.log(torch.exp(z - top).sum(dim=1, keepdim=True)) + top
    val, ids = torch.sort(z, dim=1, descending=True, stable=True)                # equal values: lower id first
    val, ids = val[:, :k], ids[:, :k].int()
    gone = torch.isinf(val)
    return torch.where(gone, torch.full_like(ids, -1), ids), torch.where(gone, val, val - lse)


def run(s):
    case = s["case"]
    if own:
        import paper_2502_16880_amd as coral
        if case["op"] == "matvec":
            return coral.coral_matvec_w4(s["x"], s["codes"], s["scales"], zeros=s["zeros"], group=case["group"],
                                         code_type=case["codes"], bias=s["bias"], residual=s["residual"], act=case["act"],
                                         out_dtype=_TORCH[case["out"]])
        rules = dict(history=s["history"], ranges=s["ranges"], penalties=s["penalties"], bias_ids=s["bias_ids"],
                     bias_values=s["bias_values"], bias_ranges=s["bias_ranges"], mask=s["mask"])
        if case["op"] == "adjust":
            return coral.coral_logits_adjust(s["logits"], **rules)
        return coral.coral_logits_topk(s["logits"], case["k"], workspace=s["workspace"], **rules)
    if case["op"] == "matvec":
        return _plain_matvec(s)
    if case["op"] == "adjust":
        return _plain_rules(s).to(_TORCH[case["dtype"]])
    return _plain_topk(s)


# ---------------------------------------------------------------- what is measured against
def work(case):
    """Every input and output once: the codes with their scales, the activations and results; the
    logits with the tokens, biases and mask bits that the rules read."""
    w, M = _BYTES[case["dtype"]], case["M"]
    if case["op"] == "matvec":
        N, K = case["N"], case["K"]
        groups = -(-K // case["group"])
        b = N * K / 2 + N * groups * (w + (1 if case["zeros"] else 0)) + M * K * w + M * N * _BYTES[case["out"]]
        return {"bytes": b + (4 * N if case["bias"] else 0) + (M * N * w if case["residual"] else 0), "flops": 2.0 * M * N * K}
    V = case["V"]
    b = M * V * w + 4 * ((1 if case["shared"] else M) * case["prompt"] + M * case["output"]) + 8 * M * case["biases"]
    b += M * -(-V // 32) * 4 if case["allowed"] < 1.0 else 0
    return {"bytes": b + (M * V * w if case["op"] == "adjust" else 8 * M * case["k"]), "flops": 4.0 * M * V}


def _exact_matvec(case, s):
    K, group = case["K"], case["group"]
    table = torch.tensor(_E2M1 if case["codes"] == "e2m1" else [float(v) for v in range(16)], dtype=torch.float64, device="cuda")
    x, parts = s["x"].double(), []
    for lo in range(0, case["N"], _ROWS):
        codes = s["codes"][lo:lo + _ROWS].int()
        value = torch.empty((codes.shape[0], K), dtype=torch.float64, device="cuda")
        value[:, 0::2] = table[codes % 16]
        value[:, 1::2] = table[torch.div(codes, 16, rounding_mode="floor")]
        column = torch.arange(K, device="cuda") // group
        if case["codes"] == "int":
            value -= 8.0 if s["zeros"] is None else s["zeros"][lo:lo + _ROWS].double()[:, column]
        value *= s["scales"][lo:lo + _ROWS].double()[:, column]
        parts.append(x @ value.t())
    y = torch.cat(parts, dim=1)
    if s["bias"] is not None:
        y += s["bias"].double()
    if case["act"] == "silu":
        y = y * torch.special.expit(y)
    elif case["act"] == "relu":
        y = y.clamp(min=0.0)
    return y if s["residual"] is None else y + s["residual"].double()


def _exact_row(case, s, m):
    """One row's logits under its rules in 64 bits."""
    z, V = s["logits"][m].double().clone(), case["V"]
    if s["history"] is not None:
        a, b, c, d = s["ranges"][m].tolist()
        prompt = torch.bincount(s["history"][a:b].long(), minlength=V)
        output = torch.bincount(s["history"][c:d].long(), minlength=V)
        rep, freq, pres = s["penalties"][m].double().tolist()
        seen = (prompt + output) > 0
        z[seen] = torch.where(z[seen] > 0, z[seen] / rep, z[seen] * rep)
        z -= freq * output.double() + pres * (output > 0).double()
    if s["bias_ids"] is not None:
        a, b = s["bias_ranges"][m].tolist()
        z[s["bias_ids"][a:b].long()] += s["bias_values"][a:b].double()
    if s["mask"] is not None:
        word = s["mask"][m].long() & 0xFFFFFFFF
        at = torch.arange(V, device="cuda")
        z[(torch.div(word[at // 32], 2 ** (at % 32), rounding_mode="floor") % 2) == 0] = -math.inf
    return z


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "matvec":
        return _exact_matvec(case, s)
    rows = torch.stack([_exact_row(case, s, m) for m in range(case["M"])])
    if case["op"] == "adjust":
        return rows
    best = torch.topk(rows, case["k"], dim=1).values
    return None, torch.where(torch.isinf(best), best, best - torch.logsumexp(rows, dim=1, keepdim=True))
