"""The 4-bit products and the rules on logits without a GPU: refusals of the C ABI and of the binding,
and the oracle against values worked out by hand and against torch."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2502_16880_amd as coral
from oracle import operators as plain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, GROUP_INDEX, UNSUPPORTED, WORKSPACE, HIP = range(7)
F32, BF16, F16 = 0, 1, 2
FAKE = 0x7000_0000_1000          # never dereferenced: every check below fails before a launch


def test_header_and_library_agree_on_names_with_digits():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "coral_lmhead.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(coral_[a-z0-9_]+)\s*\(", text))
    assert {"coral_matvec_w4", "coral_logits_adjust", "coral_logits_topk", "coral_logits_topk_workspace_bytes"} <= names
    lib = ctypes.CDLL(coral.LIB_PATH)
    assert all(hasattr(lib, n) for n in names)


# ---------------------------------------------------------------- which kernel a 4-bit product takes
PLAN = r"""
#include <cstdio>
#include <set>
#include <tuple>
#include "w4_plan.h"
int main() {
    std::set<std::tuple<int, int, int, int, int>> forms;
    for (int f32 = 0; f32 < 2; ++f32)
        for (int M = 1; M <= 64; ++M)
            for (int K = 8; K <= 1 << 20; K += 8) {
                const W4Plan p = w4_plan_held(M, K, f32 != 0);
                forms.insert({f32, p.t, p.nb, p.passes, p.spread});
            }
    for (auto [f32, t, nb, passes, spread] : forms) std::printf("form %d %d %d %d %d\n", f32, t, nb, passes, spread);
    int f32, M, N, K;
    while (std::scanf("%d %d %d %d", &f32, &M, &N, &K) == 4) {
        const W4Plan p = w4_plan_held(M, K, f32 != 0);
        const W4Grid g = w4_held_grid(p, M, N, f32 != 0);
        std::printf("call %d %d %d %d %d %d %d %d\n", w4_plan_rows(M, N, f32 != 0) ? 1 : 0, f32, p.t, p.nb, p.passes, p.spread, g.x, g.y);
    }
}
"""


def test_gpu_tests_reach_every_form_of_the_4_bit_products(tmp_path):
    """The rules (csrc/w4_plan.h) compiled for the host: every form of the kernel that some call takes is one of the GPU
    tests' calls, and the shapes meant for many rows, and for several blocks of tiles, are such."""
    import subprocess
    import test_gpu_operators as gpu
    (tmp_path / "plan.cpp").write_text(PLAN)
    exe = str(tmp_path / "plan")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2502_16880_amd", "csrc"), str(tmp_path / "plan.cpp"), "-o", exe], check=True)
    held = [(f32, M, 83, K) for f32 in (0, 1) for M, K in gpu.FORMS]
    passes = [(int(dtype == "f32"), M, N, K) for dtype, M, N, K in gpu.PASSES]
    rows = [(0, M, N, K) for M, N, K, _ in gpu.MANY_ROWS] + [(0, 50, N, 40) for N in gpu.INFINITE_ROWS]
    text = "\n".join(" ".join(map(str, c)) for c in held + passes + rows)
    out = [line.split() for line in subprocess.run([exe], input=text, check=True, capture_output=True, text=True).stdout.splitlines()]
    forms = {tuple(map(int, l[1:])) for l in out if l[0] == "form"}
    calls = [tuple(map(int, l[1:])) for l in out if l[0] == "call"]
    assert len(calls) == len(held) + len(passes) + len(rows) and len(forms) == 12 + 10
    assert {c[1:6] for c in calls[:len(held)]} == forms and not any(c[0] for c in calls[:len(held)])
    for (_, M, N, K), c in zip(passes, calls[len(held):]):
        assert c[0] == 0 and c[4] == 1 and -(-N // 16) > 24 * c[6] and c[7] == 1       # a block is 24 tiles at most
    assert all(c[0] == 1 for c in calls[len(held) + len(passes):])


# ---------------------------------------------------------------- refusals
def matvec(**kw):
    a = dict(x=FAKE, codes=FAKE + (1 << 30), scales=FAKE + (2 << 30), zeros=None, bias=None, residual=None, M=4, N=64, K=256,
             group=128, code=0, dt=BF16, act=2, out=F32, y=FAKE + (3 << 30))
    a.update(kw)
    return coral._L.coral_matvec_w4(*(a[n] for n in ("x", "codes", "scales", "zeros", "bias", "residual", "M", "N", "K", "group",
                                                     "code", "dt", "act", "out", "y")), None)


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(y=None), NULL),
    (dict(dt=3), SHAPE), (dict(act=3), SHAPE), (dict(code=2), SHAPE), (dict(out=F16), SHAPE), (dict(out=7), SHAPE),
    (dict(code=1, zeros=FAKE), SHAPE), (dict(M=0), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(group=0), SHAPE),
    (dict(M=-1), SHAPE), (dict(group=-128), SHAPE), (dict(M=65), UNSUPPORTED), (dict(K=252), UNSUPPORTED),
    (dict(K=(1 << 20) + 8), UNSUPPORTED), (dict(group=16), UNSUPPORTED), (dict(group=96), UNSUPPORTED), (dict(group=192), UNSUPPORTED),
    (dict(x=FAKE + 8), UNSUPPORTED), (dict(codes=FAKE + (1 << 30) + 4), UNSUPPORTED), (dict(scales=FAKE + (2 << 30) + 1), UNSUPPORTED),
    (dict(y=FAKE + (3 << 30) + 2), UNSUPPORTED), (dict(bias=FAKE + (4 << 30) + 2), UNSUPPORTED),
    (dict(residual=FAKE + (4 << 30) + 1), UNSUPPORTED),
    (dict(y=FAKE), UNSUPPORTED), (dict(y=FAKE + 4 * 256 * 2 - 4), UNSUPPORTED), (dict(y=FAKE + (1 << 30)), UNSUPPORTED),
    (dict(y=FAKE + (2 << 30)), UNSUPPORTED), (dict(zeros=FAKE + (3 << 30)), UNSUPPORTED), (dict(bias=FAKE + (3 << 30)), UNSUPPORTED),
    (dict(residual=FAKE + (3 << 30)), UNSUPPORTED),                  # y may be the residual where their types agree only
    (dict(residual=FAKE + (3 << 30) + 2, out=BF16), UNSUPPORTED),
])
def test_matvec_w4_refuses(kw, want):
    assert matvec(**kw) == want


def rules(**kw):
    a = dict(history=FAKE + (4 << 30), history_ranges=FAKE + (5 << 30), penalties=FAKE + (6 << 30), bias_ids=FAKE + (7 << 30),
             bias_values=FAKE + (8 << 30), bias_ranges=FAKE + (9 << 30), mask=FAKE + (10 << 30), n_history=100, n_biases=10)
    a.update(kw)
    return ctypes.byref(coral._LogitRulesStruct(**a))


RULE_REFUSALS = [
    (dict(history=None), NULL), (dict(history_ranges=None), NULL), (dict(penalties=None), NULL), (dict(bias_ids=None), NULL),
    (dict(bias_values=None), NULL), (dict(bias_ranges=None), NULL), (dict(n_history=-1), SHAPE), (dict(n_biases=-1), SHAPE),
    (dict(n_history=(1 << 29) + 1), UNSUPPORTED), (dict(n_biases=(1 << 29) + 1), UNSUPPORTED), (dict(mask=FAKE + 2), UNSUPPORTED),
    (dict(history=FAKE + 1), UNSUPPORTED), (dict(penalties=FAKE + 2), UNSUPPORTED), (dict(bias_ranges=FAKE + 1), UNSUPPORTED)]


def adjust(r=None, **kw):
    a = dict(logits=FAKE, M=4, V=1000, dt=F32, out=FAKE + (1 << 30))
    a.update(kw)
    return coral._L.coral_logits_adjust(a["logits"], r, a["M"], a["V"], a["dt"], a["out"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(logits=None), NULL), (dict(out=None), NULL), (dict(dt=5), SHAPE), (dict(M=0), SHAPE), (dict(V=0), SHAPE),
    (dict(M=65), UNSUPPORTED), (dict(V=1000001), UNSUPPORTED), (dict(logits=FAKE + 4), UNSUPPORTED),
    (dict(out=FAKE + (1 << 30) + 4), UNSUPPORTED), (dict(out=FAKE + 16), UNSUPPORTED), (dict(out=FAKE - 16), UNSUPPORTED)])
def test_logits_adjust_refuses(kw, want):
    assert adjust(**kw) == want


@pytest.mark.parametrize("kw,want", RULE_REFUSALS)
def test_logits_adjust_refuses_rules(kw, want):
    assert adjust(rules(**kw)) == want
    assert topk(rules(**kw)) == want


@pytest.mark.parametrize("part", ["history", "history_ranges", "penalties", "bias_ids", "bias_values", "bias_ranges", "mask"])
def test_outputs_over_the_rules_are_refused(part):
    assert adjust(rules(**{part: FAKE + (1 << 30) + 64})) == UNSUPPORTED
    assert topk(rules(**{part: FAKE + (1 << 30)})) == UNSUPPORTED              # the ids
    assert topk(rules(**{part: FAKE + (3 << 30) + 256})) == UNSUPPORTED        # the workspace


def topk(r=None, **kw):
    a = dict(logits=FAKE, M=4, V=1000, k=8, dt=F32, ids=FAKE + (1 << 30), logp=FAKE + (2 << 30), ws=(FAKE + (3 << 30)) & ~255,
             ws_bytes=1 << 20)
    a.update(kw)
    return coral._L.coral_logits_topk(a["logits"], r, a["M"], a["V"], a["k"], a["dt"], a["ids"], a["logp"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(logits=None), NULL), (dict(ids=None), NULL), (dict(logp=None), NULL), (dict(dt=-1), SHAPE), (dict(k=0), SHAPE),
    (dict(V=7), SHAPE), (dict(k=65), UNSUPPORTED), (dict(M=65), UNSUPPORTED), (dict(V=1000001), UNSUPPORTED),
    (dict(ids=FAKE + (1 << 30) + 2), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws=FAKE + (3 << 30) + 8), WORKSPACE),
    (dict(ws_bytes=1 << 10), WORKSPACE), (dict(ids=FAKE), UNSUPPORTED), (dict(logp=FAKE + (1 << 30)), UNSUPPORTED),
    (dict(ws=FAKE & ~255), UNSUPPORTED), (dict(logp=(FAKE + (3 << 30)) & ~255), UNSUPPORTED)])
def test_logits_topk_refuses(kw, want):
    assert topk(**kw) == want


def test_topk_workspace_bytes():
    wb = coral.coral_logits_topk_workspace_bytes
    assert wb(0, 100, 5) == wb(4, 100, 101) == wb(4, 0, 1) == wb(65, 100, 5) == wb(1, 100, 0) == wb(1, 1000, 65) == wb(1, 1000001, 1) == 0
    for V, k in ((1, 1), (5000, 10), (152064, 64), (1000000, 64)):
        sizes = [wb(M, V, k) for M in range(1, 65)]
        assert all(n % 256 == 0 for n in sizes) and sizes == sorted(sizes)     # it serves fewer rows too
        assert topk(M=64, V=V, k=k, ws_bytes=sizes[-1] - 1, ids=FAKE + (20 << 30), logp=FAKE + (21 << 30), ws=(FAKE + (30 << 30)) & ~255) == WORKSPACE


def test_row_counters_lie_in_the_score_words(tmp_path):
    """One counter a row, each in 256 bytes of its own, in the words that the heads' shared gate leaves zero between
    calls and coral_lmhead_workspace_init clears; the published lists behind them."""
    import subprocess
    (tmp_path / "c.cpp").write_text('#include <cstdio>\n#include "control_words.h"\nint main() { using namespace coral_ctrl;\n'
                                    'std::printf("%d %d %d %d %d %d\\n", kWords, kGateScores, kGateScoreWords, kPreparedWords, kRowArrival, kRowArrivalStride); }\n')
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2502_16880_amd", "csrc"), str(tmp_path / "c.cpp"), "-o", str(tmp_path / "c")], check=True)
    out = subprocess.run([str(tmp_path / "c")], check=True, capture_output=True, text=True).stdout
    words, scores, n_scores, prepared, first, stride = map(int, out.split())
    counters = [first + m * stride for m in range(64)]
    assert stride * 4 >= 256 and scores == words and prepared == scores + n_scores
    assert all(scores <= c < scores + n_scores for c in counters)
    import test_gpu_operators as gpu
    assert gpu.PREPARED == 4 * prepared and (gpu.PREPARED - 4 * words) == 4 * n_scores
    assert coral.coral_logits_topk_workspace_bytes(1, 1, 1) > 4 * prepared


def test_binding_refuses_host_tensors_and_wrong_types():
    x, codes, scales = torch.zeros(2, 64), torch.zeros(3, 32, dtype=torch.uint8), torch.zeros(3, 1)
    with pytest.raises(ValueError, match="device memory"):
        coral.coral_matvec_w4(x, codes, scales)
    with pytest.raises(TypeError):
        coral.coral_matvec_w4(x.double(), codes, scales)
    with pytest.raises(ValueError, match="device memory"):
        coral.coral_logits_adjust(torch.zeros(2, 64))
    with pytest.raises(ValueError, match="device memory"):
        coral.coral_logits_topk(torch.zeros(2, 64), 4)
    with pytest.raises(TypeError):
        coral.coral_logits_topk(torch.zeros(2, 64, dtype=torch.int32), 4)


class OnDevice(torch.Tensor):
    """A tensor without memory that passes for one on the device."""
    is_cuda = property(lambda self: True)


def on_device(*shape, dtype=torch.float32):
    return torch.Tensor._make_subclass(OnDevice, torch.empty(shape, dtype=dtype, device="meta"))


WIDE = 2 ** 32                       # what an argument of 32 bits does not see


def test_binding_refuses_sizes_beyond_32_bits(monkeypatch):
    """Arguments that ctypes would cut to their lower halves, where the operands fit the whole ones."""
    calls = []
    monkeypatch.setattr(coral, "_enqueue", lambda *a: calls.append(a))
    u8, f16 = torch.uint8, torch.float16
    x, codes = on_device(2, 256), on_device(64, 128, dtype=u8)
    coral.coral_matvec_w4(x, codes, on_device(64, 2))
    coral.coral_logits_topk(on_device(2, 100), 5, workspace=on_device(1 << 20, dtype=u8))
    coral.coral_logits_adjust(on_device(2, 100))
    assert len(calls) == 3
    for call in (lambda: coral.coral_matvec_w4(x, codes, on_device(64, 1), group=WIDE + 128),
                 lambda: coral.coral_matvec_w4(x, on_device(WIDE + 64, 128, dtype=u8), on_device(WIDE + 64, 2)),
                 lambda: coral.coral_matvec_w4(on_device(WIDE + 2, 8), on_device(64, 4, dtype=u8), on_device(64, 1)),
                 lambda: coral.coral_matvec_w4(on_device(2, WIDE + 256), on_device(64, WIDE // 2 + 128, dtype=u8), on_device(64, WIDE // 128 + 2)),
                 lambda: coral.coral_logits_adjust(on_device(1, WIDE + 100, dtype=f16)),
                 lambda: coral.coral_logits_adjust(on_device(WIDE + 1, 8, dtype=f16)),
                 lambda: coral.coral_logits_topk(on_device(1, WIDE + 100), 5, workspace=on_device(1 << 20, dtype=u8)),
                 lambda: coral.coral_logits_topk(on_device(2, 100), WIDE + 5, workspace=on_device(1 << 20, dtype=u8)),
                 lambda: coral.coral_logits_topk(on_device(2, 100), 5 - WIDE, workspace=on_device(1 << 20, dtype=u8))):
        with pytest.raises(ValueError, match="32 bits"):
            call()
    assert len(calls) == 3
    wb = coral.coral_logits_topk_workspace_bytes
    assert wb(2, 100, 5) > 0 and wb(WIDE + 2, 100, 5) == wb(2, WIDE + 100, 5) == wb(2, 100, WIDE + 5) == wb(2 - WIDE, 100, 5) == 0


# ---------------------------------------------------------------- the oracle
def test_oracle_codes_and_weights_by_hand():
    codes = np.array([[0x10, 0x98, 0xFE, 0x37]], dtype=np.uint8)               # columns 0 1 8 9 14 15 7 3
    assert plain.unpack(codes).tolist() == [[0, 1, 8, 9, 14, 15, 7, 3]]
    scales, zeros = np.array([[2.0, 10.0]]), np.array([[1, 3]], dtype=np.uint8)
    assert plain.w4_weights(codes, scales, None, 4, "int").tolist() == [[-16, -14, 0, 2, 60, 70, -10, -50]]
    assert plain.w4_weights(codes, scales, zeros, 4, "int").tolist() == [[-2, 0, 14, 16, 110, 120, 40, 0]]
    assert plain.w4_weights(codes, scales, None, 4, "e2m1").tolist() == [[0, 1, 0, -1, -40, -60, 60, 15]]
    x = np.zeros((1, 8))
    x[0, 5] = 3.0
    assert plain.matvec_w4(x, codes, scales, None, 4).tolist() == [[210.0]]
    assert plain.matvec_w4(-x, codes, scales, None, 4, act="relu", residual=np.array([[5.0]]), bias=np.array([1.0])).tolist() == [[5.0]]
    y = plain.matvec_w4(x / 70, codes, scales, None, 4, act="silu")
    assert math.isclose(y[0, 0], 3 / (1 + math.exp(-3)))


def test_oracle_rules_by_hand():
    z = np.array([[4.0, -4.0, 1.0, 2.0, 3.0, np.nan]])
    history = np.array([0, 1, 1, 9, 3, -1], dtype=np.int32)                    # prompt 0, output 1 1 9 3
    got, _ = plain.logit_rules(z, history, np.array([[0, 1, 1, 5]]), np.array([[2.0, 0.5, 0.25]]), np.array([2, 2, 77], np.int32),
                               np.array([9.0, -1.0, 5.0]), np.array([[0, 99]]), np.array([[0b001111]]))
    assert got.tolist() == [[2.0, -8.0 - 1.0 - 0.25, 0.0, 1.0 - 0.5 - 0.25, -np.inf, -np.inf]]
    ids, logp = plain.topk_logprob(got, 5)
    assert ids.tolist() == [[0, 3, 2, 1, -1]] and logp[0, 4] == -np.inf
    assert math.isclose(np.exp(logp[0, :4]).sum(), 1.0)
    ids, logp = plain.topk_logprob(np.array([[1.0, 1.0, 0.0], [-np.inf, np.nan, -np.inf]]), 2)
    assert ids.tolist() == [[0, 1], [-1, -1]] and np.all(logp[1] == -np.inf)


def test_oracle_log_probabilities_of_values_far_from_zero():
    for size in (1.0, 1e17, 3.4e38):
        ids, logp = plain.topk_logprob(np.array([[-size, -np.inf, -size, -size], [size, size, -np.inf, -np.inf]]), 2)
        assert ids.tolist() == [[0, 2], [0, 1]]
        assert np.allclose(logp, [[-math.log(3)] * 2, [-math.log(2)] * 2], rtol=0, atol=1e-15)


def test_oracle_against_torch():
    rng = np.random.default_rng(0)
    z = rng.standard_normal((3, 200)) * 3
    ids, logp = plain.topk_logprob(z, 7)
    want = torch.log_softmax(torch.from_numpy(z), dim=1).topk(7, dim=1)
    assert np.array_equal(ids, want.indices.numpy()) and np.allclose(logp, want.values.numpy(), rtol=0, atol=1e-12)
    history = rng.integers(0, 200, 60).astype(np.int32)
    got, err = plain.logit_rules(z, history, np.array([[0, 20, 20, 40]] * 3), np.array([[1.3, 0.2, 0.1]] * 3))
    prompt, output = (torch.bincount(torch.from_numpy(h).long(), minlength=200) for h in (history[:20], history[20:40]))
    output = output.double()
    t = torch.from_numpy(z)
    t = torch.where((prompt + output) > 0, torch.where(t > 0, t / 1.3, t * 1.3), t) - 0.2 * output - 0.1 * (output > 0).double()
    assert np.allclose(got, t.numpy(), rtol=0, atol=1e-12) and (err >= 0).all() and err.max() < 5 * 2.0 ** -24 * 20      # five roundings of values below 20
