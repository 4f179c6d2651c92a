"""A drafter's attention without a GPU: refusals of the C ABI and of the binding, the oracle against values
worked out by hand, and the plan of the cached kernel compiled for the host."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2502_16880_amd as coral
from oracle import attention as plain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, SHAPE, GROUP_INDEX, UNSUPPORTED, WORKSPACE, HIP = range(7)
F32, BF16, F16 = 0, 1, 2
BASE = 0x7000_0000_0000          # never dereferenced: every check below fails before a launch
L = coral._L


def at(n):
    """Made-up arrays of 1 GB each, far from each other."""
    return BASE + (n << 34)


def cache_struct(**kw):
    a = dict(k_codes=at(20), k_scales=at(21), v_codes=at(22), v_scales=at(23), pages=10, page_size=64, kv_heads=8, head_dim=128)
    a.update(kw)
    return coral._Kv4CacheStruct(*(a[n] for n, _ in coral._Kv4CacheStruct._fields_))


def ref(struct):
    return None if struct is None else ctypes.byref(struct)


# ---------------------------------------------------------------- refusals of the C ABI
def rope(rope=True, cache=None, **kw):
    r = dict(q_weight=at(10), k_weight=at(11), positions=at(12), inv_freq=at(13), eps=1e-6, rot_dim=128, interleaved=0)
    a = dict(q=at(0), q_stride=4096, k=at(1), k_stride=1024, T=5, q_heads=32, kv_heads=8, head_dim=128, dt=BF16, q_out=at(2),
             q_out_stride=4096, k_out=at(3), k_out_stride=1024, v=None, v_stride=1024, slots=None)
    for n, value in kw.items():
        (r if n in r else a)[n] = value
    s = coral._RopeStruct(*(r[n] for n, _ in coral._RopeStruct._fields_))
    return L.coral_qk_norm_rope(a["q"], a["q_stride"], a["k"], a["k_stride"], ref(s) if rope else None, a["T"], a["q_heads"], a["kv_heads"],
                                a["head_dim"], a["dt"], a["q_out"], a["q_out_stride"], a["k_out"], a["k_out_stride"], ref(cache), a["v"],
                                a["v_stride"], a["slots"], None)


@pytest.mark.parametrize("status,kw", [
    (NULL, dict(rope=False)), (NULL, dict(q=None)), (NULL, dict(k=None)), (NULL, dict(q_out=None)), (NULL, dict(k_out=None)),
    (NULL, dict(positions=None)), (NULL, dict(inv_freq=None)), (NULL, dict(v=at(4))), (NULL, dict(slots=at(4))),
    (SHAPE, dict(T=-1)), (SHAPE, dict(q_heads=-1)), (SHAPE, dict(q_heads=0, kv_heads=0)), (SHAPE, dict(dt=3)), (SHAPE, dict(rot_dim=130)),
    (SHAPE, dict(rot_dim=-2)), (SHAPE, dict(rot_dim=7)), (SHAPE, dict(eps=-1.0)), (SHAPE, dict(eps=math.nan)), (SHAPE, dict(q_stride=4088)),
    (SHAPE, dict(k_out_stride=1000)), (UNSUPPORTED, dict(head_dim=96, rot_dim=64)), (UNSUPPORTED, dict(q_heads=1025, q_stride=1025 * 128)),
    (UNSUPPORTED, dict(q=at(0) + 8)), (UNSUPPORTED, dict(k_stride=1028)), (UNSUPPORTED, dict(q_weight=at(10) + 2)),
    (UNSUPPORTED, dict(positions=at(12) + 2)), (UNSUPPORTED, dict(q_out=at(0) + 16)), (UNSUPPORTED, dict(q_out=at(0), q_out_stride=4104)),
    (UNSUPPORTED, dict(q_out=at(1))), (UNSUPPORTED, dict(k_out=at(2))), (UNSUPPORTED, dict(q_out=at(10))), (UNSUPPORTED, dict(k_out=at(13))),
    # columns of one matrix: queries' place reaches into the keys'
    (UNSUPPORTED, dict(q=at(0), q_stride=6144, k=at(0) + 8192, k_stride=6144, q_out=at(0) + 16, q_out_stride=6144)),
])
def test_qk_norm_rope_refusals(status, kw):
    assert rope(**kw) == status


@pytest.mark.parametrize("status,kw,cache", [
    (NULL, dict(), {}), (NULL, dict(v=at(4)), {}), (NULL, dict(slots=at(5)), {}), (SHAPE, dict(v=at(4), slots=at(5)), dict(kv_heads=4)),
    (SHAPE, dict(v=at(4), slots=at(5)), dict(head_dim=64)), (UNSUPPORTED, dict(v=at(4), slots=at(5)), dict(page_size=24)),
    (UNSUPPORTED, dict(v=at(4), slots=at(5)), dict(page_size=8)), (UNSUPPORTED, dict(v=at(4), slots=at(5)), dict(page_size=8192)),
    (SHAPE, dict(v=at(4), slots=at(5)), dict(pages=0)), (UNSUPPORTED, dict(v=at(4), slots=at(5)), dict(pages=1 << 26)),
    (NULL, dict(v=at(4), slots=at(5)), dict(v_scales=None)), (UNSUPPORTED, dict(v=at(4), slots=at(5)), dict(k_codes=at(20) + 4)),
    (UNSUPPORTED, dict(v=at(4), slots=at(5) + 1), {}), (UNSUPPORTED, dict(v=at(20), slots=at(5)), {}), (UNSUPPORTED, dict(v=at(4), slots=at(21)), {}),
    (UNSUPPORTED, dict(v=at(4), slots=at(5), k_out=at(22)), {}), (UNSUPPORTED, dict(v=at(4), slots=at(5), q_out=at(4)), {}),
])
def test_qk_norm_rope_refusals_with_a_cache(status, kw, cache):
    assert rope(cache=cache_struct(**cache), **kw) == status


def test_nothing_to_do_is_no_error():
    assert rope(T=0, q=None, k=None, q_out=None, k_out=None) == OK
    assert rope(T=0, rot_dim=129) == SHAPE
    c = cache_struct()
    assert L.coral_kv4_append(ref(c), None, 0, None, 0, None, 0, BF16, None) == OK
    assert L.coral_kv4_read(ref(c), None, 0, BF16, None, None, None) == OK
    assert cached(T=0, q=None, out=None) == OK
    assert prompt(T=0, keys=0, q=None, k=None, v=None, out=None) == OK


@pytest.mark.parametrize("status,cache,kw", [
    (NULL, None, {}), (NULL, {}, dict(k=None)), (NULL, {}, dict(v=None)), (NULL, {}, dict(slots=None)), (SHAPE, {}, dict(T=-1)), (SHAPE, {}, dict(dt=7)),
    (SHAPE, {}, dict(k_stride=1016)), (UNSUPPORTED, {}, dict(v_stride=1025)), (UNSUPPORTED, {}, dict(v=at(1) + 4)), (UNSUPPORTED, {}, dict(slots=at(2) + 2)),
    (UNSUPPORTED, {}, dict(k=at(22))), (UNSUPPORTED, {}, dict(slots=at(23))), (UNSUPPORTED, {}, dict(T=1 << 24)), (UNSUPPORTED, dict(head_dim=32), {}), (SHAPE, dict(kv_heads=0), {}),
    (UNSUPPORTED, dict(kv_heads=1025), dict(k_stride=1 << 20, v_stride=1 << 20)),
])
def test_kv4_append_refusals(status, cache, kw):
    a = dict(k=at(0), k_stride=1024, v=at(1), v_stride=1024, slots=at(2), T=9, dt=BF16)
    a.update(kw)
    c = None if cache is None else cache_struct(**cache)
    assert L.coral_kv4_append(ref(c), a["k"], a["k_stride"], a["v"], a["v_stride"], a["slots"], a["T"], a["dt"], None) == status


@pytest.mark.parametrize("status,kw", [
    (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(slots=None)), (SHAPE, dict(T=-1)), (SHAPE, dict(dt=-1)), (UNSUPPORTED, dict(k=at(0) + 8)),
    (UNSUPPORTED, dict(slots=at(2) + 1)), (UNSUPPORTED, dict(v=at(0) + 1024)), (UNSUPPORTED, dict(k=at(20))), (UNSUPPORTED, dict(k=at(2))),
])
def test_kv4_read_refusals(status, kw):
    a = dict(k=at(0), v=at(1), slots=at(2), T=9, dt=BF16)
    a.update(kw)
    assert L.coral_kv4_read(ref(cache_struct()), a["slots"], a["T"], a["dt"], a["k"], a["v"], None) == status


def cached(cache={}, **kw):
    a = dict(q=at(0), q_stride=4096, page_table=at(1), max_pages=6, lengths=at(2), q_offsets=at(3), history=None, tree=None, T=7, S=3, max_rows=4,
             max_length=300, q_heads=32, scale=0.1, dt=BF16, out=at(4), workspace=at(5), bytes=1 << 28)
    a.update(kw)
    c = None if cache is None else cache_struct(**cache)
    return L.coral_attention_kv4(a["q"], a["q_stride"], ref(c), a["page_table"], a["max_pages"], a["lengths"], a["q_offsets"], a["history"], a["tree"],
                                 a["T"], a["S"], a["max_rows"], a["max_length"], a["q_heads"], a["scale"], a["dt"], a["out"], a["workspace"], a["bytes"], None)


@pytest.mark.parametrize("status,kw", [
    (NULL, dict(cache=None)), (NULL, dict(q=None)), (NULL, dict(out=None)), (NULL, dict(page_table=None)), (NULL, dict(lengths=None)), (NULL, dict(q_offsets=None)),
    (NULL, dict(tree=at(6))), (NULL, dict(history=at(6))), (SHAPE, dict(T=-1)), (SHAPE, dict(S=0)), (SHAPE, dict(max_rows=0)), (SHAPE, dict(max_length=-1)),
    (SHAPE, dict(q_heads=0)), (SHAPE, dict(q_heads=31)), (SHAPE, dict(max_pages=-1)), (SHAPE, dict(scale=math.inf)), (SHAPE, dict(scale=math.nan)),
    (SHAPE, dict(dt=5)), (SHAPE, dict(q_stride=128)), (UNSUPPORTED, dict(max_rows=65)), (UNSUPPORTED, dict(S=65536)), (UNSUPPORTED, dict(q_heads=1032, q_stride=1032 * 128)),
    (UNSUPPORTED, dict(cache=dict(head_dim=80))), (UNSUPPORTED, dict(q=at(0) + 2)), (UNSUPPORTED, dict(out=at(4) + 8)), (UNSUPPORTED, dict(lengths=at(2) + 1)),
    (UNSUPPORTED, dict(tree=at(6) + 4, history=at(7))), (WORKSPACE, dict(workspace=None)), (WORKSPACE, dict(workspace=at(5) + 128)), (WORKSPACE, dict(bytes=1000)),
    (UNSUPPORTED, dict(out=at(0))), (UNSUPPORTED, dict(out=at(22))), (UNSUPPORTED, dict(out=at(3))), (UNSUPPORTED, dict(workspace=at(20))),
    (UNSUPPORTED, dict(workspace=at(4))), (UNSUPPORTED, dict(workspace=at(6), tree=at(6), history=at(7))), (SHAPE, dict(cache=dict(page_size=0))),
])
def test_attention_kv4_refusals(status, kw):
    assert cached(**kw) == status


def prompt(**kw):
    a = dict(q=at(0), q_stride=4096, k=at(1), k_stride=1024, v=at(2), v_stride=1024, q_offsets=at(3), k_offsets=None, T=100, keys=100, S=2, q_heads=32,
             kv_heads=8, head_dim=128, scale=0.1, dt=BF16, out=at(4))
    a.update(kw)
    return L.coral_attention_prompt(*(a[n] for n in ("q", "q_stride", "k", "k_stride", "v", "v_stride", "q_offsets", "k_offsets", "T", "keys", "S", "q_heads",
                                                     "kv_heads", "head_dim", "scale", "dt", "out")), None)


@pytest.mark.parametrize("status,kw", [
    (NULL, dict(q=None)), (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(out=None)), (NULL, dict(q_offsets=None)), (SHAPE, dict(T=-1)),
    (SHAPE, dict(keys=-1)), (SHAPE, dict(keys=99)), (SHAPE, dict(S=0)), (SHAPE, dict(q_heads=30)), (SHAPE, dict(kv_heads=0)), (SHAPE, dict(scale=math.inf)),
    (SHAPE, dict(dt=3)), (SHAPE, dict(k_stride=1016)), (UNSUPPORTED, dict(head_dim=96)), (UNSUPPORTED, dict(q_heads=2048, q_stride=2048 * 128)),
    (UNSUPPORTED, dict(v=at(2) + 8)), (UNSUPPORTED, dict(v_stride=1028)), (UNSUPPORTED, dict(k_stride=1 << 24)), (UNSUPPORTED, dict(q_offsets=at(3) + 2)),
    (UNSUPPORTED, dict(out=at(0))), (UNSUPPORTED, dict(out=at(1) + 512)), (UNSUPPORTED, dict(out=at(2))), (UNSUPPORTED, dict(out=at(3))),
    (UNSUPPORTED, dict(k_offsets=at(4))), (UNSUPPORTED, dict(S=65536)), (UNSUPPORTED, dict(T=1 << 24, keys=1 << 24)), (UNSUPPORTED, dict(keys=1 << 24, k_offsets=at(5))),
    (UNSUPPORTED, dict(T=1 << 23, keys=1 << 23, q_heads=1024, q_stride=1024 * 128)),         # more threads than a grid's 32 bits count
])
def test_attention_prompt_refusals(status, kw):
    assert prompt(**kw) == status


# ---------------------------------------------------------------- refusals of the binding
def test_binding_refuses_before_the_library_is_entered():
    q, k = torch.zeros((3, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    cache = coral.alloc_kv4_cache(2, 16, 2, 64, device="cpu")
    assert [tuple(t.shape) for t in cache] == [(2, 2, 16, 32), (2, 2, 16, 2)] * 2
    ids = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: coral.coral_qk_norm_rope(q, k), lambda: coral.coral_kv4_append(cache, k, k, ids), lambda: coral.coral_kv4_read(cache, ids, q.dtype),
                 lambda: coral.coral_attention_kv4(q, cache, ids[None], ids[:1], ids[:2], 1), lambda: coral.coral_attention_prompt(q, k, k, ids[:2])):
        with pytest.raises(ValueError, match="device memory"):
            call()
    with pytest.raises(ValueError, match="q or k"):
        coral.coral_qk_norm_rope(None, None)
    with pytest.raises(TypeError):
        coral.coral_qk_norm_rope(q.int(), k)
    assert coral.coral_attention_kv4_workspace_bytes(1, 1, 1 << 40, 8, 8, 128, BF16) == 0
    assert coral.coral_attention_kv4_workspace_bytes(1, 65, 100, 8, 8, 128, BF16) == 0


def test_binding_tells_dense_heads_from_others():
    dev = torch.device("cpu")
    x = torch.zeros((5, 12, 64))
    assert coral._heads_ptr(x[:, 2:6], "x", dev, torch.float32) == (x.data_ptr() + 2 * 64 * 4, 768)
    assert coral._heads_ptr(x[:1, :1], "x", dev, torch.float32)[1] == 64                 # one token has no stride
    assert coral._heads_ptr(x[::2], "x", dev, torch.float32)[1] == 1536
    assert coral._heads_ptr(x[:0], "x", dev, torch.float32)[1] == 768
    for bad in (x[:, ::2], x.transpose(0, 1), x[..., ::2], x[..., :32]):
        with pytest.raises(ValueError, match="heads one behind the other"):
            coral._heads_ptr(bad, "x", dev, torch.float32)
    with pytest.raises(ValueError, match="tokens, heads"):
        coral._heads_ptr(x[0], "x", dev, torch.float32)
    with pytest.raises(TypeError):
        coral._heads_ptr(x, "x", dev, torch.float16)


# ---------------------------------------------------------------- the oracle
def test_oracle_rotation_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    quarter = np.array([math.pi / 2, 0.0])
    assert np.allclose(plain.norm_rope(x, np.array([1]), quarter), [[[-3.0, 2.0, 1.0, 4.0]]])
    assert np.allclose(plain.norm_rope(x, np.array([1]), quarter, interleaved=True), [[[-2.0, 1.0, 3.0, 4.0]]])
    assert np.allclose(plain.norm_rope(x, np.array([2]), quarter[:1]), [[[-1.0, -2.0, 3.0, 4.0]]])          # a part of the head
    y = plain.norm_rope(x, weight=np.array([1.0, 1.0, 2.0, 0.0]), eps=0.0)
    assert np.allclose(y, x / math.sqrt(7.5) * [1, 1, 2, 0])


def test_oracle_4_bit_floats_by_hand():
    x = np.zeros(64)
    x[:16] = [6, -6, 5, 4.9, 5.1, 3.5, 3.4, 2.5, 2.6, 1.75, 1.25, 0.75, 0.25, 0.26, -0.2, 7]
    codes, scales = plain.kv4_quantise(x, "f32")
    assert scales.tolist() == [127, 1] and plain.kv4_values(codes, scales)[16:].any() == 0
    want = [6, -6, 4, 4, 6, 4, 3, 2, 3, 2, 1, 1, 0, 0.5, 0, 6]
    assert plain.kv4_values(codes, scales)[:16].tolist() == want
    x[15] = 7.01                                                                # two units are nearer than one
    codes, scales = plain.kv4_quantise(x, "f32")
    assert scales[0] == 128 and plain.kv4_values(codes, scales)[15] == 8.0
    for dtype, most in (("f32", 6 * 2.0 ** 125), ("f16", 6 * 2.0 ** 13)):
        codes, scales = plain.kv4_quantise(np.full(32, -np.inf), dtype)
        assert (plain.kv4_values(codes, scales) == -most).all()
    rng = np.random.default_rng(0)
    held = plain.kv4_values(*plain.kv4_quantise(rng.standard_normal((50, 128)) * np.exp(rng.standard_normal((50, 1)) * 20), "f32"))
    assert np.array_equal(plain.kv4_values(*plain.kv4_quantise(held, "f32")), held)       # what is held is held without loss


def test_oracle_attention_against_torch():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((5, 4, 8)), rng.standard_normal((7, 2, 8)), rng.standard_normal((7, 2, 8))
    seen = np.tril(np.ones((5, 7), bool), 2)
    seen[3] = False
    out = plain.attention(q, k, v, seen, 0.3)[0]
    t = [torch.from_numpy(a).transpose(0, 1) for a in (q, k.repeat(2, axis=1), v.repeat(2, axis=1))]
    s = (t[0] @ t[1].transpose(1, 2) * 0.3).masked_fill(~torch.from_numpy(seen), -math.inf)
    want = torch.nan_to_num(torch.softmax(s, dim=-1)) @ t[2]
    assert np.abs(out - want.transpose(0, 1).numpy()).max() < 1e-14 and (out[3] == 0).all()


# ---------------------------------------------------------------- the plan of the cached kernel
PLAN = r"""
#include <cstdio>
#include "kv4_plan.h"
int main() {
    int s, rows, length, q, kv, d, terms;
    while (std::scanf("%d %d %d %d %d %d %d", &s, &rows, &length, &q, &kv, &d, &terms) == 7) {
        const Kv4Plan p = kv4_plan(s, rows, length, q, kv, d, terms);
        std::printf("%d %d %d %d %zu\n", p.tiles, p.row_blocks, p.workgroups, p.apart ? 1 : 0, kv4_workspace(p, d));
    }
}
"""


def test_plan_covers_every_row_and_the_workspace_what_it_needs(tmp_path):
    (tmp_path / "plan.cpp").write_text(PLAN)
    exe = str(tmp_path / "plan")
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2502_16880_amd", "csrc"), str(tmp_path / "plan.cpp"), "-o", exe], check=True)
    calls = [(s, rows, length, q, kv, d, terms) for s in (1, 3, 64, 65535) for rows in (1, 5, 64) for length in (0, 1, 128, 129, 8192, 2 ** 31 - 1)
             for q, kv in ((8, 8), (32, 8), (28, 4), (1024, 1)) for d in (64, 128, 256) for terms in (1, 3)]
    text = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in calls), capture_output=True, text=True, check=True).stdout
    for (s, rows, length, q, kv, d, terms), line in zip(calls, text.splitlines()):
        tiles, blocks, groups, apart, need = map(int, line.split())
        assert tiles in (1, 2) and tiles * blocks * 16 >= rows * (q // kv) and (blocks - 1) * tiles * 16 < rows * (q // kv)
        assert tiles == 1 or d * terms <= 128
        assert 1 <= groups <= 768 and groups <= s * kv * blocks * max(1, -(-length // 128)) and apart == (s > 256)
        assert need == (16896 + groups * 2 * tiles * 16 * (d + 2) * 4 if groups > 1 and not apart else 0)
        assert all(coral.coral_attention_kv4_workspace_bytes(s, rows, length, q, kv, d, dt) >= max(need, 256) for dt in ((BF16, F16) if terms == 1 else (F32,)))
