"""A drafter's attention on a real MI355X against its 64-bit definitions (oracle/attention.py, where the
tolerances are derived), and a drafter's layer made of these calls."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from coral_inputs import CONFIGS, make_head  # noqa: E402
from oracle import attention as plain  # noqa: E402
from oracle import compare, operators  # noqa: E402

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DTYPES = ["bf16", "f16", "f32"]


@pytest.fixture(scope="module")
def coral():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_16880_amd as c
    return c


def stored(a, dtype):
    """A host array as a device tensor of the storage type, and the values it then has in float64."""
    t = torch.from_numpy(np.asarray(a, dtype=np.float32)).to(TORCH[dtype])
    return t.cuda(), t.double().numpy()


def host(t):
    return t.double().cpu().numpy()


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def guarded(shape, dtype):
    """A tensor in the middle of a larger one that holds a pattern, and a check that the rest kept it."""
    n = int(np.prod(shape))
    size = torch.empty(0, dtype=dtype).element_size()
    pad = 512 // size
    whole = torch.full((n + 2 * pad,), 77, dtype=dtype, device="cuda")

    def check():
        assert bool((whole[:pad] == 77).all()) and bool((whole[pad + n:] == 77).all()), "written outside the output"
    return whole[pad:pad + n].view(shape), check


# ---------------------------------------------------------------- norms and rotation
class Heads:
    def __init__(self, dtype, T, q_heads, kv_heads, D, rot, norm=True, interleaved=False, start=0, seed=0):
        rng = np.random.default_rng([seed, T, q_heads, D, rot])
        self.dtype, self.interleaved, self.n = dtype, interleaved, (q_heads, kv_heads)
        self.qkv, self.qkv64 = stored(rng.standard_normal((T, q_heads + 2 * kv_heads, D)), dtype)
        self.parts = (slice(0, q_heads), slice(q_heads, q_heads + kv_heads), slice(q_heads + kv_heads, None))
        self.weights = [stored(1 + 0.3 * rng.standard_normal(D), dtype) if norm else (None, None) for _ in range(2)]
        self.at = start + rng.permutation(T).astype(np.int64)
        self.positions = ints(self.at)
        self.freq = (rng.random(rot // 2) * np.power(10000.0, -np.arange(rot // 2) * 2 / max(rot, 1))).astype(np.float32)
        self.inv_freq = torch.from_numpy(self.freq).cuda()

    def args(self, rot=True):
        kw = dict(q_weight=self.weights[0][0], k_weight=self.weights[1][0], interleaved=self.interleaved)
        if rot:
            kw.update(positions=self.positions, inv_freq=self.inv_freq)
        return kw

    def inputs(self):
        return [self.qkv[:, p] for p in self.parts]

    def check(self, out, which, rot=True):
        x, w = self.qkv64[:, self.parts[which]], self.weights[which][1]
        args = (self.at, self.freq) if rot else (None, None)
        want = plain.norm_rope(x, *args, w, 1e-6, self.interleaved)
        bound = plain.norm_rope_bound(x, *args, w, 1e-6, self.interleaved, self.dtype)
        off = np.abs(host(out) - want)
        assert (off <= bound).all(), f"off by {off.max():.3g} at {np.unravel_index((off - bound).argmax(), off.shape)}"


ROPES = [(1, 32, 8, 128, 128), (3, 4, 4, 64, 64), (17, 28, 4, 128, 96), (5, 9, 3, 64, 20), (33, 8, 1, 256, 256), (2, 5, 5, 256, 84), (7, 1, 1, 128, 2),
         (1100, 14, 2, 64, 32), (1024, 32, 8, 128, 128), (1025, 7, 7, 256, 62), (4, 40, 33, 128, 42)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,q_heads,kv_heads,D,rot", ROPES)
def test_qk_norm_rope(coral, T, q_heads, kv_heads, D, rot, dtype, norm, interleaved):
    c = Heads(dtype, T, q_heads, kv_heads, D, rot, norm, interleaved, start=100000)
    q, k, _ = c.inputs()
    q_out, q_kept = guarded(q.shape, TORCH[dtype])
    k_out, k_kept = guarded(k.shape, TORCH[dtype])
    coral.coral_qk_norm_rope(q, k, q_out=q_out, k_out=k_out, **c.args())
    c.check(q_out, 0)
    c.check(k_out, 1)
    q_kept()
    k_kept()
    again = coral.coral_qk_norm_rope(q, k, **c.args())
    assert torch.equal(again[0], q_out) and torch.equal(again[1], k_out)


@pytest.mark.parametrize("dtype", DTYPES)
def test_qk_norm_rope_far_positions_keep_their_angle(coral, dtype):
    c = Heads(dtype, 40, 4, 2, 128, 128, norm=False, start=(1 << 24) - 50)
    c.freq[:3] = (1.0, 0.7, 0.31)
    c.inv_freq = torch.from_numpy(c.freq).cuda()
    out = coral.coral_qk_norm_rope(*c.inputs()[:2], **c.args())
    c.check(out[0], 0)
    c.check(out[1], 1)
    c.at, c.positions = -c.at, -c.positions                       # and a negative position turns back
    c.check(coral.coral_qk_norm_rope(*c.inputs()[:2], **c.args())[0], 0)


@pytest.mark.parametrize("T", [3, 1030])
@pytest.mark.parametrize("D,rot,interleaved", [(128, 128, False), (64, 20, False), (256, 256, True)])
def test_qk_norm_rope_in_place_and_one_of_both(coral, T, D, rot, interleaved):
    c = Heads("bf16", T, 6, 3, D, rot, True, interleaved)
    q, k, v = c.inputs()
    want = coral.coral_qk_norm_rope(q, k, **c.args())
    only_q, none = coral.coral_qk_norm_rope(q, None, **dict(c.args(), k_weight=None))
    assert none is None and torch.equal(only_q, want[0])
    none, only_k = coral.coral_qk_norm_rope(None, k, **dict(c.args(), q_weight=None))
    assert none is None and torch.equal(only_k, want[1])
    values = v.clone()
    got = coral.coral_qk_norm_rope(q, k, q_out=q, k_out=k, **c.args())
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, values)


def test_qk_norm_rope_without_rotation_and_with_one_norm(coral):
    c = Heads("f16", 9, 5, 2, 128, 64)
    q, k, _ = c.inputs()
    out = coral.coral_qk_norm_rope(q, k, **c.args(rot=False))
    c.check(out[0], 0, rot=False)
    c.check(out[1], 1, rot=False)
    c.weights[1] = (None, None)
    out = coral.coral_qk_norm_rope(q, k, **c.args())
    c.check(out[0], 0)
    c.check(out[1], 1)


# ---------------------------------------------------------------- the cache
def random_cache(coral, rng, pages, page, kv_heads, D, scales=(110, 135)):
    cache = coral.alloc_kv4_cache(pages, page, kv_heads, D)
    sides = []
    for codes, scale in ((cache[0], cache[1]), (cache[2], cache[3])):
        a = rng.integers(0, 256, tuple(codes.shape), dtype=np.uint8), rng.integers(scales[0], scales[1], tuple(scale.shape), dtype=np.uint8)
        codes.copy_(torch.from_numpy(a[0]))
        scale.copy_(torch.from_numpy(a[1]))
        sides.append(a)
    return cache, sides


def border_values(dtype, n):
    """Values at and next to every border of the 4-bit floats, under units from the smallest to the largest."""
    rng = np.random.default_rng(n)
    low, high = {"f32": (-149, 127), "bf16": (-133, 127), "f16": (-24, 15)}[dtype]
    base = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 7.5, 7.99])
    x = rng.choice(base, (n, 32)) * rng.choice([-1, 1], (n, 32)) * (1 + rng.choice([0, 0, 2.0 ** -10, -2.0 ** -9, 2.0 ** -7], (n, 32)))
    x[rng.random(n) < 0.05] = 0
    with np.errstate(over="ignore"):
        t = torch.from_numpy((x * np.exp2(rng.integers(low, high - 2, (n, 1)).astype(np.float64)))).to(TORCH[dtype])
    return t


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,kv_heads,D,page", [(1, 1, 64, 16), (5, 8, 128, 64), (37, 3, 64, 32), (64, 4, 256, 128), (700, 12, 128, 16), (33, 5, 256, 4096)])
def test_kv4_append_and_read(coral, dtype, T, kv_heads, D, page):
    rng = np.random.default_rng(T)
    pages = -(-T // page) + 2
    cache, sides = random_cache(coral, rng, pages, page, kv_heads, D)
    x = border_values(dtype, T * 2 * kv_heads * D // 32).reshape(T, 2 * kv_heads, D)
    x[0, 0, :32], x[-1, -1, -32:] = math.inf, -math.inf
    x64, x = x.double().numpy(), x.cuda()
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    slots[T // 3] = -1 if T > 2 else slots[T // 3]
    bad = T - 1 if T > 4 else -1
    if bad > 0:
        slots[bad] = pages * page                                 # the first that is none
    k, v = x[:, :kv_heads], x[:, kv_heads:]
    coral.coral_kv4_append(cache, k, v, ints(slots))
    good = (slots >= 0) & (slots < pages * page)
    at, off = slots[good] // page, slots[good] % page
    for (codes, scales), part in zip(sides, (x64[good][:, :kv_heads], x64[good][:, kv_heads:])):
        codes[at, :, off], scales[at, :, off] = plain.kv4_quantise(part, dtype)
    for got, want in zip(cache, (*sides[0], *sides[1])):
        assert np.array_equal(got.cpu().numpy(), want)            # the new ones, and all others as they were
    k_out, k_kept = guarded((T, kv_heads, D), TORCH[dtype])
    v_out, v_kept = guarded((T, kv_heads, D), TORCH[dtype])
    coral.coral_kv4_read(cache, ints(slots), TORCH[dtype], k_out, v_out)
    for out, (codes, scales) in ((k_out, sides[0]), (v_out, sides[1])):
        want = np.full((T, kv_heads, D), 77.0)
        want[good] = plain.kv4_values(codes[at, :, off], scales[at, :, off], dtype)
        want = torch.from_numpy(want).to(TORCH[dtype])
        assert torch.equal(out.cpu().nan_to_num(), want.nan_to_num())
    k_kept()
    v_kept()
    before = [t.clone() for t in cache]                           # what is read is appended without loss
    coral.coral_kv4_append(cache, k_out, v_out, ints(np.where(good, slots, -1)))
    again = coral.coral_kv4_read(cache, ints(slots), TORCH[dtype], k_out.clone(), v_out.clone())
    assert torch.equal(again[0], k_out) and torch.equal(again[1], v_out)
    assert all(a.shape == b.shape for a, b in zip(before, cache))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,kv_heads,D,page", [(1, 1, 64, 16), (37, 3, 64, 32), (64, 4, 256, 128), (700, 12, 128, 16)])
def test_kv4_append_of_what_was_read_changes_no_value_and_no_other_place(coral, dtype, T, kv_heads, D, page):
    rng = np.random.default_rng(T)
    pages = -(-T // page) + 2
    cache, sides = random_cache(coral, rng, pages, page, kv_heads, D)
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    x = border_values(dtype, T * 2 * kv_heads * D // 32).reshape(T, 2 * kv_heads, D).cuda()
    coral.coral_kv4_append(cache, x[:, :kv_heads], x[:, kv_heads:], ints(slots))
    before = [t.cpu().numpy().copy() for t in cache]
    held = coral.coral_kv4_read(cache, ints(slots), TORCH[dtype])
    skip = rng.random(T) < 0.3                                     # places that are read but not appended to
    coral.coral_kv4_append(cache, *held, ints(np.where(skip, -1, slots)))
    after = [t.cpu().numpy() for t in cache]
    at, off = slots[~skip] // page, slots[~skip] % page
    for i in (0, 2):
        old, new = (plain.kv4_values(side[i][at, :, off], side[i + 1][at, :, off], dtype) for side in (before, after))
        rounded = torch.from_numpy(old).to(TORCH[dtype]).double().numpy()      # (what is read: units of few bits below the type's smallest)
        assert np.array_equal(new, rounded)
    for old, new in zip(before, after):                            # every other place has the bytes that it had
        new = new.copy()
        new[at, :, off] = old[at, :, off]
        assert np.array_equal(old, new)


@pytest.mark.parametrize("dtype", DTYPES)
def test_kv4_read_any_byte(coral, dtype):
    rng = np.random.default_rng(5)
    cache, sides = random_cache(coral, rng, 16, 16, 2, 64, scales=(0, 256))
    out = coral.coral_kv4_read(cache, ints(np.arange(256)), TORCH[dtype])
    for got, (codes, scales) in zip(out, sides):
        want = plain.kv4_values(codes, scales, dtype).transpose(0, 2, 1, 3).reshape(256, 2, 64)
        assert torch.equal(got.cpu(), torch.from_numpy(want).to(TORCH[dtype]))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,q_heads,kv_heads,D,rot,interleaved", [(1, 32, 8, 128, 128, False), (70, 4, 4, 64, 20, False), (9, 8, 1, 256, 256, True), (1030, 6, 3, 128, 96, False), (3, 7, 7, 64, 0, False)])
def test_qk_norm_rope_into_the_cache_as_two_calls(coral, dtype, T, q_heads, kv_heads, D, rot, interleaved):
    c = Heads(dtype, T, q_heads, kv_heads, D, rot, True, interleaved)
    q, k, v = c.inputs()
    kw = c.args(rot=rot > 0)
    pages, page = T // 32 + 2, 32
    slots = np.random.default_rng(1).permutation(pages * page)[:T]
    slots[T // 2] = -1 if T > 2 else slots[T // 2]
    one, two = (random_cache(coral, np.random.default_rng(2), pages, page, kv_heads, D)[0] for _ in range(2))
    want = coral.coral_qk_norm_rope(q, k, **kw)
    coral.coral_kv4_append(two, want[1], v, ints(slots))
    got = coral.coral_qk_norm_rope(q, k, cache=one, v=v, slots=ints(slots), **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and all(torch.equal(a, b) for a, b in zip(one, two))
    three = random_cache(coral, np.random.default_rng(2), pages, page, kv_heads, D)[0]
    got = coral.coral_qk_norm_rope(q, k, k_out=False, cache=three, v=v, slots=ints(slots), **kw)
    assert got[1] is None and torch.equal(got[0], want[0]) and all(torch.equal(a, b) for a, b in zip(three, two))


# ---------------------------------------------------------------- attention: what both kinds are checked by
def check_attention(got, want, dtype, keys, where=""):
    out, mean, spread, score_off, size_v = want
    bound = plain.attention_bound(out, mean, spread, score_off, size_v, keys, dtype)
    off = np.abs(got - out)
    assert (off <= bound).all(), f"{where}: off by {off.max():.3g} at {np.unravel_index(np.argmax(off - bound), off.shape)}"
    if out.size >= 512:
        assert np.linalg.norm(off) <= plain.attention_norm_bound(out, mean, spread, score_off, size_v, dtype), where


class Cached:
    """Sequences of (tokens, rows) in a cache whose pages lie in any order."""

    def __init__(self, coral, dtype, sequences, q_heads, kv_heads, D, page, tree=False, seed=0, spare=3, q_size=1.5, behind=0):
        rng = np.random.default_rng([seed, q_heads, D, page, len(sequences)])
        self.coral, self.dtype, self.sequences, self.page = coral, dtype, sequences, page
        held = [-(-n // page) for n, _ in sequences]
        pages = sum(held) + spare
        self.cache, self.sides = random_cache(coral, rng, pages, page, kv_heads, D, scales=(124, 128))
        order = rng.permutation(pages)[:sum(held)]
        self.table = np.full((len(sequences), max(held + [1]) + 1), -1, dtype=np.int32)
        at = 0
        for s, n in enumerate(held):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.rows = [r for _, r in sequences]
        self.offsets = np.concatenate([[0], np.cumsum(self.rows)])
        T = int(self.offsets[-1]) + behind
        self.q, self.q64 = stored(rng.standard_normal((T, q_heads, D)) * q_size, dtype)
        self.history = self.tree = None
        if tree:
            self.history = np.array([max(0, n - r - int(rng.integers(0, 64 - min(r, 63)))) for n, r in sequences])
            self.tree = rng.integers(-2 ** 63, 2 ** 63, T, dtype=np.int64)
            self.tree[::5] = 0

    def seen(self, s):
        n, r = self.sequences[s]
        if self.tree is None:
            return np.arange(n)[None] <= (n - r + np.arange(r))[:, None]
        words = self.tree[self.offsets[s]:self.offsets[s + 1]].astype(np.uint64)
        out = np.zeros((r, n), bool)
        out[:, :self.history[s]] = True
        for b in range(min(64, n - self.history[s])):
            out[:, self.history[s] + b] = (words >> np.uint64(b)) & np.uint64(1) == 1
        return out

    def args(self):
        i64 = None if self.tree is None else torch.from_numpy(self.tree).cuda()
        return (self.q, self.cache, ints(self.table), ints([n for n, _ in self.sequences]), ints(self.offsets), max(self.rows + [1])), \
            dict(history=None if self.history is None else ints(self.history), tree=i64)

    def run(self, **kw):
        args, more = self.args()
        return self.coral.coral_attention_kv4(*args, **dict(more, **kw))

    def check(self, out, scale=None, only=None):
        got, D = host(out), self.q.shape[2]
        for s, (n, r) in enumerate(self.sequences):
            if only is not None and s not in only:
                continue
            k, held = plain.kv4_tokens(*self.sides[0], self.table[s], n, self.dtype)
            v, _ = plain.kv4_tokens(*self.sides[1], self.table[s], n, self.dtype)
            rows = slice(self.offsets[s], self.offsets[s + 1])
            want = plain.attention(self.q64[rows], k, v, self.seen(s) & held[None], D ** -0.5 if scale is None else scale)
            check_attention(got[rows], want, self.dtype, n, f"sequence {s} of {n} tokens, {r} rows")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (8, 2), (7, 1), (6, 3)])
@pytest.mark.parametrize("tree", [False, True])
def test_attention_kv4(coral, dtype, D, q_heads, kv_heads, tree):
    sequences = [(1, 1), (2, 1), (15, 3), (16, 1), (17, 17), (31, 2), (33, 1), (64, 64), (100, 9), (129, 1), (300, 5), (511, 40)]
    c = Cached(coral, dtype, sequences, q_heads, kv_heads, D, 16, tree)
    out, kept = guarded((sum(c.rows), q_heads, D), TORCH[dtype])
    c.run(out=out)
    c.check(out)
    kept()
    assert torch.equal(c.run(), out)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,q_heads,kv_heads,rows", [(128, 32, 8, 1), (128, 28, 4, 60), (64, 14, 2, 8), (256, 8, 4, 3), (128, 4, 4, 64), (128, 8, 1, 2), (64, 8, 8, 30), (256, 8, 1, 33)])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_attention_kv4_long(coral, dtype, D, q_heads, kv_heads, rows, page):
    c = Cached(coral, dtype, [(5003, rows), (1, 1), (2048, max(1, rows // 2))], q_heads, kv_heads, D, page, tree=rows > 1)
    out = c.run()
    c.check(out)
    assert torch.equal(c.run(), out)


def test_attention_kv4_every_number_of_shares(coral):
    """The work is cut by max_length and shared out: results differ by the order of sums only, whatever the lengths are."""
    c = Cached(coral, "f32", [(1000, 3), (130, 1), (700, 64)], 4, 2, 64, 32)
    for most in (0, 1, 129, 500, 1000, 4000, 100000):
        c.check(c.run(max_length=most))


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_kv4_many_sequences_of_any_length(coral, dtype):
    rng = np.random.default_rng(4)
    sequences = [(int(n), int(min(n, r))) for n, r in zip(np.exp(rng.uniform(0, 7, 150)).astype(int) + 1, rng.integers(1, 5, 150))]
    c = Cached(coral, dtype, sequences, 6, 2, 64, 32)
    c.check(c.run())


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_kv4_more_sequences_than_are_shared_out(coral, dtype):
    rng = np.random.default_rng(9)
    c = Cached(coral, dtype, [(int(n), 1 + int(n > 2)) for n in rng.integers(1, 200, 1030)], 4, 2, 64, 16, tree=dtype == "f16")
    c.sequences[700] = (0, 0)
    out = c.run()
    c.check(out, only=[0, 1, 500, 699, 701, 1028, 1029])
    few = Cached(coral, dtype, [(int(n), 1) for n in rng.integers(1, 3000, 250)], 2, 1, 64, 64)      # shared out, four loads of sequences
    few.check(few.run(), only=[0, 63, 64, 128, 200, 249])


def test_attention_kv4_peaked_scores(coral):
    for dtype in DTYPES:                                           # scores to +-300: references move, weights underflow
        c = Cached(coral, dtype, [(1500, 4), (40, 40)], 4, 2, 128, 64, q_size=40.0)
        c.check(c.run())
        c.check(c.run(scale=-0.25), scale=-0.25)
        c.check(c.run(scale=0.0), scale=0.0)


def test_attention_kv4_rows_that_see_nothing(coral):
    c = Cached(coral, "bf16", [(0, 3), (2, 5), (300, 2), (40, 0), (20, 1)], 4, 2, 64, 16, behind=4)
    c.sequences = [(0, 3), (2, 5), (300, 2), (40, 0), (20, 1)]
    out, kept = guarded(c.q.shape, torch.bfloat16)
    c.run(out=out)
    c.check(out, only=[0, 1, 2, 4])
    kept()
    assert bool((out[:3] == 0).all()) and bool((out[3:6] == 0).all())     # no token at all; rows before the first token
    assert bool((out[11:] == 77).all())                                   # rows behind the last sequence
    tree = torch.zeros(c.q.shape[0], dtype=torch.int64, device="cuda")
    tree[8] = 1
    out2 = c.run(history=ints([0, 0, 0, 0, 0]), tree=tree)
    assert bool((out2[:8] == 0).all()) and bool((out2[9:11] == 0).all()) and bool((out2[8] != 0).any())


def test_attention_kv4_pages_that_are_none_and_bytes_that_no_append_writes(coral):
    c = Cached(coral, "f16", [(200, 2), (333, 1), (64, 1)], 4, 2, 128, 16)
    plain_out = c.run()
    hole = c.table.copy()
    hole[0, 3], hole[0, 7], hole[1, 0], hole[1, 20], hole[2, :] = -1, 10 ** 6, -2 ** 31, 2 ** 31 - 1, -7
    c.table, whole = hole, c.table
    c.check(c.run())                                              # tokens of such pages are not seen; sequence 2 sees nothing
    assert bool((c.run()[-1] == 0).all())
    c.table = whole
    used = set(whole[whole >= 0].tolist())
    for page in set(range(c.cache[0].shape[0])) - used:           # other pages, and places behind the last token
        for t in c.cache:
            t[page] = 255
    for s, (n, _) in enumerate(c.sequences):
        for t in c.cache:
            if n % 16:
                t[int(whole[s, n // 16]), :, n % 16:] = 255
    assert torch.equal(c.run(), plain_out)
    args, _ = c.args()                                            # a token that the tree hides may hold any bytes
    n = c.sequences[1][0]
    tree, history = torch.full((4,), (1 << 62) - 2, dtype=torch.int64, device="cuda"), ints([100, n - 30, 10])
    want = c.run(tree=tree, history=history)
    for t in c.cache:
        t[int(whole[1, (n - 30) // 16]), :, (n - 30) % 16] = 255
    assert torch.equal(c.run(tree=tree, history=history), want)


def test_attention_kv4_arguments_outside_the_arrays(coral):
    c = Cached(coral, "bf16", [(100, 3), (50, 2), (70, 4)], 4, 1, 64, 32)
    (q, cache, table, lengths, offsets, rows), _ = c.args()
    want = c.run()
    room = c.table.shape[1] * 32
    c.sequences = [(room, 3), (50, 2), (70, 4)]                   # a length beyond the page table is cut to it
    long = lengths.clone()
    long[0] = 2 ** 31 - 1
    out = coral.coral_attention_kv4(q, cache, table, long, offsets, rows)
    c.check(out, only=[0])
    assert torch.equal(out[3:], want[3:])
    out.fill_(7)
    coral.coral_attention_kv4(q, cache, table, lengths, ints([-5, 3, 5, 10 ** 6]), rows, out=out)       # offsets are cut to the rows
    assert torch.equal(out, want)
    out.fill_(7)
    coral.coral_attention_kv4(q, cache, table, lengths, ints([9, 3, 5, 2]), rows, out=out)              # none, [3,5), none
    assert torch.equal(out[3:5], want[3:5]) and bool((out[:3] == 7).all()) and bool((out[5:] == 7).all())
    out.fill_(7)
    coral.coral_attention_kv4(q, cache, table, ints([-4, 50, -2 ** 31]), offsets, rows, out=out)
    assert bool((out[:3] == 0).all()) and bool((out[5:] == 0).all()) and torch.equal(out[3:5], want[3:5])
    out.fill_(7)
    coral.coral_attention_kv4(q, cache, table, lengths, offsets, 2, out=out)                            # rows behind the second
    assert bool((out[2] == 7).all()) and bool((out[7:] == 7).all()) and torch.equal(out[3:5], want[3:5])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("most", [1, 2, 3, 7, 40])
@pytest.mark.parametrize("D,q_heads,kv_heads,tree", [(64, 4, 1, False), (128, 8, 8, False), (128, 28, 4, False), (256, 2, 1, False), (128, 8, 2, True)])
def test_attention_kv4_sequences_of_more_rows_than_are_taken(coral, dtype, D, q_heads, kv_heads, tree, most):
    """Of n rows the first `most` are written, and row i still sees what row i of n does."""
    sequences = [(100, 3), (50, 2), (70, 4), (5003, 41), (20, 33), (1, 2)]
    for more in (0, 260) if dtype == "bf16" and D == 64 else (0,):          # (a sequence a workgroup beyond 256 sequences)
        c = Cached(coral, dtype, sequences + [(40, 3)] * more, q_heads, kv_heads, D, 32, tree)
        args, kw = c.args()
        out = torch.full_like(c.q, 7)
        coral.coral_attention_kv4(*args[:5], most, out=out, **kw)
        got = host(out)
        for s, (n, r) in enumerate(c.sequences[:8]):
            k, held = plain.kv4_tokens(*c.sides[0], c.table[s], n, dtype)
            v, _ = plain.kv4_tokens(*c.sides[1], c.table[s], n, dtype)
            a, taken = c.offsets[s], min(r, most)
            want = plain.attention(c.q64[a:a + taken], k, v, c.seen(s)[:taken] & held[None], D ** -0.5)
            check_attention(got[a:a + taken], want, dtype, n, f"sequence {s} of {n} tokens, {taken} of {r} rows")
            assert (got[a + taken:a + r] == 7).all()


def test_attention_kv4_a_query_that_is_not_finite_spoils_only_itself(coral):
    for dtype in DTYPES:
        c = Cached(coral, dtype, [(400, 6), (33, 2)], 4, 2, 128, 32)
        want = c.run()
        c.q[2, 1, 5], c.q[4, 3, 0] = math.nan, math.inf
        got = c.run()
        ok = torch.ones(8, 4, dtype=torch.bool)
        ok[2, 1] = ok[4, 3] = False
        assert torch.equal(got.cpu()[ok], want.cpu()[ok]) and bool(torch.isnan(got[2, 1]).any())


def test_attention_kv4_strided_queries_another_stream_and_graph_replays(coral):
    c = Cached(coral, "bf16", [(900, 4), (77, 2)], 8, 2, 128, 64)
    want = c.run()
    wide = torch.zeros((6, 12, 128), dtype=torch.bfloat16, device="cuda")
    wide[:, 3:11] = c.q
    args, _ = c.args()
    assert torch.equal(coral.coral_attention_kv4(wide[:, 3:11], *args[1:]), want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    other = coral.coral_attention_kv4(*args, stream=stream)
    stream.synchronize()
    assert torch.equal(other, want)
    # one workspace under two graphs, lengths that grow between replays
    ws = torch.zeros(coral.coral_attention_kv4_workspace_bytes(2, 4, 900, 8, 2, 128, coral.CORAL_BF16), dtype=torch.uint8, device="cuda")
    lengths, outs, graphs = args[3].clone(), [torch.zeros_like(want) for _ in range(2)], []
    for out in outs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            coral.coral_attention_kv4(args[0], args[1], args[2], lengths, args[4], 4, max_length=900, out=out, workspace=ws)
        graphs.append(graph)
    for n in (900, 500, 4, 0, 811):
        lengths.copy_(ints([n, 77]))
        eager = coral.coral_attention_kv4(args[0], args[1], args[2], lengths, args[4], 4, max_length=900)
        assert bool((ws[:16896] == 0).all())                      # the counters are as they were
        for graph, out in zip(graphs, outs):
            out.fill_(3)
            graph.replay()
            assert torch.equal(out, eager)


# ---------------------------------------------------------------- prompts
class Prompt:
    def __init__(self, coral, dtype, lengths, q_heads, kv_heads, D, seed=0, behind=0, q_size=1.5):
        rng = np.random.default_rng([seed, q_heads, D, len(lengths)])
        self.coral, self.dtype, self.lengths = coral, dtype, lengths
        n, m = [a for a, _ in lengths], [b for _, b in lengths]
        self.offsets, self.k_offsets = (np.concatenate([[0], np.cumsum(x)]) for x in (n, m))
        self.q, self.q64 = stored(rng.standard_normal((sum(n) + behind, q_heads, D)) * q_size, dtype)
        kv, kv64 = stored(rng.standard_normal((sum(m) + behind, 2 * kv_heads, D)), dtype)
        self.k, self.v, self.k64, self.v64 = kv[:, :kv_heads], kv[:, kv_heads:], kv64[:, :kv_heads], kv64[:, kv_heads:]
        self.same = n == m

    def run(self, **kw):
        return self.coral.coral_attention_prompt(self.q, self.k, self.v, ints(self.offsets), None if self.same else ints(self.k_offsets), **kw)

    def check(self, out, scale=None, rows=None):
        got, D = host(out), self.q.shape[2]
        for s, (n, m) in enumerate(self.lengths):
            pick = np.arange(n) if rows is None or n <= 300 else np.unique(np.r_[0:40, n - 70:n, rng_rows(n, rows)])
            a, b = slice(self.k_offsets[s], self.k_offsets[s + 1]), self.offsets[s] + pick
            seen = np.arange(m)[None] <= (m - n + pick)[:, None]
            want = plain.attention(self.q64[b], self.k64[a], self.v64[a], seen, D ** -0.5 if scale is None else scale)
            check_attention(got[b], want, self.dtype, m, f"sequence {s} of {n} rows, {m} keys")


def rng_rows(n, count):
    return np.random.default_rng(n).integers(0, n, count)


SHORT = [(1, 1), (2, 2), (31, 31), (32, 32), (33, 33), (63, 63), (64, 64), (65, 65), (127, 127), (128, 128), (129, 129), (200, 200)]
BEHIND = [(1, 1), (1, 500), (3, 2), (70, 0), (0, 40), (129, 200), (64, 65), (130, 31), (5, 64), (257, 321)]
SHARED = [(1, 700), (2, 130), (33, 33), (63, 600), (70, 0), (0, 40), (64, 65), (1, 1), (129, 257), (31, 95), (200, 161), (5, 1000)]      # keys shared by groups


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("q_heads,kv_heads", [(1, 1), (8, 2), (7, 1), (12, 12)])
@pytest.mark.parametrize("lengths", [SHORT, BEHIND, SHARED])
def test_attention_prompt(coral, dtype, D, q_heads, kv_heads, lengths):
    c = Prompt(coral, dtype, lengths, q_heads, kv_heads, D)
    out, kept = guarded(c.q.shape, TORCH[dtype])
    c.run(out=out)
    c.check(out)
    kept()
    assert torch.equal(c.run(), out)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,q_heads,kv_heads,lengths", [(128, 8, 2, [(2000, 2000)]), (64, 3, 3, [(1500, 1777), (700, 700)]), (256, 4, 1, [(1111, 1111)]),
                                                        (128, 28, 4, [(1, 3333), (513, 513)])])
def test_attention_prompt_long(coral, dtype, D, q_heads, kv_heads, lengths):
    c = Prompt(coral, dtype, lengths, q_heads, kv_heads, D)
    out = c.run()
    c.check(out, rows=60)
    assert torch.equal(c.run(), out)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,q_heads,kv_heads,lengths", [(64, 160, 16, [(400, 400), (130, 200), (3, 3)]), (128, 160, 32, [(257, 257), (300, 330)]), (256, 96, 8, [(600, 600), (129, 129)])])
def test_attention_prompt_many_heads(coral, dtype, D, q_heads, kv_heads, lengths):
    c = Prompt(coral, dtype, lengths, q_heads, kv_heads, D)
    out, kept = guarded(c.q.shape, TORCH[dtype])
    c.run(out=out)
    c.check(out, rows=20)
    kept()
    assert torch.equal(c.run(), out)


def test_attention_prompt_many_sequences(coral):
    rng = np.random.default_rng(8)
    n = rng.integers(0, 40, 300)
    c = Prompt(coral, "bf16", [(int(a), int(a)) for a in n], 4, 2, 64)
    c.check(c.run())


@pytest.mark.parametrize("count", [64, 65, 257, 2000, 4097])
def test_attention_prompt_sequences_beyond_those_ordered_by_length(coral, count):
    rng = np.random.default_rng(count)
    n = rng.choice([0, 1, 1, 2, 5, 31, 64, 127, 128, 129, 300], count)
    c = Prompt(coral, "bf16", [(int(a), int(a)) for a in n], 3, 1, 64, behind=5)
    out = torch.full_like(c.q, 7)
    c.run(out=out)
    ends = np.concatenate([[0], np.cumsum(n)])
    assert bool((out[ends[-1]:] == 7).all())
    for s in np.unique(np.r_[0:8, count - 8:count, rng.integers(0, count, 40)]):
        rows = slice(ends[s], ends[s + 1])
        want = plain.attention(c.q64[rows], c.k64[rows], c.v64[rows], np.tri(int(n[s]), dtype=bool), 64 ** -0.5)
        check_attention(host(out[rows]), want, "bf16", int(n[s]))
    assert bool((out[:ends[-1]] != 7).any(dim=-1).all())         # no row is left out


def test_attention_prompt_peaked_scores(coral):
    for dtype in DTYPES:
        c = Prompt(coral, dtype, [(300, 300), (40, 90)], 4, 2, 128, q_size=40.0)
        c.check(c.run())
        c.check(c.run(scale=-0.25), scale=-0.25)
        c.check(c.run(scale=0.0), scale=0.0)


def beside_a_large_one(rows, heads, D, down, dtype, rng):
    """Queries, and a key with 2^down times the weight that keys near zero have."""
    q = stored(np.full((rows, heads, D), down * math.log(2) / math.sqrt(D)) * (1 + 0.01 * rng.random((rows, heads, 1))), dtype)
    return (*q, np.ones((1, 1, D)))


def check_beside(got, want, dtype, keys):
    """The large key's score is one number for its whole row: the error of its sum in fp32 moves all values of a row
    together (by less than half of score_off: partial sums are half the whole on average), which is below a half step of
    the 16-bit types and not of fp32, so there each value's own bound is what holds."""
    if dtype != "f32":
        return check_attention(got, want, dtype, keys)
    assert (np.abs(got - want[0]) <= plain.attention_bound(*want, keys, dtype)).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("down", [14.5, 20.0, 22.3, 25.5])
@pytest.mark.parametrize("value", [0.0, 0.5])
@pytest.mark.parametrize("rows,heads,D", [(1, 8, 64), (140, 4, 128), (2, 4, 256)])
def test_attention_prompt_many_small_weights_beside_a_large_one(coral, dtype, down, value, rows, heads, D):
    """As many small weights count by what they come to (the large one's value is nothing, or of the others' size)."""
    rng, n = np.random.default_rng(8), 60000
    q, q64, first = beside_a_large_one(rows, heads, D, down, dtype, rng)
    k, k64 = stored(np.r_[first, 0.05 * rng.standard_normal((n - 1, 1, D))], dtype)
    v, v64 = stored(np.r_[np.full((1, 1, D), value), 4 * rng.random((n - 1, 1, D))], dtype)
    out = coral.coral_attention_prompt(q, k, v, ints([0, rows]), k_offsets=ints([0, n]))
    pick = np.unique(np.r_[0, rows // 2, rows - 1])
    check_beside(host(out)[pick], plain.attention(q64[pick], k64, v64, np.arange(n)[None] <= n - rows + pick[:, None], D ** -0.5), dtype, n)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("down", [22.3, 25.5])
@pytest.mark.parametrize("value", [0x00, 0x11])
@pytest.mark.parametrize("rows,heads,D", [(1, 8, 64), (3, 8, 64), (1, 8, 128), (5, 4, 128), (2, 4, 256)])
def test_attention_kv4_many_small_weights_beside_a_large_one(coral, dtype, down, value, rows, heads, D):
    """The same over the cache: by many workgroups, and (max_length 128) by one, whose waves each pass over a quarter of the keys."""
    rng, n, page = np.random.default_rng(7), 131072, 256
    q, q64, _ = beside_a_large_one(rows, heads, D, down, dtype, rng)
    cache, sides = random_cache(coral, rng, n // page, page, 1, D, scales=(127, 128))
    sides[0][1][:], sides[1][0][:] = 121, sides[1][0] & 0x77       # keys of at most 6/64, values without a sign
    sides[0][0][0, 0, 0], sides[0][1][0, 0, 0], sides[1][0][0, 0, 0] = 0x22, 127, value
    for tensors, arrays in ((cache[:2], sides[0]), (cache[2:], sides[1])):
        for t, a in zip(tensors, arrays):
            t.copy_(torch.from_numpy(a))
    table = np.arange(n // page)
    k, v = (plain.kv4_tokens(*side, table, n, dtype)[0] for side in sides)
    want = plain.attention(q64, k, v, np.arange(n)[None] <= n - rows + np.arange(rows)[:, None], D ** -0.5)
    for most in (None, 128):
        out = coral.coral_attention_kv4(q, cache, ints(table[None]), ints([n]), ints([0, rows]), rows, max_length=most)
        check_beside(host(out), want, dtype, n)


def test_attention_prompt_rows_of_no_sequence_and_offsets_outside(coral):
    c = Prompt(coral, "f16", [(100, 100), (60, 60)], 4, 2, 64, behind=5)
    out, kept = guarded(c.q.shape, torch.float16)
    c.run(out=out)
    c.check(out)
    kept()
    assert bool((out[160:] == 77).all())
    want = out.clone()
    more = torch.full_like(out, 7)
    coral.coral_attention_prompt(c.q, c.k, c.v, ints([-3, 100, 10 ** 6]), out=more)                     # cut to the rows
    assert torch.equal(more[:160], want[:160])
    more.fill_(7)
    coral.coral_attention_prompt(c.q, c.k, c.v, ints([50, 0, 100]), k_offsets=ints([50, 0, 100]), out=more)
    assert torch.equal(more[:100], want[:100]) and bool((more[100:] == 7).all())
    more.fill_(7)
    coral.coral_attention_prompt(c.q, c.k[:0], c.v[:0], ints([0, 100, 160]), k_offsets=ints([0, 0, 0]), out=more)
    assert bool((more[:160] == 0).all()) and bool((more[160:] == 7).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_attention_offsets_of_any_number(coral, dtype):
    """Offsets whose differences pass 32 bits: such sequences have no rows, or no keys."""
    low, high = -2 ** 31, 2 ** 31 - 1
    c = Cached(coral, dtype, [(100, 3), (50, 2), (70, 4)], 4, 1, 64, 32)
    (q, cache, table, lengths, _, rows), _ = c.args()
    out = torch.full_like(q, 7)
    coral.coral_attention_kv4(q, cache, table, lengths, ints([8, low, 5, 0]), 4, out=out)                   # none, [0,5), none
    n, k, v = 50, *(plain.kv4_tokens(*side, c.table[1], 50, dtype)[0] for side in c.sides)
    seen = np.arange(n)[None] <= (n - 5 + np.arange(4))[:, None]                                            # (four of five are taken)
    check_attention(host(out)[:4], plain.attention(c.q64[:4], k, v, seen, 64 ** -0.5), dtype, n)
    assert bool((out[4:] == 7).all())
    for offsets in ([8, low, low, low], [high, low, low, -7], [9, 5, low, -1]):
        out.fill_(7)
        coral.coral_attention_kv4(q, cache, table, lengths, ints(offsets), 4, out=out)
        assert bool((out == 7).all())
    p = Prompt(coral, dtype, [(40, 40), (30, 30)], 4, 2, 64, behind=5)
    want = coral.coral_attention_prompt(p.q[:70], p.k[:70], p.v[:70], ints([0, 40, 70]))
    out = torch.full_like(p.q, 7)
    for offsets in ([60, low, low], [high, low, -5], [75, 74, low]):
        coral.coral_attention_prompt(p.q, p.k, p.v, ints(offsets), out=out)
        assert bool((out == 7).all())
    coral.coral_attention_prompt(p.q, p.k, p.v, ints([60, low, 40]), out=out)                               # none, [0,40)
    assert torch.equal(out[:40], want[:40]) and bool((out[40:] == 7).all())
    out.fill_(7)
    coral.coral_attention_prompt(p.q, p.k, p.v, ints([0, 40, 70]), k_offsets=ints([60, low, low]), out=out)
    assert bool((out[:70] == 0).all()) and bool((out[70:] == 7).all())                                      # rows without keys
    out, kept = guarded(p.q.shape, TORCH[dtype])
    more = ints([75, low] * 40)                                                                             # beyond those ordered by length
    coral.coral_attention_prompt(p.q, p.k, p.v, more, k_offsets=more, out=out)
    kept()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads", [4, 256])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_prompt_values_that_are_not_finite_reach_only_rows_that_see_them(coral, dtype, D, heads):
    lengths = [(150, 150), (70, 100), (40, 40)] + [(1, 300)] * (heads == 4)        # (long enough for groups of waves to share the keys)
    c = Prompt(coral, dtype, lengths, heads, 2, D)
    want = c.run()
    spoiled = [(0, 64), (0, 100), (0, 149), (1, 99), (2, 0)]       # (sequence, key)
    clean = torch.ones(len(c.q), dtype=torch.bool)
    for i, (s, key) in enumerate(spoiled):
        c.v[int(c.k_offsets[s]) + key, 0, 3 + i] = (math.nan, math.inf, -math.inf, math.inf, math.nan)[i]
        c.k[int(c.k_offsets[s]) + key, 0, 2] = (math.inf, math.nan, math.nan, -math.inf, math.inf)[i]
        n, m = lengths[s]
        clean[int(c.offsets[s]) + max(0, key - (m - n)):int(c.offsets[s + 1])] = False
    got = c.run()
    assert torch.equal(got[clean.cuda()], want[clean.cuda()])
    assert torch.equal(got[:, heads // 2:], want[:, heads // 2:])  # heads of the other keys
    c.q[5, 3, 0] = math.nan
    again = c.run()
    rest = clean.clone()
    rest[5] = False
    assert torch.equal(again[rest.cuda()], want[rest.cuda()])
    v_only = Prompt(coral, dtype, lengths, heads, 2, D)            # a value alone makes its later rows not finite
    v_only.v[64, 1, 7] = math.inf
    got = v_only.run()
    assert not bool(torch.isfinite(got[64:150, heads // 2:, 7]).any()) and bool(torch.isfinite(got[:64]).all()) and bool(torch.isfinite(got[150:]).all())


def test_attention_prompt_strides_stream_and_graph(coral):
    rng = np.random.default_rng(3)
    wide = stored(rng.standard_normal((333, 9, 128)), "bf16")[0]
    offsets = ints([0, 100, 333])
    q, k, v = wide[:, :6], wide[:, 6:7], wide[:, 8:]
    want = coral.coral_attention_prompt(q.contiguous(), k.contiguous(), v.contiguous(), offsets)
    assert torch.equal(coral.coral_attention_prompt(q, k, v, offsets), want)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    other = coral.coral_attention_prompt(q, k, v, offsets, stream=stream)
    stream.synchronize()
    assert torch.equal(other, want)
    out, graph = torch.zeros_like(want), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        coral.coral_attention_prompt(q, k, v, offsets, out=out)
    for cut in (100, 1, 333, 128):
        offsets.copy_(ints([0, cut, 333]))
        eager = coral.coral_attention_prompt(q, k, v, offsets)
        out.fill_(3)
        graph.replay()
        assert torch.equal(out, eager)


# ---------------------------------------------------------------- far places, many rows, several streams, graphs
def test_cache_past_32_bits(coral):
    """A cache whose codes take more than 4 GiB on either side: its last pages answer as a small cache's do."""
    page, kv_heads, D, pages = 256, 8, 256, 17000
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GiB of free memory")
    big, small = coral.alloc_kv4_cache(pages, page, kv_heads, D), coral.alloc_kv4_cache(4, page, kv_heads, D)
    assert big[0].numel() > 1 << 32
    n = 700
    k, v = (torch.randn((n, kv_heads, D), dtype=torch.bfloat16, device="cuda", generator=torch.Generator("cuda").manual_seed(s)) for s in (1, 2))
    held = [pages - 1, 16400, pages - 2]                          # pages on both sides of the border and the last
    place = np.arange(n)
    slots = ints(np.asarray(held)[place // page] * page + place % page)
    coral.coral_kv4_append(big, k, v, slots)
    coral.coral_kv4_append(small, k, v, ints(place))
    for a, b in zip(coral.coral_kv4_read(big, slots, torch.bfloat16), coral.coral_kv4_read(small, ints(place), torch.bfloat16)):
        assert torch.equal(a, b)
    q = torch.randn((5, 16, D), dtype=torch.bfloat16, device="cuda")
    got, want = (coral.coral_attention_kv4(q, cache, ints([table]), ints([n]), ints([0, 5]), 5) for cache, table in ((big, held), (small, [0, 1, 2])))
    assert torch.equal(got, want) and bool(got.any())
    weight, at = torch.ones(D, dtype=torch.bfloat16, device="cuda"), ints(np.arange(n) + 10 ** 6)
    kw = dict(positions=at, inv_freq=torch.full((64,), 0.01, device="cuda"), k_weight=weight, v=v)
    assert torch.equal(coral.coral_qk_norm_rope(None, k, cache=big, slots=slots, **kw)[1], coral.coral_qk_norm_rope(None, k, cache=small, slots=ints(place), **kw)[1])
    for a, b in zip(coral.coral_kv4_read(big, slots, torch.bfloat16), coral.coral_kv4_read(small, ints(place), torch.bfloat16)):
        assert torch.equal(a, b)
    assert int(big[1].sum(dtype=torch.int64)) == int(small[1].sum(dtype=torch.int64))        # and nothing elsewhere


def test_rows_past_32_bits(coral):
    """Rows of one wide matrix, the last of them more than 4 GiB behind the first."""
    T, wide = 300, 1 << 23
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GiB of free memory")
    rows = torch.zeros((T, wide), dtype=torch.bfloat16, device="cuda")
    near = torch.randn((T, 8, 128), dtype=torch.bfloat16, device="cuda")
    rows[:, -1024:] = near.view(T, 1024)
    far = rows[:, -1024:].unflatten(1, (8, 128))
    offsets = ints([0, 140, 300])
    for a, b in zip(coral.coral_qk_norm_rope(far[:, :4], far[:, 4:6]), coral.coral_qk_norm_rope(near[:, :4], near[:, 4:6])):
        assert torch.equal(a, b)
    assert torch.equal(coral.coral_attention_prompt(far[:, :4], far[:, 4:6], far[:, 6:], offsets), coral.coral_attention_prompt(near[:, :4], near[:, 4:6], near[:, 6:], offsets))
    one, two = (coral.alloc_kv4_cache(20, 16, 2, 128) for _ in range(2))
    slots = ints(np.arange(T)[::-1].copy())
    coral.coral_kv4_append(one, far[:, 4:6], far[:, 6:], slots)
    coral.coral_kv4_append(two, near[:, 4:6], near[:, 6:], slots)
    assert all(torch.equal(a, b) for a, b in zip(one, two))
    table = ints([np.arange(20)] * 60)
    args = (ints([300] * 60), ints(np.arange(61) * 5), 5)
    assert torch.equal(coral.coral_attention_kv4(far[:, :4], one, table, *args), coral.coral_attention_kv4(near[:, :4], one, table, *args))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("q_heads,kv_heads,D", [(14, 2, 64), (9, 9, 128), (6, 3, 256)])
def test_attention_kv4_many_rows_joined_several_heads_a_wave(coral, dtype, q_heads, kv_heads, D):
    c = Cached(coral, dtype, [(20 + 11 * (s % 50), 20) for s in range(110)], q_heads, kv_heads, D, 32, behind=2)
    out = torch.full_like(c.q, 7)
    c.run(out=out)
    c.check(out, only=[0, 1, 30, 49, 50, 77, 108, 109])
    assert bool((out[2200:] == 7).all()) and bool((out[:2200] != 7).any(dim=-1).all())
    assert torch.equal(c.run()[:2200], out[:2200])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 2, 3])
def test_attention_kv4_one_long_sequence_among_short_ones(coral, dtype, rows):
    """Joined as if parts were few, where one item has hundreds: in two steps, whose counters are zero again behind each call."""
    for q_heads, kv_heads, D in ((8, 2, 64), (8, 4, 128), (4, 1, 256)):
        c = Cached(coral, dtype, [(5 + s % 3, 1) for s in range(40)] + [(60000, rows)] + [(9, 2)] * 20, q_heads, kv_heads, D, 128)
        ws = torch.zeros(coral.coral_attention_kv4_workspace_bytes(61, rows, 70000, q_heads, kv_heads, D, coral._dtype_code(c.q)), dtype=torch.uint8, device="cuda")
        out = c.run(max_length=70000, workspace=ws)
        c.check(out, only=[0, 39, 40, 41, 60])
        for _ in range(5):
            assert torch.equal(c.run(max_length=70000, workspace=ws), out) and bool((ws[:16896] == 0).all())


def test_attention_kv4_more_rows_than_a_grid_has_in_its_second_part(coral):
    c = Cached(coral, "bf16", [(150 + s % 7, 64) for s in range(1030)], 2, 1, 64, 32, tree=True)
    out = c.run()
    assert out.shape[0] > 65535
    c.check(out, only=[0, 511, 1022, 1023, 1024, 1029])


def test_two_calls_at_once_on_two_streams(coral):
    cases = [Cached(coral, "bf16", [(4000, 3), (70, 1)], 8, 2, 128, 64, seed=s) for s in range(2)]
    want = [c.run() for c in cases]
    calls = [(c.args()[0], torch.zeros(coral.coral_attention_kv4_workspace_bytes(2, 3, 4032, 8, 2, 128, coral.CORAL_BF16), dtype=torch.uint8, device="cuda"),
              torch.zeros_like(w), torch.cuda.Stream()) for c, w in zip(cases, want)]
    torch.cuda.synchronize()
    for _ in range(20):
        for args, ws, out, stream in calls:
            coral.coral_attention_kv4(*args, max_length=4032, out=out, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(out, w) for (_, _, out, _), w in zip(calls, want))


def test_attention_kv4_workspace_made_ready_by_its_call(coral):
    c = Cached(coral, "f16", [(3000, 2), (500, 7)], 8, 2, 64, 16)
    want = c.run()
    ws = torch.full((coral.coral_attention_kv4_workspace_bytes(2, 7, 4000, 8, 2, 64, coral.CORAL_F16),), 0xff, dtype=torch.uint8, device="cuda")
    coral.coral_lmhead_workspace_init(ws)
    args, _ = c.args()
    for _ in range(3):
        assert torch.equal(coral.coral_attention_kv4(*args, max_length=4000, workspace=ws), want)


# ---------------------------------------------------------------- a drafter's layer
class Layer:
    """Projections of 4 bits, norms and rotation into the cache, attention, and the projection back onto the
    residual; every step is checked against its definition, on the inputs that the device gave it."""

    def __init__(self, coral, dtype, H, q_heads, kv_heads, D, pages, page):
        self.coral, self.dtype, self.n, self.D, self.page = coral, dtype, (q_heads, kv_heads), D, page
        rng = self.rng = np.random.default_rng([H, q_heads, kv_heads, D])
        self.weights = [self.projection(H, (q_heads + 2 * kv_heads) * D), self.projection(q_heads * D, H)]
        self.norms = [stored(1 + 0.2 * rng.standard_normal(D), dtype) for _ in range(2)]
        self.freq = np.power(10000.0, -np.arange(D // 2) * 2 / D).astype(np.float32)
        self.cache, self.sides = random_cache(coral, rng, pages, page, kv_heads, D, scales=(124, 128))

    def projection(self, K, N):
        codes = self.rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
        scales = stored(0.2 * (1 + self.rng.random((N, K // 64))) / math.sqrt(K), self.dtype)
        return torch.from_numpy(codes).cuda(), scales[0], codes, scales[1]

    def project(self, x, which, residual=None):
        codes, scales, codes64, scales64 = self.weights[which]
        out = self.coral.coral_matvec_w4(x, codes, scales, group=64, residual=residual, out_dtype=x.dtype)
        args = (host(x), codes64, scales64, None, 64, "int", None, None if residual is None else host(residual))
        assert (np.abs(host(out) - operators.matvec_w4(*args)) <= operators.matvec_w4_bound(*args, out=self.dtype)).all()
        return out

    def into_cache(self, x, at, slots):
        """(q, k, v) of tokens x at positions `at`; k and v also in places `slots` of the cache."""
        qh, kh = self.n
        qkv = self.project(x, 0).unflatten(1, (qh + 2 * kh, self.D))
        q, k, v = qkv[:, :qh], qkv[:, qh:qh + kh], qkv[:, qh + kh:]
        out = self.coral.coral_qk_norm_rope(q, k, ints(at), torch.from_numpy(self.freq).cuda(), self.norms[0][0], self.norms[1][0],
                                            cache=self.cache, v=v, slots=ints(slots))
        for got, x64, (_, w) in zip(out, (host(q), host(k)), self.norms):
            want, bound = (f(x64, np.asarray(at), self.freq, w, 1e-6, False, *more) for f, more in ((plain.norm_rope, ()), (plain.norm_rope_bound, (self.dtype,))))
            assert (np.abs(host(got) - want) <= bound).all()
        for (codes, scales), part in zip(self.sides, (host(out[1]), host(v))):
            codes[slots // self.page, :, slots % self.page], scales[slots // self.page, :, slots % self.page] = plain.kv4_quantise(part, self.dtype)
        for got, want in zip(self.cache, (*self.sides[0], *self.sides[1])):
            assert np.array_equal(got.cpu().numpy(), want)
        return out[0], out[1], v

    def back(self, attended, x):
        y = self.project(attended.flatten(1), 1, residual=x)
        return y, (y.float() * torch.rsqrt(y.float().square().mean(1, keepdim=True))).to(y.dtype)


@pytest.mark.parametrize("dtype,q_heads,kv_heads,D", [("bf16", 8, 2, 64), ("f16", 4, 4, 128), ("f32", 7, 1, 64), ("bf16", 2, 1, 256)])
def test_a_drafters_layer_from_prompt_to_tree(coral, dtype, q_heads, kv_heads, D):
    cfg = CONFIGS["tiny_f32"].scaled(dtype=dtype, H=256, V=4096)
    head = make_head(cfg)
    gate, lm = (coral.device_tensor(w, dtype) for w in (head.gate_W, head.lm_W))
    gi = coral.GroupIndex(head.group_offsets, head.group_rows)
    layer = Layer(coral, dtype, 256, q_heads, kv_heads, D, pages=12, page=16)
    embed = lambda ids: (lm[ids.long()].float() * 50).to(lm.dtype)        # noqa: E731  (the rows' 0.02 to about one)
    prompts, width, k = [40, 23], 6, 5
    table = layer.rng.permutation(12)[:8].reshape(2, 4)
    place = lambda s, at: table[s][at // 16] * 16 + at % 16       # noqa: E731
    # the prompts, one behind the other
    x = embed(torch.from_numpy(layer.rng.integers(0, cfg.V, sum(prompts))).cuda())
    at = np.concatenate([np.arange(n) for n in prompts])
    slots = np.concatenate([place(s, np.arange(n)) for s, n in enumerate(prompts)])
    q, keys, values = layer.into_cache(x, at, slots)
    offsets = np.array([0, 40, 63])
    out = coral.coral_attention_prompt(q, keys, values, ints(offsets))
    for s, n in enumerate(prompts):
        r = slice(offsets[s], offsets[s + 1])
        want = plain.attention(host(q)[r], host(keys)[r], host(values)[r], np.tri(n, dtype=bool), D ** -0.5)
        check_attention(host(out)[r], want, dtype, n)
    _, hidden = layer.back(out, x)
    hidden = hidden[[39, 62]]
    # three levels of a tree behind each prompt
    score, paths, held = [None, None], [[], []], [0, 0]           # paths: a node's ancestors and itself, as bits from the prompt's end
    nodes = [hidden[:1], hidden[1:]]
    for depth in range(3):
        tokens, words = [], []
        for s in range(2):
            ids, logp, sel, parent, token, total = coral.coral_lmhead_draft_level(nodes[s].contiguous(), gate, None, lm, gi, cfg.g, k, width if depth else k, parent_score=score[s])
            as_host = nodes[s].contiguous()
            as_host = host(as_host).astype(np.float32) if dtype == "f32" else as_host.view(torch.int16).cpu().numpy().view(np.uint16)
            compare.check_grouped_logprob(as_host, head.gate_W, None, head.lm_W, head.group_offsets, head.group_rows, cfg.g, k, dtype, *(t.cpu().numpy() for t in (ids, logp, sel)))
            first = held[s]
            old = paths[s][-1] if depth else [0]
            paths[s].append([old[p] | 1 << (first + i) for i, p in enumerate(parent.cpu().tolist())])
            held[s] += len(paths[s][-1])
            score[s] = total
            tokens.append(token)
            words.append(paths[s][-1])
        rows = [len(w) for w in words]
        x = embed(torch.cat(tokens))
        at = np.concatenate([np.full(r, prompts[s] + depth) for s, r in enumerate(rows)])
        slots = np.concatenate([place(s, prompts[s] + np.arange(held[s] - rows[s], held[s])) for s in range(2)])
        q = layer.into_cache(x, at, slots)[0]
        tree = np.array(words[0] + words[1], dtype=np.int64)
        offsets, lengths = np.concatenate([[0], np.cumsum(rows)]), [n + h for n, h in zip(prompts, held)]
        out = coral.coral_attention_kv4(q, layer.cache, ints(table), ints(lengths), ints(offsets), max(rows), history=ints(prompts), tree=torch.from_numpy(tree).cuda())
        for s, n in enumerate(lengths):
            r = slice(offsets[s], offsets[s + 1])
            (kk, _), (vv, _) = (plain.kv4_tokens(*side, table[s], n, dtype) for side in layer.sides)
            seen = np.ones((rows[s], n), bool)
            seen[:, prompts[s]:] = (tree[r, None] >> np.arange(held[s])) & 1 == 1
            assert (seen[:, prompts[s]:].sum(axis=1) == depth + 1).all()
            check_attention(host(out)[r], plain.attention(host(q)[r], kk, vv, seen, D ** -0.5), dtype, n)
        _, hidden = layer.back(out, x)
        nodes = [hidden[:rows[0]], hidden[rows[0]:]]


def test_a_layer_in_one_graph_as_eagerly(coral):
    """Projection, norms and rotation into the cache, attention and the projection back as one graph: replays
    with tokens, places and lengths that change between them give what eager calls give."""
    graph_side, eager_side = (Layer(coral, "bf16", 256, 8, 2, 64, pages=12, page=16) for _ in range(2))
    x, at, slots = torch.zeros((3, 256), dtype=torch.bfloat16, device="cuda"), ints([0] * 3), ints([-1] * 3)
    table, offsets, lengths = ints(np.arange(12).reshape(1, 12)), ints([0, 3]), ints([0])
    freq = torch.from_numpy(graph_side.freq).cuda()
    ws = torch.zeros(coral.coral_attention_kv4_workspace_bytes(1, 3, 192, 8, 2, 64, coral.CORAL_BF16), dtype=torch.uint8, device="cuda")

    def step(layer, workspace=None):
        (codes, scales, _, _), (codes2, scales2, _, _) = layer.weights
        qkv = coral.coral_matvec_w4(x, codes, scales, group=64, out_dtype=x.dtype).unflatten(1, (12, 64))
        q, _ = coral.coral_qk_norm_rope(qkv[:, :8], qkv[:, 8:10], at, freq, layer.norms[0][0], layer.norms[1][0], k_out=False, cache=layer.cache, v=qkv[:, 10:], slots=slots)
        out = coral.coral_attention_kv4(q, layer.cache, table, lengths, offsets, 3, workspace=workspace)
        return coral.coral_matvec_w4(out.flatten(1), codes2, scales2, group=64, residual=x, out_dtype=x.dtype)

    step(graph_side, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(graph_side, ws)
    for first in (0, 3, 90, 15, 189):
        x.copy_(torch.from_numpy(graph_side.rng.standard_normal((3, 256))))
        at.copy_(ints(first + np.arange(3)))
        slots.copy_(at)
        lengths.copy_(ints([first + 3]))
        want = step(eager_side)
        torch.cuda.synchronize()
        graph.replay()
        assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(graph_side.cache, eager_side.cache))


# ---------------------------------------------------------------- binding
def test_binding_refuses_other_shapes_types_and_places(coral):
    q, k = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    cache, ids, offsets = coral.alloc_kv4_cache(2, 16, 2, 64), ints([0, 1, 2]), ints([0, 3])
    table, lengths = ints([[0, 1]]), ints([3])
    for error, call in [
            (TypeError, lambda: coral.coral_qk_norm_rope(q, k.float())), (ValueError, lambda: coral.coral_qk_norm_rope(q, k[:2])),
            (ValueError, lambda: coral.coral_qk_norm_rope(q, k, positions=ids)), (ValueError, lambda: coral.coral_qk_norm_rope(q, k, cache=cache)),
            (ValueError, lambda: coral.coral_qk_norm_rope(q, k, k_out=False)), (TypeError, lambda: coral.coral_qk_norm_rope(q, k, q_weight=torch.ones(64, device="cuda"))),
            (ValueError, lambda: coral.coral_qk_norm_rope(q, k.cpu())), (ValueError, lambda: coral.coral_qk_norm_rope(q, k, q_out=k)),
            (coral.CoralError, lambda: coral.coral_qk_norm_rope(q[..., :48].contiguous(), None)),
            (TypeError, lambda: coral.coral_kv4_append(cache, k, k.half(), ids)), (ValueError, lambda: coral.coral_kv4_append(cache, q, q, ids)),
            (TypeError, lambda: coral.coral_kv4_append(cache, k, k, ids.long())), (ValueError, lambda: coral.coral_kv4_append(cache, k, k, ids[:2])),
            (TypeError, lambda: coral.coral_kv4_read(cache, ids, torch.float64)), (ValueError, lambda: coral.coral_kv4_read(cache, ids, k.dtype, k_out=k[:2])),
            (ValueError, lambda: coral.coral_kv4_append((cache[0], cache[0], cache[2], cache[3]), k, k, ids)),
            (ValueError, lambda: coral.coral_attention_kv4(q[:, :, :32].contiguous(), cache, table, lengths, offsets, 3)),
            (ValueError, lambda: coral.coral_attention_kv4(q, cache, table[0], lengths, offsets, 3)), (TypeError, lambda: coral.coral_attention_kv4(q, cache, table, lengths.long(), offsets, 3)),
            (ValueError, lambda: coral.coral_attention_kv4(q, cache, table, lengths, offsets[:1], 3)), (coral.CoralError, lambda: coral.coral_attention_kv4(q, cache, table, lengths, offsets, 65)),
            (coral.CoralError, lambda: coral.coral_attention_kv4(q, cache, table, lengths, offsets, 3, tree=torch.zeros(3, dtype=torch.int64, device="cuda"))),
            (coral.CoralError, lambda: coral.coral_attention_kv4(q[:, :3].contiguous(), cache, table, lengths, offsets, 3)),
            (ValueError, lambda: coral.coral_attention_prompt(q, k, k[:2], offsets)), (TypeError, lambda: coral.coral_attention_prompt(q, k, k.half(), offsets)),
            (coral.CoralError, lambda: coral.coral_attention_prompt(q, torch.cat([k, k]), torch.cat([k, k]), offsets)),
            (ValueError, lambda: coral.coral_attention_prompt(q, k.transpose(0, 1), k, offsets))]:
        with pytest.raises(error):
            call()


def test_calls_without_tokens(coral):
    q, k = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    cache, none = coral.alloc_kv4_cache(2, 16, 2, 64), ints(np.zeros(0, int))
    assert coral.coral_qk_norm_rope(q, k, positions=none, inv_freq=torch.ones(32, device="cuda"))[0].shape == (0, 4, 64)
    coral.coral_kv4_append(cache, k, k, none)
    assert coral.coral_kv4_read(cache, none, torch.float16)[1].shape == (0, 2, 64)
    assert coral.coral_attention_kv4(q, cache, ints([[0, 1]]), ints([5]), ints([0, 0]), 1).shape == (0, 4, 64)
    assert coral.coral_attention_prompt(q, k, k, ints([0, 0])).shape == (0, 4, 64)
