"""The 4-bit products and the rules on logits on a real MI355X against their 64-bit definitions
(oracle/operators.py), and the step they make up together: 4-bit head, rules, candidates, tree level.

Tolerances come from the arithmetic (matvec_w4_bound, logit_rules' error): the products' sums stay
within the worst case of fp32 sums in any order, and beside it their relative error over a matrix
within 2e-6, five times what sums of random terms of this kind come to: a term of size t adds a
rounding of at most 2^-24 of a partial sum of about sqrt(n) times six t (the codes' offset), averaged
over signs about 2e-7 to 4e-7 of the result."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from oracle import operators as plain  # noqa: E402
import oracle  # noqa: E402

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


def guarded(shape, dtype):
    """A tensor in the middle of a larger one that holds a pattern, and a check that the rest kept it."""
    n = int(np.prod(shape))
    size = torch.empty(0, dtype=dtype).element_size()
    pad = 256 // size
    whole = torch.full((n + 2 * pad,), 77, dtype=dtype, device="cuda")

    def check():
        assert bool((whole[:pad] == 77).all()) and bool((whole[pad + n:] == 77).all()), "written outside the output"
    return whole[pad:pad + n].view(shape), check


# ---------------------------------------------------------------- 4-bit products
class Product:
    def __init__(self, dtype, M, N, K, group, kind="int", zeros=True, bias=False, residual=False, seed=0):
        rng = np.random.default_rng([seed, M, N, K, group])
        self.dtype, self.group, self.kind, groups = dtype, group, kind, -(-K // group)
        self.x, self.x64 = stored(rng.standard_normal((M, K)), dtype)
        self.codes_host = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
        self.scales, self.scales64 = stored((0.5 + rng.random((N, groups))) * 0.01 * rng.choice([-1.0, 1.0], (N, groups)), dtype)
        self.zeros_host = rng.integers(0, 16, (N, groups), dtype=np.uint8) if zeros and kind == "int" else None
        self.bias_host = rng.standard_normal(N).astype(np.float32) if bias else None
        self.residual, self.residual64 = stored(rng.standard_normal((M, N)), dtype) if residual else (None, None)
        self.codes = torch.from_numpy(self.codes_host).cuda()
        self.zeros = None if self.zeros_host is None else torch.from_numpy(self.zeros_host).cuda()
        self.bias = None if self.bias_host is None else torch.from_numpy(self.bias_host).cuda()

    def run(self, coral, act="identity", **kw):
        args = dict(zeros=self.zeros, group=self.group, code_type=self.kind, bias=self.bias, residual=self.residual, act=act)
        args.update(kw)
        return coral.coral_matvec_w4(self.x, self.codes, self.scales, **args)

    def check(self, y, act="identity", rows=slice(None)):
        out = {v: n for n, v in TORCH.items()}[y.dtype]
        pick = lambda a: None if a is None else a[rows]                             # noqa: E731
        args = dict(zeros=pick(self.zeros_host), group=self.group, kind=self.kind, bias=pick(self.bias_host),
                    residual=None if self.residual64 is None else self.residual64[:, rows], act=act)
        want = plain.matvec_w4(self.x64, self.codes_host[rows], self.scales64[rows], **args)
        bound = plain.matvec_w4_bound(self.x64, self.codes_host[rows], self.scales64[rows], out=out, **args)
        got = y.double().cpu().numpy()[:, rows]
        off = np.abs(got - want)
        assert (off <= bound).all(), f"off by {off.max():.3g} at {np.unravel_index((off - bound).argmax(), off.shape)}"
        norm = np.linalg.norm(want)
        if norm > 0:
            assert np.linalg.norm(off) <= (2e-6 + 2 * plain.HALF_STEP[out] * (out != "f32")) * norm


SIZES = [(1, 1, 8, 32), (1, 16, 128, 128), (2, 17, 40, 32), (3, 5, 264, 64), (4, 33, 384, 384), (5, 257, 1032, 128), (7, 50, 2568, 32),
         (8, 64, 4096, 128), (15, 31, 520, 64), (16, 100, 4104, 256), (17, 129, 768, 128), (31, 40, 992, 32), (33, 70, 1280, 64),
         (48, 48, 136, 128), (64, 15, 3584, 128), (64, 300, 4096, 32), (1, 1000, 14336, 128), (20, 34, 14336, 64)]


@pytest.mark.parametrize("kind,zeros", [("int", False), ("int", True), ("e2m1", False)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K,group", SIZES)
def test_matvec_w4(coral, dtype, kind, zeros, M, N, K, group):
    c = Product(dtype, M, N, K, group, kind, zeros)
    y, untouched = guarded((M, N), torch.float32)
    c.run(coral, out=y)
    c.check(y)
    untouched()
    assert torch.equal(c.run(coral), y)                            # the same bits every time


@pytest.mark.parametrize("kind,zeros", [("int", False), ("int", True), ("e2m1", False)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K", [(4, 4096), (20, 2048), (7, 1000), (33, 4096)])
def test_matvec_w4_many_tiles_a_workgroup(coral, dtype, kind, zeros, group, M, K):
    N = 20011
    c = Product(dtype, M, N, K, group, kind, zeros, seed=8)
    runs = [c.run(coral) for _ in range(4)]
    assert all(torch.equal(y, runs[0]) for y in runs) and bool(torch.isfinite(runs[0]).all())
    c.check(runs[0], rows=np.unique(np.r_[0:200, N - 200:N, 0:N:53]))


# many tokens and many rows, one and two rounds of workgroups, the last ones not full
MANY = [(64, 55700, 136, 32), (33, 139300, 136, 64), (50, 83600, 392, 128), (63, 83601, 8, 32), (64, 60001, 1032, 256), (40, 90000, 256, 64),
        (64, 110001, 136, 32), (33, 131072, 264, 64), (50, 106000, 392, 128), (63, 120017, 8, 32), (64, 215000, 40, 256), (49, 105700, 1032, 64)]


@pytest.mark.parametrize("kind,zeros", [("int", False), ("int", True), ("e2m1", False)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K,group", MANY)
def test_matvec_w4_many_rows(coral, dtype, kind, zeros, M, N, K, group):
    c = Product(dtype, M, N, K, group, kind, zeros, seed=5)
    y, untouched = guarded((M, N), torch.float32)
    c.run(coral, out=y)
    rows = np.unique(np.r_[0:700, N - 700:N, 0:N:97])
    c.check(y, rows=rows)
    untouched()
    assert bool(torch.isfinite(y).all()) and torch.equal(c.run(coral), y)
    few = Product(dtype, 16, N, K, group, kind, zeros, seed=5)     # the same rows through the other kernel
    few.x, few.codes, few.scales, few.zeros = c.x[:16].contiguous(), c.codes, c.scales, c.zeros
    want = few.run(coral)
    assert float((y[:16] - want).abs().max()) <= 1e-4 * float(want.abs().max())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_matvec_w4_many_rows_epilogue(coral, dtype):
    M, N, K = 45, 108000, 200
    c = Product(dtype, M, N, K, 64, bias=True, residual=True, seed=6)
    y, untouched = guarded((M, N), TORCH[dtype])
    c.run(coral, "silu", out=y)
    c.check(y, "silu", rows=np.r_[0:300, N - 300:N])
    untouched()
    same = c.residual.clone()
    assert torch.equal(c.run(coral, "silu", residual=same, out=same), y)


@pytest.mark.parametrize("N", [33, 83600, 110000])
@pytest.mark.parametrize("K,group", [(40, 32), (200, 64), (648, 128)])
@pytest.mark.parametrize("M", [3, 50])
def test_matvec_w4_infinite_scales_of_a_rows_last_group(coral, M, N, K, group):
    c = Product("bf16", M, N, K, group, seed=7)
    c.scales[1::2, -1] = float("inf")
    y = c.run(coral)
    first = (K - 1) // group * group
    w = torch.from_numpy(plain.unpack(c.codes_host[1::2, first // 2:]).astype(np.float32)).cuda()
    zero = c.zeros[1::2, -1:].float()
    last = c.x[:, first:].float() @ (w - zero).t()
    sure = last.abs() > 1e-3
    assert torch.equal(y[:, 1::2][sure], (last.sign() * float("inf"))[sure]) and bool(torch.isfinite(y[:, ::2]).all())


# Every form of the kernel that takes tiles of rows one after the other (units of columns a wave, tiles of tokens, passes,
# fp32 parts one after the other or spread), few rows and the last of them and of the columns not full.
FORMS = [(M, K) for M in (1, 5, 16, 20) for K in (1000, 2040, 2568, 4040, 4104, 5000, 7000, 8184, 9000)] + [(11, 4096), (50, 2568), (50, 8200), (64, 4104)]


@pytest.mark.parametrize("kind,zeros", [("int", False), ("int", True), ("e2m1", False)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K", FORMS)
def test_matvec_w4_forms(coral, dtype, kind, zeros, group, M, K):
    N = 83
    c = Product(dtype, M, N, K, group, kind, zeros, seed=11)
    y, untouched = guarded((M, N), torch.float32)
    c.run(coral, out=y)
    c.check(y)
    untouched()
    assert torch.equal(c.run(coral), y)


# Columns in passes, more tiles a workgroup than a block holds the sums of.
PASSES = [("bf16", 2, 110011, 8328), ("f16", 20, 110011, 4232), ("f32", 3, 200003, 4232), ("f32", 9, 110011, 4232)]


@pytest.mark.parametrize("kind,zeros", [("int", False), ("int", True), ("e2m1", False)])
@pytest.mark.parametrize("group", [32, 64, 384])
@pytest.mark.parametrize("dtype,M,N,K", PASSES)
def test_matvec_w4_passes_over_many_rows(coral, dtype, kind, zeros, group, M, N, K):
    gen = torch.Generator("cuda").manual_seed(N + K + group)
    x, x64 = stored(np.random.default_rng(12).standard_normal((M, K)), dtype)
    codes = torch.randint(0, 256, (N, K // 2), generator=gen, device="cuda", dtype=torch.uint8)
    scales = ((0.5 + torch.rand((N, -(-K // group)), generator=gen, device="cuda")) * 0.01).to(TORCH[dtype])
    zero = torch.randint(0, 16, scales.shape, generator=gen, device="cuda", dtype=torch.uint8) if zeros else None
    runs = [coral.coral_matvec_w4(x, codes, scales, zero, group=group, code_type=kind) for _ in range(3)]
    assert bool(torch.isfinite(runs[0]).all()) and all(torch.equal(y, runs[0]) for y in runs)
    at = np.unique(np.r_[0:40, N - 40:N, 0:N:701])
    on = torch.from_numpy(at).cuda()
    args = (codes[on].cpu().numpy(), scales[on].double().cpu().numpy(), None if zero is None else zero[on].cpu().numpy(), group, kind)
    want, bound = plain.matvec_w4(x64, *args), plain.matvec_w4_bound(x64, *args)
    off = np.abs(runs[0][:, on].double().cpu().numpy() - want)
    assert (off <= bound).all() and np.linalg.norm(off) <= 2e-6 * np.linalg.norm(want)
    # a workgroup's first and last tiles, and those at the ends of its blocks: rows of a matrix of ones
    ones = torch.full_like(codes, 0x99 if kind == "int" else 0x22)
    flat = torch.ones_like(scales)
    y = coral.coral_matvec_w4(torch.ones_like(x), ones, flat, None, group=group, code_type=kind)
    assert bool((y == K).all())


# Many tokens and rows that fill the rounds of the kernel for them, beside the shapes above.
MANY_ROWS = [(64, 96017, 136, 32), (33, 96100, 392, 64), (50, 100003, 264, 128), (63, 131072, 8, 32), (64, 192100, 1032, 256), (40, 200001, 256, 64)]


@pytest.mark.parametrize("kind,zeros", [("int", False), ("int", True), ("e2m1", False)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K,group", MANY_ROWS)
def test_matvec_w4_many_rows_against_few_tokens(coral, dtype, kind, zeros, M, N, K, group):
    test_matvec_w4_many_rows(coral, dtype, kind, zeros, M, N, K, group)


INFINITE_ROWS = [96033, 192200]


@pytest.mark.parametrize("N", INFINITE_ROWS)
@pytest.mark.parametrize("K,group", [(40, 32), (200, 64), (648, 128)])
def test_matvec_w4_infinite_scales_with_many_rows(coral, N, K, group):
    test_matvec_w4_infinite_scales_of_a_rows_last_group(coral, 50, N, K, group)


@pytest.mark.parametrize("act", ["identity", "silu", "relu"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K", [(1, 512, 512), (9, 131, 1024), (40, 77, 640)])
def test_matvec_w4_epilogue(coral, dtype, act, M, N, K):
    c = Product(dtype, M, N, K, 128, bias=True, residual=True, seed=1)
    y, untouched = guarded((M, N), TORCH[dtype])
    c.run(coral, act, out=y)
    c.check(y, act)
    untouched()
    c.check(c.run(coral, act), act)                                # fp32 results
    same = c.residual.clone()
    assert torch.equal(c.run(coral, act, residual=same, out=same), y)      # over the residual


def test_matvec_w4_is_the_premix_of_a_router(coral):
    """act = silu, residual = x: what coral_router_premix computes from the same weights in 16 bits."""
    H, M = 512, 6
    c = Product("bf16", M, H, H, 128, zeros=False, seed=2)
    c.residual, c.residual64 = c.x, c.x64
    u = c.run(coral, "silu", out_dtype=torch.bfloat16)
    c.check(u, "silu")
    c.scales.fill_(1 / 64)                                         # weights that bf16 holds exactly
    w = torch.from_numpy((plain.unpack(c.codes_host).astype(np.float32) - 8) / 64).bfloat16().cuda()
    u, want = c.run(coral, "silu", out_dtype=torch.bfloat16), coral.coral_router_premix(c.x, w, "silu")
    assert float((u.float() - want.float()).abs().max()) <= 2 * 2.0 ** -8 * float(want.abs().max())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("M", [4, 16, 50])
def test_matvec_w4_tokens_are_independent(coral, bad, M):
    c = Product("bf16", M, 96, 512, 64, seed=3)
    y = c.run(coral)
    c.x[M // 2, 100] = bad
    z = c.run(coral)
    keep = [m for m in range(M) if m != M // 2]
    assert torch.equal(z[keep], y[keep])


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("kind,zeros,group", [("int", True, 32), ("int", False, 64), ("int", True, 128), ("e2m1", False, 32), ("e2m1", False, 128)])
def test_matvec_w4_tokens_are_independent_with_many_rows(coral, bad, kind, zeros, group):
    M = 50
    c = Product("bf16", M, 110000, 264, group, kind, zeros, seed=9)
    y = c.run(coral)
    c.x[M // 2, 100] = bad
    z = c.run(coral)
    keep = [m for m in range(M) if m != M // 2]
    assert torch.equal(z[keep], y[keep])


def test_matvec_w4_zero_scales_and_extreme_values(coral):
    c = Product("f32", 3, 40, 256, 32, seed=4)
    c.scales[::2] = 0.0
    assert bool((c.run(coral)[:, ::2] == 0).all())
    for size in (1e-30, 1e30):
        c = Product("f32", 3, 40, 256, 32, seed=4)
        c.x *= size
        c.x64 = c.x.double().cpu().numpy()
        c.check(c.run(coral))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,group", [(3, 70, 32), (20, 70, 128), (50, 96017, 64)])
def test_matvec_w4_zero_points_of_all_bytes(coral, dtype, M, N, group):
    c = Product(dtype, M, N, 520, group, seed=13)
    c.zeros_host = np.random.default_rng(14).integers(0, 256, c.zeros_host.shape, dtype=np.uint8)
    c.zeros = torch.from_numpy(c.zeros_host).cuda()
    c.check(c.run(coral), rows=np.unique(np.r_[0:40, N - 30:N]))


@pytest.mark.parametrize("zeros", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,N", [(3, 70), (20, 70), (50, 96017)])
def test_matvec_w4_largest_activations(coral, dtype, M, N, zeros):
    """(47 + zero) sum |x| over 128 columns just inside fp32: nothing overflows on the way.  (All activations are
    equal: the worst case of the sums' roundings applies, not what random signs leave of it.)"""
    c = Product(dtype, M, N, 256, 128, zeros=zeros, seed=15)
    if zeros:
        c.zeros_host[:] = 255
        c.zeros.fill_(255)
    c.x, c.x64 = stored(np.full((M, 256), 0.99 * np.finfo(np.float32).max / 128 / (47 + (255 if zeros else 8))), dtype)
    c.scales, c.scales64 = stored(np.full(c.scales64.shape, 2.0 ** -10), dtype)
    y = c.run(coral)
    assert bool(torch.isfinite(y).all())
    args = (c.x64, c.codes_host[:50], c.scales64[:50], c.zeros_host[:50] if zeros else None, 128)
    off = np.abs(y[:, :50].double().cpu().numpy() - plain.matvec_w4(*args))
    assert (off <= plain.matvec_w4_bound(*args)).all()


@pytest.mark.parametrize("kind,zeros", [("int", False), ("int", True), ("e2m1", False)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N", [(2, 70), (9, 70), (50, 96017)])
def test_matvec_w4_subnormal_activations(coral, dtype, kind, zeros, M, N):
    """Values below the type's smallest normal number count as they are; of fp32 ones what lies below 2^-133, the
    smallest step of their bf16 parts, is dropped: less than that a value, times its weight."""
    c = Product(dtype, M, N, 256, 64, kind, zeros, seed=16)
    rng = np.random.default_rng(17)
    x = rng.integers(-60, 61, (M, 256)) * 2.0 ** -24 if dtype == "f16" else rng.standard_normal((M, 256)) * (1e-36 if dtype == "f32" else 1e-38)
    c.x, c.x64 = stored(x, dtype)
    c.scales, c.scales64 = stored(np.full(c.scales64.shape, 2.0 ** 10), dtype)
    y = c.run(coral)[:, :50].double().cpu().numpy()
    args = (c.codes_host[:50], c.scales64[:50], c.zeros_host[:50] if zeros else None, 64, kind)
    bound = plain.matvec_w4_bound(c.x64, *args)
    if dtype == "f32":
        bound += 2.0 ** -133 * np.abs(plain.w4_weights(*args)).sum(axis=1)
    off = np.abs(y - plain.matvec_w4(c.x64, *args))
    assert (off <= bound).all() and (dtype == "f32" or (off == 0).all())


def test_matvec_w4_just_above_what_three_bf16_values_hold(coral):
    """fp32 activations whose lowest bit is 2^-133, a whole number of the parts' smallest steps: nothing is dropped."""
    c = Product("f32", 3, 70, 256, 64, seed=18)
    n = np.random.default_rng(19).integers(-2 ** 23, 2 ** 23, (3, 256))
    c.x, c.x64 = stored(n * 2.0 ** -133, "f32")
    assert np.array_equal(c.x64, n * 2.0 ** -133)
    c.scales, c.scales64 = stored(np.full(c.scales64.shape, 2.0 ** 10), "f32")
    c.check(c.run(coral))


def test_matvec_w4_beyond_4_gib_of_codes(coral):
    """Rows whose codes lie past 2^32 bytes."""
    N, K = 150000, 58368
    codes = torch.empty((N, K // 2), dtype=torch.uint8, device="cuda").random_(0, 256, generator=torch.Generator("cuda").manual_seed(1))
    scales = torch.full((N, K // 512), 0.01, device="cuda").bfloat16()
    x, x64 = stored(np.random.default_rng(5).standard_normal((2, K)), "bf16")
    y = coral.coral_matvec_w4(x, codes, scales, group=512)
    at = np.array([0, 1, 73500, 73601, N - 17, N - 2, N - 1])
    host = codes[torch.from_numpy(at).cuda()].cpu().numpy()
    s64 = scales[torch.from_numpy(at).cuda()].double().cpu().numpy()
    want, bound = plain.matvec_w4(x64, host, s64, group=512), plain.matvec_w4_bound(x64, host, s64, group=512)
    assert (np.abs(y[:, torch.from_numpy(at).cuda()].double().cpu().numpy() - want) <= bound).all()


def test_matvec_w4_beyond_4_gib_of_scales(coral):
    """Columns that the waves hold beyond the row's last one have no scale, however many scales there are: not the
    one that lies 4 GiB on."""
    K, group, at = 127 * 8192 + 128, 32, 0x7ffffffe
    n_groups, N = K // group, 66100
    assert N * n_groups > at + 2
    codes = torch.full((N, K // 2), 0x99, dtype=torch.uint8, device="cuda")         # weights of one
    scales = torch.full((N, n_groups), 0.5, device="cuda", dtype=torch.bfloat16)
    scales.view(-1)[at] = float("inf")                             # seen from the first row, the last two bytes below 4 GiB
    x = torch.zeros((2, K), device="cuda", dtype=torch.bfloat16)
    x[:, ::4096] = 1.0
    y = coral.coral_matvec_w4(x, codes, scales, group=group)
    own = at // n_groups                                           # the row whose scale it is
    y[:, own] = 0.5 * 255
    assert bool((y == 0.5 * len(range(0, K, 4096))).all()), torch.nonzero(y != 0.5 * 255)[:4].tolist()


def shifted(t, n=1):
    """The same values, n elements behind a 256-byte boundary."""
    whole = torch.empty(t.numel() + n, dtype=t.dtype, device=t.device)        # (the allocator gives such boundaries)
    whole[n:] = t.reshape(-1)
    return whole[n:].view(t.shape)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,N,K,group", [(3, 83, 1000, 32), (9, 83, 2568, 128), (20, 83, 5000, 64), (50, 96017, 136, 32)])
def test_matvec_w4_operands_aligned_to_their_type_only(coral, dtype, M, N, K, group):
    """Scales, zero points, bias, residual and results one element behind a boundary (x and codes are on 16 bytes)."""
    c = Product(dtype, M, N, K, group, bias=True, residual=True, seed=20)
    want = c.run(coral, "silu", out_dtype=TORCH[dtype])
    c.scales, c.zeros, c.bias, c.residual = (shifted(t) for t in (c.scales, c.zeros, c.bias, c.residual))
    assert torch.equal(c.run(coral, "silu", out=shifted(torch.zeros_like(want))), want)
    assert torch.equal(c.run(coral, "silu", residual=c.residual, out=c.residual), want)


def test_matvec_w4_on_another_stream_and_in_a_graph(coral):
    c = Product("bf16", 4, 200, 1024, 128, seed=6)
    want = c.run(coral)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    y = c.run(coral, stream=stream)
    stream.synchronize()
    assert torch.equal(y, want)
    out = torch.zeros_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(coral, out=out)
    for n in range(3):
        c.x.normal_(generator=torch.Generator("cuda").manual_seed(n))
        want = c.run(coral)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_matvec_w4_binding_refuses(coral):
    c = Product("bf16", 4, 32, 256, 64)
    ok = dict(x=c.x, codes=c.codes, scales=c.scales, zeros=c.zeros, group=64)
    coral.coral_matvec_w4(**ok)
    for change, error in ((dict(codes=c.codes.int()), TypeError), (dict(codes=c.codes[:, :64]), ValueError),
                          (dict(scales=c.scales.float()), TypeError), (dict(scales=c.scales[:, :3]), ValueError),
                          (dict(zeros=c.zeros.int()), TypeError), (dict(group=128), ValueError), (dict(group=0), ValueError),
                          (dict(code_type="e2m1"), coral.CoralError), (dict(code_type="int8"), ValueError), (dict(act="gelu"), ValueError),
                          (dict(out_dtype=torch.float16), TypeError), (dict(bias=c.x[0, :32]), TypeError),
                          (dict(residual=c.x), ValueError), (dict(out=torch.empty((4, 31), device="cuda")), ValueError),
                          (dict(x=torch.empty((256, 4), device="cuda").bfloat16().t()), ValueError), (dict(x=c.x[:, :250].contiguous()), ValueError),
                          (dict(zeros=c.zeros.cpu()), ValueError), (dict(x=c.x[:0]), coral.CoralError)):
        with pytest.raises(error):
            coral.coral_matvec_w4(**dict(ok, **change))


# ---------------------------------------------------------------- rules on logits
class Rules:
    """Random rules for M rows of V tokens; grid: values on which 32 bits compute exactly."""

    def __init__(self, M, V, prompt, output, biases, allowed, shared=False, grid=False, seed=0):
        rng = np.random.default_rng([seed, M, V, prompt, output, biases])
        self.host = dict.fromkeys(("history", "ranges", "penalties", "bias_ids", "bias_values", "bias_ranges", "mask"))
        h = self.host
        if prompt + output:
            prompts = 1 if shared else M
            h["history"] = np.floor(rng.random(prompts * prompt + M * output) ** 3 * (V + 2) - 1).astype(np.int32)      # -1 and V too
            at = np.zeros(M, int) if shared else np.arange(M) * prompt
            out = prompts * prompt + np.arange(M) * output
            h["ranges"] = np.stack([at, at + prompt, out, out + output], axis=1).astype(np.int32)
            h["penalties"] = (np.array([2.0, 0.5, 0.25]) * np.ones((M, 1)) if grid else
                              np.stack([rng.uniform(0.7, 1.5, M), rng.uniform(-0.5, 0.5, M), rng.uniform(-0.5, 0.5, M)], 1)).astype(np.float32)
        if biases:
            n = M * biases
            h["bias_ids"] = rng.integers(-1, V + 1, n).astype(np.int32)
            h["bias_ids"][n // 2:n // 2 + 3] = V // 2                             # the same token again
            h["bias_values"] = (rng.integers(-20, 20, n) * 0.25 if grid else rng.standard_normal(n) * 3).astype(np.float32)
            h["bias_values"][::7] = -np.inf
            h["bias_ranges"] = np.stack([np.arange(M) * biases, np.arange(M) * biases + biases], 1).astype(np.int32)
        if allowed < 1:
            keep = rng.random((M, -(-V // 32), 32)) < allowed
            h["mask"] = (keep.astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32).view(np.int32)

    def device(self):
        return {n: None if a is None else torch.from_numpy(a).cuda() for n, a in self.host.items()}


def check_adjusted(y, z64, rules):
    """y against the rules on z64: every value within the roundings of fp32 and of its type."""
    dtype = {v: n for n, v in TORCH.items()}[y.dtype]
    want, err = plain.logit_rules(z64, **rules.host)
    got = y.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        assert np.array_equal(got == -np.inf, want == -np.inf)
        off = np.where(np.isfinite(want), np.abs(got - want), 0.0)
        assert (off <= err + plain.HALF_STEP[dtype] * (np.abs(np.where(np.isfinite(want), want, 0)) + err) * (dtype != "f32")
                + (2.0 ** -25 if dtype == "f16" else 0)).all()
        assert np.array_equal(np.isnan(got), np.isnan(want))


def check_topk(ids, logp, z64, rules, k):
    """Candidates against the rules on z64: at every rank a value as large as the oracle's within both
    values' roundings, no token twice, and log-probabilities within the roundings of the sum: each of V
    terms' exp within four units (of its result and of its argument, up to 32 in size), 2^-24 per
    addition of sums of 64 lanes, 32 values a lane and 256 parts."""
    want, err = plain.logit_rules(z64, **rules.host)
    want_ids, want_logp = plain.topk_logprob(want, k)
    got, lp = ids.cpu().numpy(), logp.double().cpu().numpy()
    assert np.array_equal(got >= 0, want_ids >= 0) and (got[got < 0] == -1).all() and np.array_equal(lp == -np.inf, want_ids < 0)
    for m in range(len(got)):
        n = int((got[m] >= 0).sum())
        if n == 0:
            continue
        a, b = got[m, :n], want_ids[m, :n]
        assert len(set(a.tolist())) == n
        assert (np.abs(want[m, a] - want[m, b]) <= 2 * err[m].max()).all()
        tol = 2 * err[m].max() + 2.0 ** -24 * (400 + 40 + 2 * np.abs(want_logp[m, :n]) + 2 * np.abs(want[m, b]))
        assert (np.abs(lp[m, :n] - want_logp[m, :n]) <= tol).all(), np.abs(lp[m, :n] - want_logp[m, :n]).max()


ROWS = [  # M, V, prompt, output, biases, allowed, shared
    (1, 1, 3, 2, 2, 1.0, False), (1, 5, 0, 4, 0, 0.5, False), (2, 31, 7, 0, 3, 0.7, False), (3, 33, 5, 9, 0, 0.4, True),
    (1, 1000, 100, 50, 20, 0.3, False), (5, 1003, 0, 0, 0, 0.02, False), (4, 4096, 64, 64, 64, 1.0, False), (3, 4097, 300, 77, 5, 0.6, True),
    (7, 8191, 1000, 3, 33, 0.001, False), (64, 2049, 40, 30, 7, 0.5, True), (9, 50257, 3000, 400, 100, 0.3, False),
    (2, 128256, 2000, 500, 300, 1.0, False), (64, 70001, 300, 100, 10, 0.5, True)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,V,prompt,output,biases,allowed,shared", ROWS)
def test_logits_adjust(coral, dtype, M, V, prompt, output, biases, allowed, shared):
    r = Rules(M, V, prompt, output, biases, allowed, shared)
    z, z64 = stored(np.random.default_rng(V).standard_normal((M, V)) * 3, dtype)
    y, untouched = guarded((M, V), TORCH[dtype])
    coral.coral_logits_adjust(z, out=y, **r.device())
    check_adjusted(y, z64, r)
    untouched()
    assert torch.equal(coral.coral_logits_adjust(z, out=z, **r.device()), y)       # in place


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,V,prompt,output,biases,allowed,shared", ROWS)
def test_logits_topk(coral, dtype, M, V, prompt, output, biases, allowed, shared):
    r = Rules(M, V, prompt, output, biases, allowed, shared)
    z, z64 = stored(np.random.default_rng(V).standard_normal((M, V)) * 3, dtype)
    ws = torch.zeros(coral.coral_logits_topk_workspace_bytes(M, V, min(V, 64)), dtype=torch.uint8, device="cuda")
    for k in sorted({1, min(V, 10), min(V, 64)}):
        ids, untouched = guarded((M, k), torch.int32)
        logp, untouched_too = guarded((M, k), torch.float32)
        coral.coral_logits_topk(z, k, topk_ids=ids, topk_logprob=logp, workspace=ws, **r.device())
        check_topk(ids, logp, z64, r, k)
        untouched()
        untouched_too()
        again = coral.coral_logits_topk(z, k, **r.device())                        # its own workspace: the same bits
        assert torch.equal(again[0], ids) and torch.equal(again[1], logp)
    assert int(ws[:512].view(torch.int32).abs().sum()) == 0                        # the control words, as they were


PREPARED = (128 + 4096) * 4         # bytes of control words and score words, where the rows' counters lie


@pytest.mark.parametrize("M,V,k", [(1, 9000, 3), (64, 30000, 64), (24, 300000, 20), (5, 1000, 10)])
def test_logits_topk_leaves_its_counters_as_they_were(coral, M, V, k):
    ws = torch.zeros(max(coral.coral_logits_topk_workspace_bytes(M, V, k), PREPARED), dtype=torch.uint8, device="cuda")
    z = torch.randn((M, V), device="cuda", generator=torch.Generator("cuda").manual_seed(M))
    first = coral.coral_logits_topk(z, k, workspace=ws)
    for _ in range(3):
        again = coral.coral_logits_topk(z, k, workspace=ws)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
        assert int(ws[:PREPARED].view(torch.int32).abs().sum()) == 0


def test_logits_topk_and_a_head_with_a_shared_gate_in_one_workspace(coral):
    """The head's score words are the rows' counters: zero whenever one call takes them from the other."""
    M, H, V, G, k = 1, 4096, 64000, 256, 10
    gen = torch.Generator("cuda").manual_seed(3)
    hidden, gate, head = (torch.randn(s, device="cuda", generator=gen).bfloat16() * 0.02 for s in ((M, H), (G, H), (V, H)))
    gi = coral.GroupIndex(np.arange(G + 1) * (V // G), np.arange(V, dtype=np.int32))
    z = torch.randn((64, V), device="cuda", generator=gen)
    ws = torch.empty(max(coral.coral_lmhead_workspace_bytes(M, H, V, G, 4, k, coral.CORAL_BF16),
                         coral.coral_logits_topk_workspace_bytes(64, V, k)), dtype=torch.uint8, device="cuda")
    coral.coral_lmhead_workspace_init(ws)
    want = [t.clone() for t in coral.coral_lmhead_grouped(hidden, gate, None, head, gi, 4, k)]
    want_ids, want_logp = coral.coral_logits_topk(z, k)
    scores = ws[512:PREPARED].view(torch.int32)
    for _ in range(4):
        got = coral.coral_lmhead_grouped(hidden, gate, None, head, gi, 4, k, workspace=ws)
        assert int(scores.abs().sum()) == 0 and all(torch.equal(a, b) for a, b in zip(got, want))
        ids, logp = coral.coral_logits_topk(z, k, workspace=ws)
        assert int(scores.abs().sum()) == 0 and torch.equal(ids, want_ids) and torch.equal(logp, want_logp)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,V,k", [(1, 700, 64), (3, 5001, 20), (16, 20000, 64)])
def test_logits_topk_ties_go_to_the_lower_id(coral, dtype, M, V, k):
    """Values on a coarse grid, where every operation is exact: ids equal to the oracle's one by one."""
    r = Rules(M, V, 60, 40, 10, 0.6, grid=True)
    z, z64 = stored(np.random.default_rng(k).integers(-8, 9, (M, V)) * 0.5, dtype)
    ids, logp = coral.coral_logits_topk(z, k, **r.device())
    want, err = plain.logit_rules(z64, **r.host)
    assert np.array_equal(ids.cpu().numpy(), plain.topk_logprob(want, k)[0])
    check_topk(ids, logp, z64, r, k)
    y = coral.coral_logits_adjust(z, **r.device())
    assert np.array_equal(y.double().cpu().numpy(), want)
    plain_ids, _ = coral.coral_logits_topk(y, k)                                   # the rules first, then the ranking
    assert torch.equal(plain_ids, ids)


def test_all_equal_and_constant_rows(coral):
    z = torch.zeros((2, 9000), device="cuda")
    z[1] = -3e38
    ids, logp = coral.coral_logits_topk(z, 64)
    assert torch.equal(ids, torch.arange(64, dtype=torch.int32, device="cuda").expand(2, 64))
    assert float((logp + np.log(9000)).abs().max()) < 1e-6 * 9.2


def test_masked_nan_and_infinities_do_not_matter(coral):
    M, V = 3, 5000
    z, z64 = stored(np.random.default_rng(0).standard_normal((M, V)), "f32")
    keep = np.random.default_rng(1).random((M, V)) < 0.5
    words = np.zeros((M, -(-V // 32) * 32), dtype=np.uint64)
    words[:, :V] = keep
    mask = torch.from_numpy((words.reshape(M, -1, 32) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32).view(np.int32)).cuda()
    want = coral.coral_logits_topk(z, 20, mask=mask)
    y = coral.coral_logits_adjust(z, mask=mask)
    gone = torch.from_numpy(~keep).cuda()
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(torch.float32).min):
        dirty = torch.where(gone, torch.full_like(z, bad), z)
        got = coral.coral_logits_topk(dirty, 20, mask=mask)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(coral.coral_logits_adjust(dirty, mask=mask), y)


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinite_logits_are_the_first_candidates(coral, dtype):
    """(What their rows' log-probabilities are is left open.)"""
    z = torch.randn((3, 9001), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(TORCH[dtype])
    z[0, 8999] = z[2, 17] = z[2, 5000] = float("inf")
    ids, _ = coral.coral_logits_topk(z, 20)
    assert torch.equal(ids, torch.sort(z, dim=1, descending=True, stable=True).indices[:, :20].int())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 2, 3, 7, 9, 64])
def test_many_rows_of_few_tokens(coral, dtype, V):
    r = Rules(64, V, 3, 2, 2, 0.7)
    z, z64 = stored(np.random.default_rng(V).standard_normal((64, V)), dtype)
    for k in sorted({1, (V + 1) // 2, V}):
        check_topk(*coral.coral_logits_topk(z, k, **r.device()), z64, r, k)
    check_adjusted(coral.coral_logits_adjust(z, **r.device()), z64, r)


def test_rules_aligned_to_their_type_only(coral):
    r = Rules(9, 5003, 70, 31, 7, 0.5)
    d = r.device()
    moved = {n: None if t is None else torch.cat([t.reshape(-1)[:1], t.reshape(-1)])[1:].view(t.shape) for n, t in d.items()}
    z = torch.randn((9, 5003), device="cuda")
    assert torch.equal(coral.coral_logits_adjust(z, **moved), coral.coral_logits_adjust(z, **d))
    a, b = coral.coral_logits_topk(z, 12, **moved), coral.coral_logits_topk(z, 12, **d)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_rows_that_nothing_is_left_of(coral):
    M, V, k = 4, 6000, 10
    z = torch.randn((M, V), device="cuda")
    mask = torch.full((M, -(-V // 32)), -1, dtype=torch.int32, device="cuda")
    mask[1] = 0
    mask[2] = 0
    mask[2, 100] = 1 << 5                                                          # token 3205 alone
    z[3] = float("nan")
    z[3, 17] = 0.5
    ids, logp = coral.coral_logits_topk(z, k, mask=mask)
    assert bool((ids[1] == -1).all()) and bool((logp[1] == -float("inf")).all())
    for m, token in ((2, 3205), (3, 17)):                                          # one token: probability one
        assert ids[m].tolist() == [token] + [-1] * 9 and logp[m, 0] == 0 and bool((logp[m, 1:] == -float("inf")).all())
    assert bool((coral.coral_logits_adjust(z, mask=mask)[1] == -float("inf")).all())
    parent, token, score = coral.coral_tree_expand(None, ids[1:3].contiguous(), logp[1:3].contiguous(), 4)
    assert token.tolist() == [3205, -1, -1, -1] and parent.tolist() == [1, -1, -1, -1]


def test_lowest_values_are_candidates(coral):
    """Masks added by the caller as the type's lowest value: ordinary, very small logits."""
    for dtype in DTYPES:
        low = torch.finfo(TORCH[dtype]).min
        z = torch.full((1, 3000), low, dtype=TORCH[dtype], device="cuda")
        z[0, 1234] = 1.0
        ids, logp = coral.coral_logits_topk(z, 3)
        assert ids.tolist() == [[1234, 0, 1]] and logp[0, 0] == 0 and float(logp[0, 1]) < -6e4


# A mask, or biases of -inf, that leave n lanes of a workgroup with a candidate (vectors of 16 bytes are the lanes'), all
# of very low values: keys next to that of -inf.
LOW = {"f32": (-3.4028234663852886e38, -2e38, -1.7e38), "bf16": (-3.3895313892515355e38, -2e38), "f16": (-65504.0,)}


@pytest.mark.parametrize("how", ["mask", "bias"])
@pytest.mark.parametrize("k", [1, 10, 64])
@pytest.mark.parametrize("dtype", DTYPES)
def test_candidates_next_to_minus_infinity(coral, dtype, k, how):
    lanes, V, E = [1, 2, k, k + 5, k + 20, k + 21], 9000, 4 if dtype == "f32" else 8
    for low in LOW[dtype]:
        M = 2 * len(lanes)
        host = np.full((M, V), low)
        host[len(lanes):, ::E] *= 1 - 0.004 * np.arange(len(range(0, V, E)))[None, :] % 0.4        # different ones too
        z, z64 = stored(host, dtype)
        keep = np.zeros((M, V), dtype=bool)
        for m in range(M):
            n = lanes[m % len(lanes)]
            first = 4096 * (m % 2)                                 # in the first slice, or in the second
            keep[m, first:first + n * E:E] = True
        r = Rules(M, V, 0, 0, 0, 1.0)
        if how == "mask":
            words = np.zeros((M, -(-V // 32) * 32), dtype=np.uint64)
            words[:, :V] = keep
            r.host["mask"] = (words.reshape(M, -1, 32) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32).view(np.int32)
        else:
            ids = [np.flatnonzero(~row).astype(np.int32) for row in keep]
            ends = np.cumsum([len(i) for i in ids])
            r.host["bias_ids"] = np.concatenate(ids)
            r.host["bias_values"] = np.full(int(ends[-1]), -np.inf, dtype=np.float32)
            r.host["bias_ranges"] = np.stack([ends - [len(i) for i in ids], ends], 1).astype(np.int32)
        ids, logp = coral.coral_logits_topk(z, k, **r.device())
        want_ids, want_logp = plain.topk_logprob(plain.logit_rules(z64, **r.host)[0], k)
        assert np.array_equal(ids.cpu().numpy(), want_ids)
        # equal values' exponentials are 1 and others' 0 (they are 1e35 apart; fp16's 200): the sum is exact, log is off by
        # 2^-23 at most, the differences by 2^-24 each
        got, real = logp.double().cpu().numpy(), want_ids >= 0
        assert np.array_equal(got == -np.inf, ~real)
        assert (np.abs(got[real] - want_logp[real]) <= 2.0 ** -22 * np.abs(want_logp[real])).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_one_token_of_the_lowest_value(coral, dtype):
    for low in LOW[dtype]:
        ids, logp = coral.coral_logits_topk(torch.full((3, 1), low, device="cuda").to(TORCH[dtype]), 1)
        assert ids.tolist() == [[0]] * 3 and logp.tolist() == [[0.0]] * 3


@pytest.mark.parametrize("k", [1, 10, 64])
def test_few_ordinary_values_among_the_lowest(coral, k):
    """Fewer lanes than k with an ordinary value, the rest at the type's lowest, and lanes without a candidate."""
    for lanes in (k, k + 5, k + 20):
        z = torch.full((2, 3000), -float("inf"), device="cuda")
        z[:, :lanes * 4:4] = torch.finfo(torch.float32).min
        z[0, :(k // 2) * 4:4] = torch.linspace(-3, 3, k // 2, device="cuda")
        want_ids, want_logp = plain.topk_logprob(z.double().cpu().numpy(), k)
        ids, logp = coral.coral_logits_topk(z, k)
        assert np.array_equal(ids.cpu().numpy(), want_ids)
        off = np.abs(logp.double().cpu().numpy() - want_logp)
        # (as check_topk's: ordinary values and their sum)
        assert (off <= 2.0 ** -24 * (450 + 4 * np.abs(want_logp))).all()


def test_ranges_and_ids_outside_the_arrays_are_passed_over(coral):
    V = 3000
    z, z64 = stored(np.random.default_rng(2).standard_normal((5, V)), "f32")
    r = Rules(5, V, 20, 10, 6, 1.0)
    big = 2 ** 31 - 1
    r.host["ranges"] = np.array([[0, big, 0, big], [-big, 20, 10, 5], [50, 50, 149, 150], [big, -big, big, big], [140, 10 ** 9, -5, 3]], np.int32)
    r.host["bias_ranges"] = np.array([[-7, big], [0, 0], [29, 31], [5, 2], [-big, 3]], np.int32)
    check_adjusted(coral.coral_logits_adjust(z, **r.device()), z64, r)
    ids, logp = coral.coral_logits_topk(z, 10, **r.device())
    check_topk(ids, logp, z64, r, 10)


def test_empty_history_and_no_biases(coral):
    z, z64 = stored(np.random.default_rng(3).standard_normal((2, 1500)), "bf16")
    r = Rules(2, 1500, 1, 1, 1, 1.0)
    for n in ("history", "bias_ids", "bias_values"):
        r.host[n] = r.host[n][:0]
    assert torch.equal(coral.coral_logits_adjust(z, **r.device()), z)
    assert torch.equal(coral.coral_logits_topk(z, 7, **r.device())[0], coral.coral_logits_topk(z, 7)[0])


def test_counts_of_one_token_many_times(coral):
    """A token 100 000 times in the output, long prompts shared by all rows."""
    M, V = 6, 2000
    history = np.concatenate([np.arange(90000) % 1500, np.full(100000, 7)]).astype(np.int32)
    r = Rules(M, V, 0, 0, 0, 1.0)
    r.host.update(history=history, ranges=np.array([[0, 90000, 90000, 190000 - m] for m in range(M)], np.int32),
                  penalties=np.full((M, 3), (1.25, 2.0 ** -10, 0.5), np.float32))
    z, z64 = stored(np.random.default_rng(4).standard_normal((M, V)), "f32")
    check_adjusted(coral.coral_logits_adjust(z, **r.device()), z64, r)


def test_an_infinite_frequency_penalty_bans_the_outputs_tokens_only(coral):
    """Tokens of the prompt alone have no count: there is nothing to multiply the penalty with."""
    V = 5000
    z, z64 = stored(np.random.default_rng(6).standard_normal((3, V)) * 3, "f32")
    r = Rules(3, V, 40, 30, 0, 1.0)
    r.host["penalties"][:, 1] = [np.inf, np.nan, -np.inf]
    r.host["ranges"][1, 3] = r.host["ranges"][1, 2]               # no output
    check_adjusted(coral.coral_logits_adjust(z, **r.device()), z64, r)
    want, _ = plain.logit_rules(z64, **r.host)
    ids, _ = coral.coral_logits_topk(z[:2].contiguous(), 10, **{n: None if t is None else t[:2].contiguous() if n in ("ranges", "penalties") else t
                                                                 for n, t in r.device().items()})
    assert np.array_equal(ids.cpu().numpy(), plain.topk_logprob(want[:2], 10)[0])


def test_logits_of_the_widest_rows(coral):
    """As many rows, and as wide, as the calls take (rows that do not start on 16 bytes)."""
    M, V = 64, 1000000 - 3
    z = torch.randn((M, V), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    top = torch.randint(0, V, (M, 3), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    z.scatter_(1, top, torch.tensor([[30.0, 20.0, 25.0]], device="cuda").expand(M, 3).contiguous())
    ids, _ = coral.coral_logits_topk(z, 3)
    assert torch.equal(ids.long()[:, 0], top[:, 0]) and torch.equal(ids.long()[:, 2], top[:, 1])
    banned = top[:, 0].int().contiguous()
    rows = torch.arange(M, device="cuda", dtype=torch.int32)
    got = coral.coral_logits_adjust(z, bias_ids=banned, bias_values=torch.full((M,), -float("inf"), device="cuda"),
                                    bias_ranges=torch.stack([rows, rows + 1], 1).contiguous())
    z.scatter_(1, top[:, :1], -float("inf"))
    assert torch.equal(got, z)


# More published candidates than the workgroup's merge takes at once: one wave merges the lists.
@pytest.mark.parametrize("V,k", [(262145, 64), (300000, 64), (1000000, 64), (1000000, 20), (999993, 17)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_topk_many_lists(coral, dtype, V, k):
    M = 6
    gen = torch.Generator("cuda").manual_seed(V + k)
    z = torch.randn((M, V), device="cuda", generator=gen) * 3
    z[1] = torch.randint(-8, 9, (V,), device="cuda", generator=gen) * 0.5          # equal values
    z[2, V // 2:V // 2 + 100] += 50                                                 # the best in one slice
    z[3] = -float("inf")
    z[3, 5::V // 9] = torch.arange(len(range(5, V, V // 9)), device="cuda") * 0.25  # fewer candidates than k
    z[4] = 2.0
    z[5] = torch.linspace(0, 40, V, device="cuda")                                  # the best last
    z = z.to(TORCH[dtype])
    ids, logp = coral.coral_logits_topk(z, k)
    z64 = z.double()
    val, at = torch.sort(z64, dim=1, descending=True, stable=True)
    val, at = val[:, :k], at[:, :k].int()
    real = val > -float("inf")
    assert torch.equal(ids, torch.where(real, at, torch.full_like(at, -1)))
    want = val - torch.logsumexp(z64, dim=1, keepdim=True)
    assert torch.equal(logp == -float("inf"), ~real)
    # (as in check_topk, without rules)
    tol = 2.0 ** -24 * (440 + 2 * want[real].abs() + 2 * val[real].abs())
    assert bool(((logp.double() - want)[real].abs() <= tol).all())


def test_logits_calls_on_streams_and_in_graphs(coral):
    M, V, k = 4, 30000, 12
    r = Rules(M, V, 200, 100, 20, 0.5)
    d = r.device()
    z = torch.randn((M, V), device="cuda")
    want, want_y = coral.coral_logits_topk(z, k, **d), coral.coral_logits_adjust(z, **d)
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.zeros(coral.coral_logits_topk_workspace_bytes(M, V, k), dtype=torch.uint8, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    got = [[coral.coral_logits_topk(z, k, workspace=w, stream=s, **d) for s, w in zip(streams, spaces)] for _ in range(20)]
    torch.cuda.synchronize()
    for pair in got:
        for g in pair:
            assert torch.equal(g[0], want[0]) and torch.equal(g[1], want[1])
    ids, logp, y = torch.empty_like(want[0]), torch.empty_like(want[1]), torch.empty_like(z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        coral.coral_logits_topk(z, k, topk_ids=ids, topk_logprob=logp, workspace=spaces[0], **d)
        coral.coral_logits_adjust(z, out=y, **d)
    for n in range(3):
        z.normal_(generator=torch.Generator("cuda").manual_seed(n))
        want, want_y = coral.coral_logits_topk(z, k, **d), coral.coral_logits_adjust(z, **d)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ids, want[0]) and torch.equal(logp, want[1]) and torch.equal(y, want_y)


def test_logits_binding_refuses(coral):
    z = torch.zeros((2, 100), device="cuda")
    d = Rules(2, 100, 5, 5, 2, 0.5).device()
    coral.coral_logits_adjust(z, **d)
    bad = [(dict(history=d["history"].long()), TypeError), (dict(ranges=d["ranges"][:, :3]), ValueError), (dict(ranges=None), ValueError),
           (dict(penalties=d["penalties"].double()), TypeError), (dict(bias_values=d["bias_values"][:1]), ValueError),
           (dict(mask=d["mask"][:, :2]), ValueError), (dict(mask=d["mask"].cpu()), ValueError), (dict(bias_ids=None), ValueError)]
    for change, error in bad:
        for call in (lambda **kw: coral.coral_logits_adjust(z, **kw), lambda **kw: coral.coral_logits_topk(z, 3, **kw)):
            with pytest.raises(error):
                call(**dict(d, **change))
    for call in (lambda: coral.coral_logits_topk(z, 0), lambda: coral.coral_logits_topk(z, 65), lambda: coral.coral_logits_topk(z, 101),
                 lambda: coral.coral_logits_topk(z, 5, workspace=torch.zeros(512, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(coral.CoralError):
            call()
    with pytest.raises(ValueError):
        coral.coral_logits_adjust(torch.zeros((100, 2), device="cuda").t())
    with pytest.raises(ValueError):
        coral.coral_logits_adjust(z, out=torch.zeros((2, 99), device="cuda"))
    with pytest.raises(TypeError):
        coral.coral_logits_adjust(z, out=z.half())


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_tree_level_from_a_4_bit_head(coral, dtype):
    """4-bit head, rules, candidates, expansion of the level: each from what the one before left on the
    device, on one stream, one workspace shared with the grouped head of the same step."""
    M, H, V, k, n_next = 6, 512, 5003, 8, 10
    c = Product(dtype, M, V, H, 64, seed=9)
    r = Rules(M, V, 150, 40, 12, 0.3, shared=True)
    head = torch.randn((V - 3, H), device="cuda").to(TORCH[dtype])
    gate = torch.randn((8, H), device="cuda").to(TORCH[dtype])
    gi = coral.GroupIndex(np.arange(9) * ((V - 3) // 8), np.arange(V - 3, dtype=np.int32))
    code = {"f32": coral.CORAL_F32, "bf16": coral.CORAL_BF16, "f16": coral.CORAL_F16}[dtype]
    size = max(coral.coral_lmhead_workspace_bytes(M, H, V - 3, 8, 2, k, code), coral.coral_logits_topk_workspace_bytes(M, V, k))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    coral.coral_lmhead_workspace_init(ws)
    d = r.device()
    parent = -torch.rand(M, device="cuda")
    grouped = [t.clone() for t in coral.coral_lmhead_grouped(c.x, gate, None, head, gi, 2, k, workspace=ws)]
    logits = c.run(coral)
    ids, logp = coral.coral_logits_topk(logits, k, workspace=ws, **d)
    level = coral.coral_tree_expand(parent, ids, logp, n_next)
    again = coral.coral_lmhead_grouped(c.x, gate, None, head, gi, 2, k, workspace=ws)
    c.check(logits)
    check_topk(ids, logp, logits.double().cpu().numpy(), r, k)
    want = oracle.tree_expand(parent.cpu().numpy(), ids.cpu().numpy(), logp.cpu().numpy(), n_next)
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(level, want))
    assert all(torch.equal(a, b) for a, b in zip(grouped, again))
