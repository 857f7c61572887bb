"""gc_quantize_rows and gc_matmul_i8 against their definitions.

Both are compared bit for bit.  The scale is one fp32 product (with 1/127, rounded), an 8-bit integer the nearest one to
the quotient of x and that scale, which fp64 holds closely enough to tell every side of every border.  A
product is an integer below 2^31, rounded to fp32, and two fp32 products in a stated order, then one rounding
to bf16 where that is the output's type."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def binding():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2101_06983_b200 import binding as b
    return b


def _padded(rows, cols, dtype, unit, fill, pad=0):
    """A [rows x cols] view with rows on 16-byte boundaries, `pad` units of 16 bytes more between them."""
    ld = -(-cols // unit) * unit + pad * unit
    big = torch.full((rows, ld), fill, dtype=dtype, device="cuda")
    return big, big[:, :cols]


def _quantized(x):
    """The definition, on the host in 64 bits."""
    x = x.detach().cpu().float().numpy()
    amax = np.abs(x).max(axis=1)
    scale = (amax * np.float32(1 / 127)).astype(np.float32)
    q = np.zeros(x.shape, np.int8)
    for i, s in enumerate(scale):
        if not np.isfinite(amax[i]):
            scale[i] = np.nan
        elif s > 0:
            q[i] = np.clip(np.rint(x[i].astype(np.float64) / np.float64(s)), -127, 127).astype(np.int8)
    return torch.from_numpy(q), torch.from_numpy(scale)


def _check_quantize(binding, x, pad=0):
    rows, d = x.shape
    big, q = _padded(rows, d, torch.int8, 16, 99, pad)
    scale = torch.full((rows + 2,), -5.0, device="cuda")
    binding.gc_quantize_rows(x, q, scale[1:rows + 1])
    torch.cuda.synchronize()
    want_q, want_s = _quantized(x)
    got = scale[1:rows + 1].cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want_s))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want_s))
    assert torch.equal(q.cpu(), want_q)
    assert bool((big[:, d:] == 99).all()) and scale[0].item() == scale[-1].item() == -5.0


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,d", [(1, 1), (1, 768), (3, 15), (5, 16), (7, 17), (9, 31), (33, 500), (8, 512), (300, 513),
                                    (1, 4096), (2, 1024), (17, 1025), (640, 768), (4, 8191), (3, 8192), (5, 8193),
                                    (2, 20011), (5000, 64), (7104, 129), (7111, 256), (7200, 257), (7103, 512), (7104, 512),
                                    (7105, 513), (7333, 768), (7120, 769)])
def test_rows(binding, rows, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(rows * 7 + d)
    unit = 8 if dtype == BF else 4
    for pad in (0, 1):
        _, x = _padded(rows, d, dtype, unit, 1e9, pad)         # what lies between the rows is no value of theirs
        x.copy_(torch.randn(rows, d, generator=gen, device="cuda"))
        _check_quantize(binding, x, pad)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("d", [96, 3000])
def test_values_next_to_borders(binding, d, dtype):
    """Values on and a few units in the last place around every border between two integers, for many scales."""
    gen = np.random.default_rng(d)
    rows = 200
    x = np.zeros((rows, d), np.float32)
    for i in range(rows):
        top = np.float32(2.0 ** gen.uniform(-30, 30))
        s = np.float32(top * np.float32(1 / 127))
        half = (gen.integers(-127, 127, d).astype(np.float64) + 0.5) * np.float64(s)
        v = half.astype(np.float32)
        v = (v.view(np.int32) + gen.integers(-2, 3, d).astype(np.int32)).view(np.float32)
        v[gen.integers(0, d)] = top
        x[i] = np.clip(v, -top, top)
    _, xs = _padded(rows, d, dtype, 8, 0.0)
    xs.copy_(torch.from_numpy(x).cuda())
    _check_quantize(binding, xs)


def test_every_bf16_quotient(binding):
    """Every mantissa of a row's largest value against every bf16 value down to 2^-10 of it, both signs, at exponents from
    the smallest that have an fp32 reciprocal to the largest."""
    mant = torch.arange(128, 256, dtype=torch.float64)
    rows = []
    for e in (-98, -30, -7, 0, 1, 60, 110):
        for a in mant:
            top = a * 2.0 ** (e - 7)
            x = torch.cat([mant * 2.0 ** (e - 7 - j) for j in range(11)])
            x = x[x <= top]
            row = torch.zeros(2 * 11 * 128, dtype=torch.float64)
            row[:len(x)], row[len(row) // 2:len(row) // 2 + len(x)] = x, -x
            rows.append(row)
    x = torch.stack(rows).to(BF)
    assert torch.equal(x.double(), torch.stack(rows))
    _check_quantize(binding, x.cuda())
    _check_quantize(binding, x.cuda()[:, :1408].contiguous()[:, 700:1212].contiguous().repeat(25, 1))


def test_exact_ties(binding):
    """A scale of one: halves go to the even integer."""
    x = torch.arange(-126, 127, device="cuda").float()[None, :] + 0.5
    x = torch.cat([x, torch.full((1, 1), 127.0, device="cuda")], dim=1)
    _, xs = _padded(1, x.shape[1], F32, 4, 0.0)
    xs.copy_(x)
    _check_quantize(binding, xs)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("size", [3e38, 1e30, 1e-20, 1e-30, 1e-36, 1e-38, 1e-43, 1e-45])
def test_magnitudes_of_rows(binding, size, dtype):
    x = ((torch.rand(6, 200, dtype=torch.float64) * 2 - 1) * size).to(dtype)
    x[0] = 0
    x[1, 5:] = 0
    _, xs = _padded(6, 200, dtype, 8, 0.0)
    xs.copy_(x.cuda())
    _check_quantize(binding, xs)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("d", [1, 40, 1500])
def test_rows_that_are_not_finite(binding, d, dtype):
    x = torch.randn(9, d)
    x[1, d // 2], x[3, 0], x[5, d - 1] = math.nan, math.inf, -math.inf
    x[7] = 0
    _, xs = _padded(9, d, dtype, 8, 0.0)
    xs.copy_(x.to(dtype).cuda())
    _check_quantize(binding, xs)


# ---- product ---------------------------------------------------------------------------------------------

def _operands(rows, cols, k, seed, pad=0, low=-127):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    mats, scales = [], []
    for n in (rows, cols):
        big, m = _padded(n, k, torch.int8, 16, 77, pad)       # what lies between the rows is no value of theirs
        m.copy_(torch.randint(low, 128, (n, k), generator=gen, device="cuda", dtype=torch.int32))
        mats.append(m)
        scales.append(torch.rand(n, generator=gen, device="cuda") * 0.01 + 1e-4)
    return mats[0], scales[0], mats[1], scales[1]


def _product(A, sa, B, sb, dtype):
    # integers below 2^53: exact in fp64 in any order
    total = A.double() @ B.double().t()
    return (total.float() * sa[:, None] * sb).to(dtype)


def _check_product(binding, A, sa, B, sb, dtype, pad=0):
    rows, cols = A.shape[0], B.shape[0]
    big, out = _padded(rows + 1, cols, dtype, 8, 5.0, pad)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    binding.gc_matmul_i8(A, sa, B, sb, out[:rows], st)
    torch.cuda.synchronize()
    want = _product(A, sa, B, sb, dtype)
    assert st.item() == 0
    assert torch.equal(out[:rows], want)
    assert bool((big[:, cols:] == 5).all()) and bool((big[rows] == 5).all())
    again = torch.empty_like(big)[:rows, :cols]
    binding.gc_matmul_i8(A, sa, B, sb, again)
    assert torch.equal(again, want)


SHAPES = [
    # rows, cols, k
    (1, 1, 1), (1, 128, 768), (1, 129, 16), (2, 1000, 100), (15, 127, 127), (16, 128, 128), (17, 130, 129), (31, 64, 33),
    (32, 256, 256), (33, 257, 500), (37, 5021, 1000), (48, 300, 768), (64, 64, 64), (65, 512, 768), (100, 99, 98),
    (127, 640, 384), (128, 128, 1024), (129, 129, 129), (200, 3000, 96), (255, 255, 255), (256, 256, 256),
    (257, 300, 640), (300, 1, 768), (513, 1030, 2050), (1000, 777, 36), (1531, 2062, 768), (2048, 2048, 128), (4097, 40, 72),
    (8, 40, 16384), (300, 500, 8192),
    # contractions shared by clusters of eight and of four, and just not
    (1, 1, 2048), (1, 2304, 2048), (1, 2305, 2048), (1, 4736, 3000), (2, 4737, 2000), (16, 129, 1921), (16, 129, 1920),
    (17, 2304, 4096), (17, 2305, 4096), (33, 500, 3969), (64, 100, 5000), (64, 100, 3968), (65, 100, 5000), (5, 131, 131071),
]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,cols,k", SHAPES)
def test_products(binding, rows, cols, k, dtype):
    A, sa, B, sb = _operands(rows, cols, k, seed=rows + cols + k, pad=k % 3)
    _check_product(binding, A, sa, B, sb, dtype, pad=cols % 2)


# Where every CTA (or pair) has three tiles and more, however large they are: accumulators, staging buffers and the places of
# the scales are used again.  Odd widths and counts, short and long contractions, for each form with bf16 outputs.
LONG_RUNS = [
    ("tcgen05-pairs-staged", 4100, 8197, 768), ("tcgen05-pairs-staged", 3001, 20011, 300),
    ("tcgen05-pairs", 16390, 771, 4096), ("tcgen05-pairs", 20, 60001, 5978), ("tcgen05-pairs", 70, 60001, 1500),
    ("tcgen05-staged", 2500, 9001, 90), ("tcgen05-staged", 19315, 1363, 65), ("tcgen05-staged", 151, 60003, 23),
    ("tcgen05", 16, 60001, 16), ("tcgen05", 9, 70005, 100),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("plan,rows,cols,k", LONG_RUNS)
def test_products_of_many_tiles(binding, plan, rows, cols, k, dtype):
    if dtype is BF:
        assert binding.gc_matmul_i8_plan_name(rows, cols, k, binding.GC_BF16) == plan
        m, n = (rows, cols) if "staged" in plan else (cols, rows)
        m_rows, units = (256, 74) if "pairs" in plan else (128, 148)
        assert -(-m // m_rows) * -(-n // 256) > 3 * units
    A, sa, B, sb = _operands(rows, cols, k, seed=rows + k, pad=k % 2)
    _check_product(binding, A, sa, B, sb, dtype, pad=cols % 3)


@pytest.mark.parametrize("rows", [1, 40, 700])
def test_the_longest_contraction(binding, rows):
    """-128 times -128 over the longest rows: the sum still fits 31 bits."""
    k = 131071
    A = torch.full((rows, -(-k // 16) * 16), -128, dtype=torch.int8, device="cuda")[:, :k]
    B = torch.full((130, -(-k // 16) * 16), -128, dtype=torch.int8, device="cuda")[:, :k]
    B[7] = 127
    one = torch.ones(1000, device="cuda")
    out = torch.empty(rows, 132, device="cuda")[:, :130]
    binding.gc_matmul_i8(A, one[:rows], B, one[:130], out)
    want = torch.full((rows, 130), float(np.float32(k * 16384)), device="cuda")
    want[:, 7] = float(np.float32(-128 * 127 * k))
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("cols,k", [(1001, 77), (7, 768), (4097, 1)])
def test_single_rows_need_no_pitch(binding, cols, k, dtype):
    """One query of any width into contiguous tensors of those widths."""
    x = torch.randn(1, k, device="cuda")
    q, s = torch.empty(1, k, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
    binding.gc_quantize_rows(x, q, s)
    want_q, want_s = _quantized(x)
    assert torch.equal(q.cpu(), want_q) and torch.equal(s.cpu(), want_s)
    _, _, B, sb = _operands(1, cols, k, seed=cols)
    guard = torch.full((cols + 16,), 5.0, dtype=dtype, device="cuda")
    out = guard[:cols].view(1, cols)
    binding.gc_matmul_i8(q, s, B, sb, out)
    assert torch.equal(out, _product(q, s, B, sb, dtype)) and bool((guard[cols:] == 5).all())
    # and one channel
    out = torch.empty(cols, 1, dtype=dtype, device="cuda")
    wide = torch.empty(cols, 8, dtype=dtype, device="cuda")[:, :1]
    binding.gc_matmul_i8(B, sb, q, s, wide)
    assert torch.equal(wide, _product(B, sb, q, s, dtype))
    with pytest.raises(binding.GradCacheError) as e:
        binding.gc_matmul_i8(B, sb, q, s, out)                  # rows of 2 or 4 bytes
    assert e.value.status == 5


def test_one_buffer_on_both_sides(binding):
    A, sa, _, _ = _operands(300, 1, 200, seed=1)
    _check_product(binding, A, sa, A, sa, F32)


def test_scales_that_are_not_finite_or_zero(binding):
    A, sa, B, sb = _operands(50, 70, 64, seed=2)
    sa[3], sa[5], sb[7], sb[9] = math.nan, 0.0, math.nan, 0.0
    A[3] = 0
    out = torch.empty(50, 72, device="cuda")[:, :70]
    binding.gc_matmul_i8(A, sa, B, sb, out)
    want = _product(A, sa, B, sb, F32)
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want))
    assert bool(torch.isnan(out[3]).all()) and bool(torch.isnan(out[:, 7]).all())


def test_outputs_beyond_32_bits(binding):
    """An output of more than 2^32 bytes: its last rows."""
    rows, cols, k = 36000, 32768, 32
    A, sa, B, sb = _operands(rows, cols, k, seed=3)
    out = torch.empty(rows, cols, device="cuda")
    binding.gc_matmul_i8(A, sa, B, sb, out)
    for r in (0, 18000, rows - 300):
        assert torch.equal(out[r:r + 300], _product(A[r:r + 300], sa[r:r + 300], B, sb, F32))


def test_inputs_beyond_32_bits(binding):
    """An index of more than 2^32 bytes, made from bf16 rows of more, at its far end; one query against it."""
    n, d = 6_000_000, 768
    x = torch.zeros(n, d, dtype=BF, device="cuda")
    x[-5000:] = torch.randn(5000, d, device="cuda")
    x[n // 2 - 500:n // 2 + 500] = torch.randn(1000, d, device="cuda")
    q, s = torch.full((n, d), 99, dtype=torch.int8, device="cuda"), torch.full((n,), -1.0, device="cuda")
    binding.gc_quantize_rows(x, q, s)
    for part in (slice(n - 5000, n), slice(n // 2 - 500, n // 2 + 500), slice(0, 1000)):
        want_q, want_s = _quantized(x[part])
        assert torch.equal(q[part].cpu(), want_q) and torch.equal(s[part].cpu(), want_s)
    del x
    for rows in (1, 70):
        A, sa, _, _ = _operands(rows, 1, d, seed=rows)
        out = torch.full((rows, n), -1.0, device="cuda")
        binding.gc_matmul_i8(A, sa, q, s, out)
        for part in (slice(n - 5000, n), slice(n // 2 - 500, n // 2 + 500), slice(0, 1000)):
            assert torch.equal(out[:, part], _product(A, sa, q[part], s[part], F32))
        del out


@pytest.mark.parametrize("rows,cols,k", [(1, 5000, 768), (600, 900, 256), (3, 200, 4096)])
def test_captured_and_on_another_stream(binding, rows, cols, k):
    A, sa, B, sb = _operands(rows, cols, k, seed=4)
    x = torch.randn(rows, k, device="cuda")
    out = torch.empty(rows, -(-cols // 8) * 8, dtype=BF, device="cuda")[:, :cols]
    s = torch.cuda.Stream()

    def step():
        binding.gc_quantize_rows(x, A, sa)
        binding.gc_matmul_i8(A, sa, B, sb, out)

    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            step()
    for _ in range(3):
        x.copy_(torch.randn(rows, k, device="cuda"))
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            g.replay()
        torch.cuda.synchronize()
        q, scale = _quantized(x)
        assert torch.equal(A.cpu(), q) and torch.equal(sa.cpu(), scale)
        assert torch.equal(out, _product(A, sa, B, sb, BF))


def test_calls_that_overlap(binding):
    """Products on four streams at once."""
    jobs = []
    for i in range(4):
        ops = _operands(300 + i, 2000, 512, seed=i)
        jobs.append((ops, torch.empty(300 + i, 2000, device="cuda"), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for ops, out, s in jobs:
            with torch.cuda.stream(s):
                binding.gc_matmul_i8(*ops, out)
    torch.cuda.synchronize()
    for ops, out, s in jobs:
        assert torch.equal(out, _product(*ops, F32))


def test_different_calls_that_overlap(binding):
    """Every kernel of these calls, and Steps 2 and 3, on streams of their own at the same time: each stream's results
    are those of its calls alone."""
    from paper_2101_06983_b200 import inputs

    def products(rows, cols, k, dtype):
        x = torch.randn(rows, k, device="cuda").to(dtype)
        A, sa, B, sb = _operands(rows, cols, k, seed=rows)
        out = torch.empty(rows, cols, dtype=dtype, device="cuda")

        def step():
            binding.gc_quantize_rows(x, A, sa)
            binding.gc_matmul_i8(A, sa, B, sb, out)
        return step, [A, sa, out]

    def clipped(sizes):
        g = [torch.randn(n, device="cuda") for n in sizes]
        out = [torch.empty_like(t) for t in g]
        lst, norm = binding.GradList(g, out), torch.empty(1, device="cuda")
        ws = torch.empty(binding.gc_grad_workspace_bytes(len(g)), dtype=torch.uint8, device="cuda")
        return lambda: binding.gc_grad_clip(lst, 0.5, norm, ws=ws), [norm, *out]

    def trained():
        prob = inputs.random_problem(700, 1400, 256, "bf16", seed=5, tau=0.5, scale=256 ** -0.5)
        Q, P, pos = binding.problem_tensors(prob)
        out = binding.Outputs(700, 1400, 256, binding.GC_BF16)
        X, dW = torch.randn(700, 320, device="cuda").bfloat16(), torch.empty(256, 320, device="cuda")
        ws = torch.empty(max(256, binding.gc_cache_apply_workspace_bytes(700, 256, 320)), dtype=torch.uint8, device="cuda")
        lst, norm = binding.GradList([dW]), torch.empty(1, device="cuda")
        ws2 = torch.empty(binding.gc_grad_workspace_bytes(1), dtype=torch.uint8, device="cuda")

        def step():
            binding.gc_build_cache(Q, P, pos, prob.tau, 0, out.loss, out.row_lse, out.dQ, out.dP, out.pos_logit, out.ws,
                                   out.dev_status)
            binding.gc_cache_apply(out.dQ, X, dW, False, ws=ws)
            binding.gc_grad_clip(lst, 0.01, norm, ws=ws2)
        return step, [out.loss, out.dQ, out.dP, dW, norm]

    jobs = [products(1000, 3000, 768, F32), products(1, 500, 4096, F32), products(600, 2048, 1024, BF), products(30, 9000, 640, BF),
            clipped([3000001]), clipped([1000, 20000, 5]), trained()]
    want = []
    for step, outs in jobs:
        step()
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs])
        for t in outs:
            t.zero_()
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(25):
        for (step, _), s in zip(jobs, streams):
            with torch.cuda.stream(s):
                step()
    torch.cuda.synchronize()
    for (_, outs), w in zip(jobs, want):
        for a, b in zip(outs, w):
            assert torch.equal(a, b)


def test_refusals_of_tensors(binding):
    A, sa, B, sb = _operands(16, 32, 64, seed=5)
    out = torch.empty(16, 32, device="cuda")
    for bad in ((A, sa, B[:, :32], sb, out), (A, sa[:3], B, sb, out), (A, sa, B, sb, out[:, :31]), (A.t(), sa, B, sb, out),
                (A.cpu(), sa, B, sb, out)):
        with pytest.raises(ValueError):
            binding.gc_matmul_i8(*bad)
    for bad in ((A.to(torch.uint8), sa, B, sb, out), (A, sa.double(), B, sb, out), (A, sa, B, sb, out.half()),
                (A, torch.empty(32, device="cuda")[::2], B, sb, out)):
        with pytest.raises(TypeError):
            binding.gc_matmul_i8(*bad)
    with pytest.raises(TypeError):
        binding.gc_quantize_rows(out, torch.empty(16, 32, device="cuda"), sa)
    with pytest.raises(ValueError):
        binding.gc_quantize_rows(out, A, sa)


# ---- from the cache to an 8-bit index --------------------------------------------------------------------------

def test_a_step_then_the_encoder_in_8_bits(binding):
    """Step 2, Step 3 over sub-batches, the two matrices' gradients clipped together, a step, and the encoder run in 8
    bits: representations, scores of queries against passages, and the loss of those scores.

    The tolerance of a representation: of k terms x w, each of x and w is off by at most half a step of its row, s / 2
    (and what 127 s and the row's largest value differ by, 2^-23 of it); three fp32 roundings after that."""
    from paper_2101_06983_b200 import inputs
    B, N, d, d_in, tau = 256, 512, 128, 192, 1.0
    lr, bound = 0.5, 0.05
    sbits, Xs = inputs.encoder_inputs(B, d_in, seed=31)
    tbits, Xt = inputs.encoder_inputs(N, d_in, seed=32)
    _, Wf = inputs.encoder_inputs(d, d_in, seed=33, sigma=d_in ** -0.5 * 0.6)
    _, Wg = inputs.encoder_inputs(d, d_in, seed=34, sigma=d_in ** -0.5 * 0.6)
    dev = lambda bits: torch.from_numpy(bits.view(np.int16)).view(BF).cuda()  # noqa: E731
    xs, xt = dev(sbits), dev(tbits)
    W = [torch.from_numpy(w.astype(np.float32)).cuda() for w in (Wf, Wg)]
    Q, P = (xs.float() @ W[0].t()).bfloat16(), (xt.float() @ W[1].t()).bfloat16()
    pos = torch.arange(0, N, 2, dtype=torch.int32, device="cuda")
    out = binding.build_cache(Q, P, pos, tau)
    g = [torch.empty(d, d_in, device="cuda") for _ in range(2)]
    for rep, x, dw in ((out.dQ, xs, g[0]), (out.dP, xt, g[1])):
        for lo in range(0, x.shape[0], 100):
            binding.gc_cache_apply(rep[lo:lo + 100], x[lo:lo + 100], dw, lo > 0)
    raw = [t.clone() for t in g]
    norm = torch.zeros(1, device="cuda")
    binding.gc_grad_clip(g, bound, norm)
    want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in raw))
    assert want > bound and abs(norm.item() - want) <= 2.0 ** -20 * want
    for t, r in zip(g, raw):
        assert float((t.double() - r.double() * (bound / (want + 1e-6))).abs().max()) <= 2.0 ** -19 * float(r.abs().max())
    reps = []
    for x, w, dw in zip((xs, xt), W, g):
        w -= lr * dw
        n = x.shape[0]
        x8, sx = torch.empty(n, d_in, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        w8, sw = torch.empty(d, d_in, dtype=torch.int8, device="cuda"), torch.empty(d, device="cuda")
        rep = torch.empty(n, d, device="cuda")
        binding.gc_quantize_rows(x, x8, sx)
        binding.gc_quantize_rows(w, w8, sw)
        binding.gc_matmul_i8(x8, sx, w8, sw, rep)
        xd, wd = x.double(), w.double()
        ex = (0.5 + 2.0 ** -16) * sx.double()[:, None]
        ew = (0.5 + 2.0 ** -16) * sw.double()
        limit = ex * wd.abs().sum(1) + ew * xd.abs().sum(1, keepdim=True) + d_in * ex * ew
        assert bool(((rep.double() - xd @ wd.t()).abs() <= limit * (1 + 2.0 ** -20) + 2.0 ** -22 * rep.double().abs()).all())
        reps.append(rep)
    # scores of 8-bit representations, as distances of the tiled loss
    q8 = [(torch.empty(r.shape, dtype=torch.int8, device="cuda"), torch.empty(r.shape[0], device="cuda")) for r in reps]
    for r, (q, s) in zip(reps, q8):
        binding.gc_quantize_rows(r, q, s)
    cache = binding.DistanceCache(pos, B, N, tau)
    scores = torch.empty(B, N, device="cuda")
    binding.gc_matmul_i8(*q8[0], *q8[1], scores)
    cache.accumulate(scores, 0, 0)
    cache.finish()
    torch.cuda.synchronize()
    assert cache.dev_status.item() == 0
    s64 = scores.double()
    ref = (torch.logsumexp(s64, dim=1) - s64[torch.arange(B, device="cuda"), pos.long()]).mean().item()
    assert abs(cache.loss.item() - ref) <= 1e-5 * abs(ref)
    dense = reps[0].double() @ reps[1].double().t()
    e = [(0.5 + 2.0 ** -16) * s.double() for _, s in q8]
    limit = e[0][:, None] * reps[1].double().abs().sum(1) + e[1] * reps[0].double().abs().sum(1, keepdim=True) \
        + d * e[0][:, None] * e[1]
    assert bool(((s64 - dense).abs() <= limit * (1 + 2.0 ** -20) + 2.0 ** -22 * s64.abs()).all())
