"""gc_grad_norm, gc_grad_scale and gc_grad_clip against the definition in 64 bits.

Tolerances.  The norm: at most 32 squares are summed in fp32, in four chains of 8 fused multiply-adds that two
further additions join, 10 roundings of at most 2^-24 each; everything beyond is fp64, the square root halves
the relative error and rounding the result adds 2^-24: below 2^-20.  The scaled values are compared with what
the returned sum of squares gives: its square root, the division and the rounding to fp32 are IEEE operations, the
product is rounded once, so they are equal bit for bit."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TOL_NORM = 2.0 ** -20
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def binding():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a CUDA device")
    from paper_2101_06983_b200 import binding as b
    return b


def _sum64(tensors):
    return math.fsum(float((t.detach().cpu().double().flatten() ** 2).sum()) for t in tensors)


def _factor(sq, max_norm):
    c = min(1.0, float(np.float32(max_norm)) / (math.sqrt(sq) + 1e-6))       # the bound is a C float
    return torch.tensor(c, dtype=torch.float64).float()


def _scaled(t, c):
    return (t.detach().cpu().float() * c).to(t.dtype)


class Call:
    """A list with its outputs, on guard: every output starts as a pattern that must be gone."""

    def __init__(self, binding, grads, out=None):
        self.b, self.list = binding, binding.GradList(grads, out)
        self.norm = torch.full((1,), -1.0, device="cuda")
        self.sq = torch.full((1,), -1.0, dtype=torch.float64, device="cuda")
        self.st = torch.zeros(1, dtype=torch.int32, device="cuda")
        # a workspace that holds anything
        self.ws = torch.full((binding.gc_grad_workspace_bytes(len(grads)),), 0xff, dtype=torch.uint8, device="cuda")

    def get_norm(self):
        self.b.gc_grad_norm(self.list, self.norm, self.sq, self.ws, self.st)
        torch.cuda.synchronize()
        return self.sq.item()

    def clip(self, max_norm):
        self.b.gc_grad_clip(self.list, max_norm, self.norm, self.sq, self.ws, self.st)
        torch.cuda.synchronize()
        return self.sq.item()


def _flat(sizes, dtypes, skip=0, seed=0):
    """Tensors one after the other in a buffer for each type, `skip` values before the first."""
    gen = torch.Generator().manual_seed(seed)
    bufs = {t: torch.zeros(skip + 64 + sum(n for n, x in zip(sizes, dtypes) if x is t), dtype=t) for t in set(dtypes)}
    at = {t: skip for t in bufs}
    spans = []
    for n, t in zip(sizes, dtypes):
        bufs[t][at[t]:at[t] + n] = (torch.randn(n, generator=gen) * 10 ** float(torch.rand(1, generator=gen) * 4 - 3)).to(t)
        spans.append((t, at[t], n))
        at[t] += n
    dev = {t: b.cuda() for t, b in bufs.items()}
    return dev, [dev[t][a:a + n] for t, a, n in spans], spans


SIZES = [
    [1], [0], [], [7], [8], [4095], [4096], [4097], [8192], [8193], [100003],
    [1, 1, 1], [5, 0, 3, 17, 1024, 4097, 2], list(range(0, 90)), [1000003, 3, 512],
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("skip", [0, 1, 3])
@pytest.mark.parametrize("case", range(len(SIZES)))
def test_norm_and_clip(binding, case, skip, dtype):
    sizes = SIZES[case]
    types = [dict(f32=F32, bf16=BF).get(dtype) or (BF if i % 2 else F32) for i in range(len(sizes))]
    bufs, grads, spans = _flat(sizes, types, skip, seed=case)
    want = _sum64(grads)
    call = Call(binding, grads)
    before = {t: b.clone() for t, b in bufs.items()}
    sq = call.get_norm()
    assert abs(sq - want) <= 2 * TOL_NORM * want
    assert abs(call.norm.item() - math.sqrt(want)) <= TOL_NORM * math.sqrt(want)
    assert all(torch.equal(b, before[t]) for t, b in bufs.items())
    # not over the bound: nothing changes
    again = call.clip(2 * math.sqrt(want) + 1)
    assert abs(again - want) <= 2 * TOL_NORM * want
    assert all(torch.equal(b, before[t]) for t, b in bufs.items())
    # over it, into other buffers, then in place: the same bits, and nothing beside the tensors changes
    bound = 0.3 * math.sqrt(want)
    outs = {t: torch.full_like(b, 7.0) for t, b in bufs.items()}
    into = Call(binding, grads, [outs[t][a:a + n] for t, a, n in spans])
    c = _factor(into.clip(bound), bound)
    expect = {t: torch.full_like(b, 7.0).cpu() for t, b in bufs.items()}
    for t, a, n in spans:
        expect[t][a:a + n] = _scaled(before[t][a:a + n], c)
    for t in outs:
        assert torch.equal(outs[t].cpu(), expect[t])
        assert torch.equal(bufs[t], before[t])
    assert call.clip(bound) == into.sq.item()
    for (t, a, n), g in zip(spans, grads):
        assert torch.equal(g.cpu(), expect[t][a:a + n])
    gaps = {t: torch.ones(b.numel(), dtype=torch.bool) for t, b in bufs.items()}
    for t, a, n in spans:
        gaps[t][a:a + n] = False
    for t, b in bufs.items():
        assert torch.equal(b.cpu()[gaps[t]], before[t].cpu()[gaps[t]])
    assert call.st.item() == 0 and into.st.item() == 0


@pytest.mark.parametrize("dtype", [F32, BF])
def test_starts_that_differ(binding, dtype):
    """Source and destination on different places within 16 bytes."""
    for n in (1, 30, 5000, 70001):
        for a, b in ((0, 1), (1, 0), (3, 2), (2, 5)):
            src = torch.randn(n + 8, device="cuda").to(dtype)
            dst = torch.full((n + 8,), 7.0, device="cuda", dtype=dtype)
            call = Call(binding, [src[a:a + n]], [dst[b:b + n]])
            sq = call.clip(0.01)
            want = _sum64([src[a:a + n]])
            assert abs(sq - want) <= 2 * TOL_NORM * want
            assert torch.equal(dst[b:b + n].cpu(), _scaled(src[a:a + n], _factor(sq, 0.01)))
            assert bool((dst[:b] == 7).all()) and bool((dst[b + n:] == 7).all())


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,cols,ld,ldo", [(1, 100, 100, 120), (3, 1, 5, 7), (200, 768, 776, 784), (77, 333, 340, 333),
                                              (129, 64, 72, 64), (1000, 8, 16, 24), (5, 20011, 20020, 20016)])
def test_matrices_with_pitch(binding, dtype, rows, cols, ld, ldo):
    big = torch.randn(rows, ld, device="cuda").to(dtype)
    dst = torch.full((rows, ldo), 7.0, device="cuda", dtype=dtype)
    view = big[:, :cols]
    call = Call(binding, [view], [dst[:, :cols]])
    sq = call.clip(0.5)
    want = _sum64([view])
    assert abs(sq - want) <= 2 * TOL_NORM * want
    expect = _scaled(view, _factor(sq, 0.5))
    assert torch.equal(dst[:, :cols].cpu(), expect)
    assert bool((dst[:, cols:] == 7).all())
    pads = big[:, cols:].clone()
    place = Call(binding, [view])
    assert place.get_norm() == place.clip(0.5)
    assert torch.equal(view.cpu(), expect) and torch.equal(big[:, cols:], pads)


def test_column_ranges_of_one_matrix(binding):
    big = torch.randn(100, 96, device="cuda")
    before = big.clone()
    call = Call(binding, [big[:, 32:64], big[:, :32], big[:, 70:]])
    c = _factor(call.clip(1.0), 1.0)
    expect = _scaled(before, c)
    expect[:, 64:70] = before.cpu()[:, 64:70]
    assert torch.equal(big.cpu(), expect)


def test_many_column_ranges_of_one_matrix(binding):
    """More ranges than can be compared two by two, and rows of the other type between them."""
    n = 7000
    big = torch.randn(3, 4 * n, device="cuda")
    gap = big[1, 7:9].view(BF)                                  # of which a range leaves the first two free
    gap.copy_(torch.tensor([1.5, -2.0, 1.0, 1.0]))
    before = big.clone()
    ranges = [big[:, 4 * i:4 * i + 3] for i in range(1, n)] + [gap[:2]]
    call = Call(binding, ranges)
    want = _sum64(ranges)
    sq = call.clip(1.0)
    assert abs(sq - want) <= 2 * TOL_NORM * want
    expect = before.cpu()
    c = _factor(sq, 1.0)
    for k in range(3):
        expect[:, 4 + k::4] = _scaled(before, c)[:, 4 + k::4]
    expect.view(BF)[1, 14:16] = _scaled(before.view(BF)[1, 14:16], c)
    assert torch.equal(big.cpu().view(torch.int32), expect.view(torch.int32))


def test_orders_of_dimensions(binding):
    a = torch.randn(12, 7, 5, 3, device="cuda").to(memory_format=torch.channels_last)
    b = torch.randn(40, 30, device="cuda").t()
    before = [a.clone(), b.clone()]
    call = Call(binding, [a, b])
    c = _factor(call.clip(1.0), 1.0)
    assert torch.equal(a.cpu(), _scaled(before[0], c)) and torch.equal(b.cpu(), _scaled(before[1], c))


def test_strides_of_single_places(binding):
    """A 1 x 1 convolution's gradient of one memory format, its output of another: both lie alike."""
    g = torch.randn(64, 3, 1, 1, device="cuda")
    for src, like in ((g, g.as_strided(g.shape, (3, 1, 3, 3))), (g.as_strided(g.shape, (3, 1, 3, 3)), g)):
        out = torch.empty_strided(like.shape, like.stride(), device="cuda")
        call = Call(binding, [src], [out])
        c = _factor(call.clip(0.5), 0.5)
        assert torch.equal(out.cpu(), _scaled(src, c))


@pytest.mark.parametrize("n", [31, 32, 33, 40, 95, 96, 97, 223, 224, 225, 539, 540, 541, 580, 1400])
def test_lists_of_many_tensors(binding, n):
    """More tensors than one launch takes."""
    sizes = [(i * 37) % 200 + (5000 if i % 101 == 0 else 0) for i in range(n)]
    types = [BF if i % 3 else F32 for i in range(n)]
    bufs, grads, spans = _flat(sizes, types, seed=n)
    before = {t: b.clone() for t, b in bufs.items()}
    want = _sum64(grads)
    call = Call(binding, grads)
    sq = call.clip(0.25)
    assert abs(sq - want) <= 2 * TOL_NORM * want
    c = _factor(sq, 0.25)
    for (t, a, k), g in zip(spans, grads):
        assert torch.equal(g.cpu(), _scaled(before[t][a:a + k], c))
    assert abs(call.get_norm() - _sum64(grads)) <= 2 * TOL_NORM * 0.0625


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("size", [3e38, 1e25, 1e-19, 1e-30, 1e-38, 1e-45, 0.0])
def test_magnitudes(binding, dtype, size):
    """Squares beyond fp32's range on both sides, alone and beside ordinary values."""
    x = (torch.rand(5000) * 0.5 + 0.5).double() * size
    x = x.to(dtype).cuda()
    call = Call(binding, [x])
    want = _sum64([x])
    sq = call.get_norm()
    assert abs(sq - want) <= 2 * TOL_NORM * want
    assert call.st.item() == 0
    if math.sqrt(want) < 3e38:
        assert abs(call.norm.item() - math.sqrt(want)) <= TOL_NORM * math.sqrt(want) + 2.0 ** -150
    before = x.clone()
    c = _factor(sq, 1.0)
    assert call.clip(1.0) == sq
    assert torch.equal(x.cpu(), _scaled(before, c))
    mixed = torch.randn(5000, device="cuda").to(dtype)
    mixed[::7] = before[::7]
    both = Call(binding, [mixed, torch.zeros(100, device="cuda"), torch.ones(9, device="cuda")])
    want = _sum64([mixed]) + 9
    assert abs(both.get_norm() - want) <= 2 * TOL_NORM * want


def test_a_norm_beyond_a_float(binding):
    """Finite gradients whose norm is none: the float is infinite, the sum of squares holds, no flag, and they are scaled."""
    x = torch.tensor([3e38, -3e38], device="cuda")
    before = x.clone()
    call = Call(binding, [x])
    want = _sum64([x])
    sq = call.clip(1e30)
    assert abs(sq - want) <= 2 * TOL_NORM * want
    assert math.isinf(call.norm.item()) and call.st.item() == 0
    assert torch.equal(x.cpu(), _scaled(before, _factor(sq, 1e30)))


def test_a_tensor_listed_twice(binding):
    """The norm counts it twice; it is scaled into two outputs, but not where it lies."""
    x = torch.randn(70001, device="cuda")
    outs = [torch.empty_like(x) for _ in range(2)]
    call = Call(binding, [x, x], outs)
    sq = call.clip(3.0)
    assert sq == call.get_norm() and abs(sq - 2 * _sum64([x])) <= 2 * TOL_NORM * sq
    c = _factor(sq, 3.0)
    assert all(torch.equal(o.cpu(), _scaled(x, c)) for o in outs)
    with pytest.raises(binding.GradCacheError) as e:
        binding.gc_grad_clip([x, x], 3.0, call.norm)
    assert e.value.status == 10


def test_bounds_at_the_ends(binding):
    x = torch.randn(3000, device="cuda")
    before = x.clone()
    call = Call(binding, [x])
    call.clip(math.inf)
    assert torch.equal(x, before)
    call.clip(0.0)
    assert bool((x == 0).all())
    call.clip(1.0)                                   # a norm of zero
    assert call.norm.item() == 0 and bool((x == 0).all()) and call.st.item() == 0


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_values_that_are_not_finite(binding, dtype, bad):
    for n, at in ((1, 0), (3, 2), (9000, 8999), (70000, 5)):
        src = torch.randn(n + 1, device="cuda").to(dtype)[1:]
        src[at] = bad
        dst = torch.zeros(n + 1, device="cuda", dtype=dtype)[1:]
        before = src.clone()
        bits = torch.int32 if dtype == F32 else torch.int16
        place, into = Call(binding, [src]), Call(binding, [src], [dst])
        place.clip(1e-3)
        into.clip(1e-3)
        assert torch.equal(src.view(bits), before.view(bits))
        assert torch.equal(dst.view(bits), before.view(bits))
        assert place.st.item() == into.st.item() == binding.GC_DEV_GRAD_NONFINITE
        assert not math.isfinite(place.norm.item())
        place.st.zero_()
        place.get_norm()
        assert place.st.item() == binding.GC_DEV_GRAD_NONFINITE


def test_sums_that_are_no_sums(binding):
    """gc_grad_scale with a sum of squares that no gradients have: values stay, the flag is set."""
    x = torch.randn(70000, device="cuda")
    before = x.clone()
    for bad in (-1.0, math.nan, math.inf):
        sq = torch.tensor([bad], dtype=torch.float64, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        binding.gc_grad_scale([x], sq, 1e-3, st)
        torch.cuda.synchronize()
        assert torch.equal(x, before) and st.item() == binding.GC_DEV_GRAD_NONFINITE


def test_sums_of_two_ranks(binding):
    """Gradients that two ranks hold in part: each norms its own, the sums are added, each scales its own."""
    whole = torch.randn(70000, device="cuda")
    parts = [whole[:30011].clone(), whole[30011:].clone()]
    sums = []
    for p in parts:
        sq = torch.zeros(1, dtype=torch.float64, device="cuda")
        binding.gc_grad_norm([p], sq_sum=sq)
        sums.append(sq)
    total = sums[0] + sums[1]
    for p in parts:
        binding.gc_grad_scale([p], total, 2.0)
    torch.cuda.synchronize()
    c = _factor(total.item(), 2.0)
    assert torch.equal(torch.cat(parts).cpu(), _scaled(whole, c))


def test_clip_over_ranks_of_one(binding):
    """The library's calls behind sharded.clip_over_ranks, with one rank."""
    from paper_2101_06983_b200 import sharded
    xs = [torch.randn(5000, device="cuda"), torch.randn(300, 7, device="cuda").to(BF)]
    before = [x.clone() for x in xs]
    sq = torch.zeros(1, dtype=torch.float64, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = sharded.clip_over_ranks(binding.GradList(xs), 1.5, sq, dev_status=st)
    assert got is sq and abs(sq.item() - _sum64(before)) <= 2 * TOL_NORM * _sum64(before)
    for x, b in zip(xs, before):
        assert torch.equal(x.cpu(), _scaled(b, _factor(sq.item(), 1.5)))
    xs[1][4, 2] = math.nan
    before = [x.clone() for x in xs]
    sharded.clip_over_ranks(xs, 0.1, sq, dev_status=st)
    assert st.item() == binding.GC_DEV_GRAD_NONFINITE
    assert torch.equal(xs[0], before[0]) and torch.equal(xs[1].view(torch.int16), before[1].view(torch.int16))


def test_captured_calls_that_share_a_workspace(binding):
    """Two captured calls with one workspace, replayed in turn on values that change between, on a stream of
    their own; the eager call gives the same bits."""
    xs = [torch.zeros(300007, device="cuda"), torch.zeros(5000, device="cuda", dtype=BF)]
    outs = [torch.zeros_like(x) for x in xs]
    calls = [Call(binding, [x], [o]) for x, o in zip(xs, outs)]
    calls[1].ws = calls[0].ws
    s = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(s):
        for k in calls:
            binding.gc_grad_clip(k.list, 0.5, k.norm, k.sq, k.ws, k.st)
        s.synchronize()
        for k in calls:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                binding.gc_grad_clip(k.list, 0.5, k.norm, k.sq, k.ws, k.st)
            graphs.append(g)
    for turn in range(3):
        for x in xs:
            x.copy_(torch.randn(x.shape, device="cuda") * (turn + 1))
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        for x, o, k in zip(xs, outs, calls):
            assert torch.equal(o.cpu(), _scaled(x, _factor(k.sq.item(), 0.5)))
            got, sq = o.clone(), k.sq.item()
            assert k.clip(0.5) == sq and torch.equal(o, got)


def test_two_streams_at_once(binding):
    """Calls that overlap, each with a workspace of its own."""
    calls, want = [], []
    for i in range(4):
        x = torch.randn(2000003, device="cuda")
        o = torch.zeros_like(x)
        calls.append((Call(binding, [x], [o]), torch.cuda.Stream(), x, o))
    torch.cuda.synchronize()
    for _ in range(10):
        for k, s, x, o in calls:
            with torch.cuda.stream(s):
                binding.gc_grad_clip(k.list, 0.5, k.norm, k.sq, k.ws, k.st)
    torch.cuda.synchronize()
    for k, s, x, o in calls:
        assert torch.equal(o.cpu(), _scaled(x, _factor(k.sq.item(), 0.5)))


def test_offsets_beyond_32_bits(binding):
    """A tensor of more than 2^32 bytes, ones at its far end."""
    n = (1 << 31) + 12345
    x = torch.zeros(n, dtype=BF, device="cuda")
    x[-3:] = 2.0
    x[n // 2] = 1.0
    call = Call(binding, [x])
    assert call.clip(1.3) == 13.0
    c = _factor(13.0, 1.3)
    assert x[-3:].float().cpu().tolist() == _scaled(torch.full((3,), 2.0, dtype=BF), c).float().tolist()
    assert x[n // 2].float().item() == _scaled(torch.ones(1, dtype=BF), c).float().item()
    assert int((x != 0).sum()) == 4


def test_refusals(binding):
    x, y = torch.zeros(8, 64, device="cuda"), torch.zeros(8, 64, device="cuda", dtype=BF)
    norm = torch.zeros(1, device="cuda")
    with pytest.raises(TypeError):
        binding.GradList([x.half()])
    with pytest.raises(ValueError):
        binding.GradList([x], [y])
    with pytest.raises(ValueError):
        binding.GradList([x], [x, x])
    with pytest.raises(ValueError):
        binding.GradList([x[:, ::2]])
    with pytest.raises(TypeError):
        binding.gc_grad_norm([x], norm.double())
    with pytest.raises(ValueError):
        binding.gc_grad_norm([x], norm.cpu())
    for list_, status in (([x, x[2:]], 10), ([x[:1].expand(8, 64)], 2)):
        with pytest.raises(binding.GradCacheError) as e:
            binding.gc_grad_clip(list_, 1.0, norm)
        assert e.value.status == status
    with pytest.raises(binding.GradCacheError) as e:
        binding.gc_grad_clip([x], -1.0, norm)
    assert e.value.status == 2
    with pytest.raises(binding.GradCacheError) as e:
        binding.gc_grad_clip([x], 1.0, norm, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 6
