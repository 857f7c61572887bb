"""Gradient norm, clipping, 8-bit rows and their product: what is refused before any device work, with
addresses that are never read (no GPU needed)."""
import ctypes

import pytest
import torch

NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, LIMIT, ALIAS = 1, 2, 3, 5, 6, 9, 10


@pytest.fixture(scope="module")
def binding():
    from paper_2101_06983_b200 import _build
    _build.build()
    from paper_2101_06983_b200 import binding as b
    return b


def _list(binding, *tensors):
    arr = (binding._Tensor * max(len(tensors), 1))()
    for x, t in zip(arr, tensors):
        a = dict(data=0x10000, out=None, rows=4, cols=64, ld=64, ld_out=64, dtype=0)
        a.update(t)
        for k, v in a.items():
            setattr(x, k, v)
    return arr, len(tensors)


def _clip(binding, *tensors, max_norm=1.0, norm=0x100, ws=0x100000, wsb=1 << 20, n=None):
    arr, count = _list(binding, *tensors)
    return binding._lib.gc_grad_clip(arr, count if n is None else n, max_norm, None, norm, ws, wsb, None, None)


def _norm(binding, *tensors, sq=0x200, norm=0x100, ws=0x100000, wsb=1 << 20):
    arr, count = _list(binding, *tensors)
    return binding._lib.gc_grad_norm(arr, count, sq, norm, ws, wsb, None, None)


def _passes(status):
    """Not refused for its arguments: without a B200 the call ends at the device."""
    return status in (7, 8)


needs_no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not real ones")


def test_lists_that_are_refused(binding):
    assert _clip(binding, {}, norm=None) == NULL
    assert _norm(binding, {}, sq=None, norm=None) == NULL
    assert _clip(binding, dict(data=None)) == NULL
    assert binding._lib.gc_grad_clip(None, 1, 1.0, None, 0x100, 0x100000, 1 << 20, None, None) == NULL
    assert binding._lib.gc_grad_scale(_list(binding, {})[0], 1, None, 1.0, None, None) == NULL
    assert _clip(binding, {}, n=-1) == SHAPE
    assert _clip(binding, {}, max_norm=-1.0) == SHAPE
    assert _clip(binding, {}, max_norm=float("nan")) == SHAPE
    assert _clip(binding, dict(rows=-1)) == SHAPE
    assert _clip(binding, dict(cols=-1)) == SHAPE
    assert _clip(binding, dict(ld=63)) == SHAPE
    assert _clip(binding, dict(ld=0)) == SHAPE                      # one row repeated
    assert _clip(binding, dict(out=0x90000, ld_out=63)) == SHAPE
    assert _clip(binding, dict(rows=1 << 40, cols=1 << 40, ld=1 << 40)) == SHAPE
    assert _clip(binding, dict(rows=2, cols=(1 << 31) + 1, ld=(1 << 31) + 1)) == LIMIT
    assert _clip(binding, {}, n=(1 << 20) + 1) == LIMIT
    assert _clip(binding, dict(dtype=2)) == DTYPE
    assert _clip(binding, dict(data=0x10002)) == ALIGN
    assert _clip(binding, dict(data=0x10001, dtype=1)) == ALIGN
    assert _clip(binding, dict(out=0x90002)) == ALIGN
    assert _clip(binding, {}, ws=None) == WORKSPACE
    assert _clip(binding, {}, ws=0x100010) == WORKSPACE
    assert _clip(binding, {}, wsb=64) == WORKSPACE


def test_lists_of_too_many_values(binding):
    """A tensor may be listed any number of times for its norm, but a list has an end: its tiles are counted in 32 bits, and
    the workspace holds the partial sums of one launch for each 540 tensors."""
    big = dict(rows=1 << 20, cols=(1 << 17) - 1, ld=1 << 17, dtype=1)            # single elements, 2^26 tiles
    assert _norm(binding, *[big] * 540) == LIMIT
    assert _norm(binding, *[big] * 33) == LIMIT
    assert _norm(binding, *[dict(rows=1, cols=1 << 40)] * 4, {}) == LIMIT
    assert _clip(binding, *[dict(big, data=(k + 1) << 48) for k in range(33)]) == LIMIT
    if not torch.cuda.is_available():
        assert _passes(_norm(binding, *[big] * 32))
        assert _passes(_norm(binding, *[dict(rows=1, cols=1 << 40)] * 4))


def test_places_that_two_tensors_share(binding):
    assert _clip(binding, {}, {}) == ALIAS                          # the same tensor twice
    assert _clip(binding, {}, dict(data=0x10000 + 4 * 255)) == ALIAS
    assert _clip(binding, dict(data=0x10000 + 4 * 255), {}) == ALIAS
    assert _clip(binding, dict(out=0x90000), dict(data=0x20000, out=0x90000)) == ALIAS
    assert _clip(binding, dict(out=0x90000), dict(data=0x90000, out=0xa0000)) == ALIAS      # read and written
    assert _clip(binding, dict(out=0x10100)) == ALIAS                # onto itself, further on
    assert _clip(binding, dict(out=0x10000, rows=4, cols=32, ld=64, ld_out=32)) == ALIAS
    a = dict(cols=32, ld=64)
    assert _clip(binding, a, dict(a, data=0x10000 + 4 * 31)) == ALIAS
    assert _clip(binding, a, dict(a, data=0x10000 + 4 * 33)) == ALIAS        # its rows end in the first's
    assert _clip(binding, a, dict(a, data=0x10000 + 4 * 32, ld=60)) == ALIAS
    # a long tensor with two inside it, the second not its neighbour in the order of addresses
    assert _clip(binding, dict(rows=1, cols=1 << 12), dict(data=0x20000), dict(data=0x10000 + 4 * 2000)) == ALIAS


def _flats(n, gap=0):
    """Tensors of two flat buffers in turn, each with an output in another buffer."""
    at = {k: v for k, v in enumerate((0x10000000, 0x20000000, 0x30000000, 0x40000000))}
    out = []
    for i in range(n):
        size = 4 * (i % 7 + 1) * 5
        out.append(dict(data=at[i % 2], out=at[2 + i % 2], rows=1, cols=size // 4, ld=0, ld_out=0))
        at[i % 2] += size + gap
        at[2 + i % 2] += size + gap
    return out


@pytest.mark.parametrize("n,gap", [(40, 0), (200, 512), (30, 1 << 17)])
def test_shared_places_in_long_lists(binding, n, gap):
    """One output moved onto another, onto a source, or onto itself: in strands, and in no order at all."""
    import random
    for order in (0, 1):
        tensors = _flats(n, gap)
        if order:
            random.Random(n).shuffle(tensors)
        for a, b, key in ((3, n - 2, "out"), (n - 1, 0, "data"), (n // 2, n // 2, "data")):
            bad = [dict(t) for t in tensors]
            bad[a]["out"] = tensors[b][key] + (4 if a == b else 0)
            assert _clip(binding, *bad) == ALIAS
        # two sources may share a place, but not with their gradients scaled where they lie
        twice = [dict(t) for t in tensors]
        twice[1]["data"] = twice[2]["data"]
        if torch.cuda.is_available():
            continue                                     # the addresses are not real ones
        assert _passes(_clip(binding, *tensors))
        assert _passes(_clip(binding, *twice))
        assert _passes(_clip(binding, *[dict(t, out=None) for t in tensors]))
        assert _clip(binding, *[dict(t, out=None) for t in twice]) == ALIAS


def _bytes(t, where):
    es, ld = (2 if t["dtype"] else 4), t["ld" if where == "data" else "ld_out"]
    rows = range(t["rows"])
    return t[where], [range(t[where] + i * ld * es, t[where] + i * ld * es + t["cols"] * es) for i in rows], \
        ld * es if t["rows"] > 1 else 0


def _shares(tensors):
    """Whether a byte that is written belongs to another tensor, or to a matrix of another pitch that reaches
    across it: every byte looked at."""
    spans = []
    for t in tensors:
        spans.append((*_bytes(t, "data")[1:], t["out"] is None))
        if t["out"] is not None:
            spans.append((*_bytes(t, "out")[1:], True))
    sets = [{b for r in rows for b in r} for rows, _, _ in spans]
    for i, (a, pa, wa) in enumerate(spans):
        for k, (b, pb, wb) in enumerate(spans[:i]):
            if (wa or wb) and (sets[i] & sets[k] or pa and pb and pa != pb and a[0][0] < b[-1][-1] + 1
                               and b[0][0] < a[-1][-1] + 1):
                return True
    return False


@needs_no_gpu
def test_shared_places_byte_by_byte(binding):
    """Small lists of rows, matrices of a few pitches and both types, packed closely enough to meet."""
    import random
    rng = random.Random(3)
    seen = [0, 0]
    for turn in range(6000):
        tensors, pitch = [], rng.choice([8, 12, 24])
        for _ in range(rng.randint(2, 6)):
            dtype, rows = rng.randint(0, 1), rng.choice([1, 1, 2, 3, 5])
            es = 2 if dtype else 4
            p = pitch if rng.random() < 0.9 else 16
            cols = rng.randint(1, max(1, p // es // rng.choice([1, 2, 3])))
            if rows == 1 and rng.random() < 0.2:
                cols = rng.randint(1, 20)
            place = lambda: 0x1000 + 4 * rng.randint(0, 60 if turn % 2 else 25)  # noqa: E731
            tensors.append(dict(data=place(), out=None if rng.random() < 0.7 else place() + 0x200 * rng.randint(0, 1),
                                rows=rows, cols=cols, ld=p // es, ld_out=p // es, dtype=dtype))
            if tensors[-1]["out"] == tensors[-1]["data"]:
                tensors[-1]["out"] = None
        want = _shares(tensors)
        seen[want] += 1
        got = _clip(binding, *tensors)
        assert got == ALIAS if want else _passes(got), tensors
    assert min(seen) > 500


@needs_no_gpu
def test_many_column_ranges_of_one_matrix(binding):
    """A matrix cut into more column ranges than can be compared two by two; then one of them moved by an element, or
    scaled into another."""
    n, width = 9000, 3
    ranges = [dict(data=0x100000 + 4 * width * i, rows=5, cols=width, ld=n * width) for i in range(n)]
    assert _passes(_clip(binding, *ranges))
    # ranges in no order, and of the upper and the lower half of the rows
    ranges = [dict(r, rows=3) for r in ranges] + [dict(r, rows=2, data=r["data"] + 4 * 3 * n * width) for r in ranges]
    assert _passes(_clip(binding, *ranges[::-1]))
    for k in (0, n // 3, n + 17, 2 * n - 2):
        bad = [dict(r) for r in ranges]
        bad[k]["data"] += 4
        assert _clip(binding, *bad) == ALIAS
        bad[k].update(data=ranges[k]["data"], out=ranges[k + 1]["data"], ld_out=n * width)
        assert _clip(binding, *bad) == ALIAS


@needs_no_gpu
def test_lists_that_are_taken(binding):
    assert _passes(_clip(binding))
    assert _passes(_clip(binding, dict(data=None, rows=0)))
    assert _passes(_clip(binding, {}, dict(data=0x10000 + 4 * 256)))
    assert _passes(_clip(binding, dict(data=0x10000 + 4 * 256), {}))
    assert _passes(_norm(binding, {}, {}))                           # read twice: counts twice
    assert _passes(_clip(binding, dict(out=0x90000), dict(out=0xa0000)))
    a = dict(cols=32, ld=64)
    assert _passes(_clip(binding, a, dict(a, data=0x10000 + 4 * 32)))          # column halves of one matrix
    assert _passes(_clip(binding, a, dict(data=0x10000 + 4 * 40, rows=1, cols=16, ld=0)))
    assert _passes(_clip(binding, {}, max_norm=float("inf")))
    assert _passes(_clip(binding, {}, max_norm=0.0))


def test_status_strings_of_lists(binding):
    seen = {binding.status_string(i) for i in range(12)}
    assert len(seen) == 12 and "unknown status" not in seen


def test_workspace_of_a_list(binding):
    assert binding.gc_grad_workspace_bytes(-1) == 0
    assert binding.gc_grad_workspace_bytes((1 << 20) + 1) == 0
    for n in (0, 1, 500, 1000, 1 << 20):
        assert binding.gc_grad_workspace_bytes(n) > 0 and binding.gc_grad_workspace_bytes(n) % 256 == 0
    assert binding.gc_grad_workspace_bytes(1 << 20) > binding.gc_grad_workspace_bytes(1)


def test_lists_of_host_tensors_are_refused(binding):
    with pytest.raises(ValueError):
        binding.GradList([torch.zeros(4)])
    with pytest.raises(ValueError):
        binding.GradList([], out=[torch.zeros(4)])
    with pytest.raises(ValueError):
        binding.gc_quantize_rows(torch.zeros(2, 16), torch.zeros(2, 16, dtype=torch.int8), torch.zeros(2))


def test_status_words_of_other_types_are_refused(binding):
    """Kernels set bits of a 32-bit word there."""
    norm, sq, f = torch.zeros(1), torch.zeros(1, dtype=torch.float64), torch.zeros(1, 16)
    q, s = torch.zeros(1, 16, dtype=torch.int8), torch.zeros(1)
    for bad in (torch.zeros(1, dtype=torch.uint8), torch.zeros(1), torch.zeros(1, dtype=torch.int64),
                torch.zeros(0, dtype=torch.int32)):
        for call in (lambda: binding.gc_grad_norm([f], norm, dev_status=bad),
                     lambda: binding.gc_grad_scale([f], sq, 1.0, dev_status=bad),
                     lambda: binding.gc_grad_clip([f], 1.0, norm, dev_status=bad),
                     lambda: binding.gc_matmul_i8(q, s, q, s, torch.zeros(1, 1), dev_status=bad)):
            with pytest.raises(TypeError):
                call()


def test_matrices_of_gradients(binding):
    """How tensors are described: one row where they are dense, whatever the order of their dimensions."""
    z = torch.zeros(6, 8, 4)
    f = binding._as_matrix
    assert f(z) == (1, 192, 192) and f(z.permute(2, 0, 1)) == (1, 192, 192)
    assert f(z[0].t()) == (1, 32, 32)
    assert f(z[0][:, :3]) == (8, 3, 4)
    assert f(z[0][:, 1]) == (8, 1, 4)
    assert f(z[0][:, 1:2]) == (8, 1, 4)
    assert f(torch.zeros(())) == (1, 1, 1) and f(torch.zeros(0, 5)) == (1, 0, 0)
    assert f(z[0], torch.zeros(8, 6)[:, :4]) == (8, 4, 4)
    assert f(torch.zeros(1).expand(5)) == (5, 1, 0)                  # refused by the library
    for bad in (z[:, :, :3], z[0][:, ::2]):
        with pytest.raises(ValueError):
            f(bad)
    with pytest.raises(ValueError):
        f(z[0].t(), torch.zeros(4, 8))


def test_strides_that_say_nothing(binding):
    """A dimension of size 1 may have any stride, and a tensor without values any strides: 1 x 1 convolutions of one
    memory format beside outputs of another, which lie alike."""
    f = binding._as_matrix
    conv = torch.zeros(64, 3, 1, 1)
    last = conv.as_strided((64, 3, 1, 1), (3, 1, 3, 3))
    assert f(conv, last) == f(last, conv) == (1, 192, 192)
    one = torch.zeros(1, 5, 7)
    odd = one.as_strided((1, 5, 7), (1, 7, 1))
    assert f(one, odd) == f(odd, one) == (1, 35, 35)
    with pytest.raises(ValueError):
        f(torch.zeros(64, 3, 2, 1), torch.zeros(64, 2, 3, 1).permute(0, 2, 1, 3))      # these lie differently
    assert f(torch.zeros(0, 4, 6)[:, :, ::2]) == (1, 0, 0)
    assert f(torch.zeros(4, 0, 6)[:, :, ::2], torch.zeros(4, 0, 3)) == (1, 0, 0)


def _quantize(binding, **over):
    a = dict(X=0x10000, ldx=64, rows=4, d=64, dtype=0, q=0x20000, ldq=64, scale=0x30000)
    a.update(over)
    return binding._lib.gc_quantize_rows(*a.values(), None)


def _matmul(binding, **over):
    a = dict(A=0x10000, lda=64, sa=0x100, B=0x20000, ldb=64, sb=0x200, rows=4, cols=8, k=64, dtype=0, out=0x30000, ldo=8,
             status=None)
    a.update(over)
    return binding._lib.gc_matmul_i8(*a.values(), None)


def test_8_bit_calls_that_are_refused(binding):
    assert _quantize(binding, X=None) == NULL and _quantize(binding, q=None) == NULL
    assert _quantize(binding, scale=None) == NULL
    assert _quantize(binding, dtype=2) == DTYPE
    for bad in (dict(rows=0), dict(d=0), dict(ldx=63), dict(ldq=63)):
        assert _quantize(binding, **bad) == SHAPE
    for bad in (dict(X=0x10004), dict(ldx=66), dict(q=0x20008), dict(ldq=72), dict(dtype=1, ldx=68)):
        assert _quantize(binding, **bad) == ALIGN
    assert _quantize(binding, rows=(1 << 30) + 1) == LIMIT
    for name in ("A", "B", "sa", "sb", "out"):
        assert _matmul(binding, **{name: None}) == NULL
    assert _matmul(binding, dtype=7) == DTYPE
    for bad in (dict(rows=0), dict(cols=0), dict(k=0), dict(lda=63), dict(ldb=63), dict(ldo=7)):
        assert _matmul(binding, **bad) == SHAPE
    for bad in (dict(A=0x10008), dict(B=0x20008), dict(out=0x30008), dict(lda=72), dict(ldb=72), dict(ldo=9),
                dict(dtype=1, ldo=12)):
        assert _matmul(binding, **bad) == ALIGN
    assert _matmul(binding, k=131072, lda=131072, ldb=131072) == LIMIT
    assert _matmul(binding, cols=(1 << 30) + 1, ldo=(1 << 30) + 4) == LIMIT


def test_names_of_product_plans(binding):
    """Each form of the product is chosen for some sizes (148 SMs)."""
    name = binding.gc_matmul_i8_plan_name
    assert name(1, 768, 4096, binding.GC_F32) == name(1, 768, 4096, binding.GC_BF16) == "tcgen05-split"
    assert name(4100, 8197, 768, binding.GC_BF16) == "tcgen05-pairs-staged"
    assert name(4100, 8197, 768, binding.GC_F32) == name(16390, 771, 4096, binding.GC_BF16) == "tcgen05-pairs"
    assert name(2500, 9001, 90, binding.GC_BF16) == "tcgen05-staged"
    assert name(2500, 9001, 90, binding.GC_F32) == name(16, 60001, 16, binding.GC_BF16) == "tcgen05"
    for bad in ((0, 1, 1, 0), (1, 0, 1, 0), (1, 1, 0, 0), (1, 1, 131072, 0), (1, 1, 1, 2), ((1 << 30) + 1, 1, 1, 0)):
        assert name(*bad) == "invalid"
