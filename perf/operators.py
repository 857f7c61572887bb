"""What stands around the gradient cache in a user's program, as measured work: the global norm of the
gradients that Step 3 leaves and their clipping, and the trained linear encoder run in 8-bit integers
(rows quantised with a scale each, and the product of two such matrices: encoding, and scores of queries
against stored passages).

A case is a dict of plain values.  `op` names the operator:

  norm      the global 2-norm of a list of gradients
  clip      the norm, and the gradients scaled to at most max_norm: into buffers of their own, or in place
  quantize  8-bit rows: scale_i = max_j |x_ij| / 127, q_ij = x_ij / scale_i to the nearest integer, ties to even
  product   out_ij = a_scale_i b_scale_j sum_k A_ik B_jk over 8-bit A and B

With `own` false a pass computes the plain form in torch operations; with `own` true it calls the library.
"""
from __future__ import annotations

import math

import torch

own = False

#: Added to the norm before the division, so that a zero norm has a factor.
EPS = 1e-6


def listed():
    return [
        # the two matrices that gc_cache_apply fills, query and passage encoder
        dict(name="norm_two_encoders_f32", op="norm", layers=0, width=768, inner=768, vocab=0, dtype="f32", odd=0),
        # every gradient of a 12-layer encoder with its embedding table, in half the bits
        dict(name="norm_12_layers_bf16", op="norm", layers=12, width=768, inner=2048, vocab=30000, dtype="bf16", odd=0),
        # the same two matrices clipped in place, the bound above the norm: what most steps of a run are
        dict(name="clip_two_encoders_inplace_f32", op="clip", layers=0, width=768, inner=768, vocab=0, dtype="f32",
             odd=0, over=0),
        # many small tensors of odd lengths that do not start on 16-byte boundaries, both types in one list
        dict(name="clip_odd_mixed", op="clip", layers=4, width=333, inner=517, vocab=1001, dtype="mixed", odd=1, over=1),
        # every gradient of a 12-layer encoder, over the bound
        dict(name="clip_12_layers_f32", op="clip", layers=12, width=768, inner=2048, vocab=30000, dtype="f32", odd=0,
             over=1),
        # a wide encoder
        dict(name="clip_24_layers_bf16", op="clip", layers=24, width=1024, inner=4096, vocab=30000, dtype="bf16", odd=0,
             over=1),
        # one query's representation before it is scored
        dict(name="quantize_one_f32", op="quantize", rows=1, d=768, dtype="f32"),
        # the corpus of the largest batch turned into an 8-bit index
        dict(name="quantize_corpus_bf16", op="quantize", rows=131072, d=768, dtype="bf16"),
        # one query against that index
        dict(name="scores_one_query", op="product", rows=1, cols=131072, k=768, out="f32"),
        # a handful of queries, a width and a count that no tile divides
        dict(name="scores_odd_37", op="product", rows=37, cols=50021, k=1000, out="f32"),
        # the scores of an evaluation batch
        dict(name="scores_batch4096", op="product", rows=4096, cols=8192, k=768, out="f32"),
        # a corpus shard through the linear encoder
        dict(name="encode_16384_bf16", op="product", rows=16384, cols=768, k=4096, out="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "clip", "clip", "quantize", "product", "product", "product"])
    if op in ("norm", "clip"):
        case = dict(op=op, layers=rng.randint(0, 16), width=_log_int(rng, 32, 1024), inner=_log_int(rng, 32, 2200),
                    vocab=rng.choice([0, _log_int(rng, 100, 40000)]), dtype=rng.choice(["f32", "bf16", "mixed"]),
                    odd=rng.choice([0, 0, 1]))
        if op == "clip":
            case["over"] = rng.choice([0, 1, 1])
        return case
    if op == "quantize":
        d = rng.choice([128, 512, 768, 1024, _log_int(rng, 8, 8192)])
        return dict(op=op, rows=_log_int(rng, 1, 100e6 / d), d=d, dtype=rng.choice(["f32", "bf16"]))
    k = rng.choice([128, 384, 768, 1024, _log_int(rng, 16, 8192)])
    rows = _log_int(rng, 1, 8192)
    most = min(131072, 5e7 / rows, 1.5e8 / k, 1e11 / (rows * k))
    return dict(op=op, rows=rows, cols=_log_int(rng, 8, max(most, 16)), k=k, out=rng.choice(["f32", "bf16"]))


def _shapes(case):
    """The gradients of an encoder of `layers` layers in its order: table, then per layer four square
    matrices with their biases, two of width x inner with theirs, two pairs of width; no layers: two matrices."""
    w, n = case["width"], case["inner"]
    table = [(case["vocab"], w)] if case["vocab"] else []
    layer = 4 * [(w, w), (w,)] + [(n, w), (n,), (w, n), (w,)] + 4 * [(w,)]
    return table + (case["layers"] * layer if case["layers"] else 2 * [(w, n)])


def _types(case, n):
    if case["dtype"] == "mixed":
        return [torch.bfloat16 if i % 3 else torch.float32 for i in range(n)]
    return [{"f32": torch.float32, "bf16": torch.bfloat16}[case["dtype"]]] * n


def _places(case):
    """(type, first value, shape) of each gradient in its type's flat buffer, and the buffers' lengths.
    Tensors start on 256-byte boundaries, with `odd` set one after the other."""
    shapes, ends, places = _shapes(case), {}, []
    for shape, t in zip(shapes, _types(case, len(shapes))):
        first = ends.get(t, 0)
        places.append((t, first, shape))
        end = first + math.prod(shape)
        ends[t] = end if case["odd"] else -(-end // 128) * 128
    return places, ends


def _views(places, flat):
    return [flat[t][a:a + math.prod(shape)].view(shape) for t, a, shape in places]


def _eight_bits(rows, k, gen):
    """Rows of normal values as 8-bit integers with their scales, the row pitch a multiple of 16 bytes."""
    q = torch.empty(rows, -(-k // 16) * 16, dtype=torch.int8, device="cuda")
    scale = torch.empty(rows, device="cuda")
    step = max(1, (1 << 26) // k)
    for i in range(0, rows, step):
        x = torch.randn(min(step, rows - i), k, generator=gen, device="cuda") * k ** -0.5
        s = x.abs().amax(dim=1) / 127
        q[i:i + step, :k] = torch.round(x / s[:, None]).to(torch.int8)
        scale[i:i + step] = s
    return q[:, :k], scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case=case)
    if case["op"] in ("norm", "clip"):
        # gradients of one size in a tensor, of different sizes between tensors
        places, ends = _places(case)
        flat = {t: torch.zeros(n, dtype=t, device="cuda") for t, n in ends.items()}
        s["grads"] = _views(places, flat)
        sizes = torch.exp(torch.randn(len(places), generator=gen, device="cuda")).tolist()
        for g, size in zip(s["grads"], sizes):
            g.copy_(torch.randn(g.shape, generator=gen, device="cuda") * (1e-3 * size))
        s["norm"] = torch.empty(1, device="cuda")
        if case["op"] == "clip":
            s["kept"] = flat
            s["out"] = s["grads"]
            about = math.sqrt(sum((1e-3 * size) ** 2 * g.numel() for g, size in zip(s["grads"], sizes)))
            s["max_norm"] = about * (0.37 if case["over"] else 2.7)
            if case["over"]:
                s["kept"] = {t: torch.zeros_like(v) for t, v in flat.items()}
                s["out"] = _views(places, s["kept"])
            s["kept"] = [s["kept"][t] for t in sorted(s["kept"], key=str)]
        if own:         # the list's description and the workspace, as a training program keeps them
            from paper_2101_06983_b200 import binding as gc
            s["list"] = gc.GradList(s["grads"], s["out"] if case["op"] == "clip" and case["over"] else None)
            s["ws"] = torch.empty(gc.gc_grad_workspace_bytes(len(places)), dtype=torch.uint8, device="cuda")
    elif case["op"] == "quantize":
        rows, d = case["rows"], case["d"]
        t = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        x = torch.empty(rows, -(-d // 8) * 8, dtype=t, device="cuda")
        step = max(1, (1 << 26) // d)
        for i in range(0, rows, step):
            n = min(step, rows - i)
            x[i:i + n, :d] = torch.randn(n, d, generator=gen, device="cuda") * d ** -0.5
        s["x"] = x[:, :d]
        s["q"] = torch.empty(rows, -(-d // 16) * 16, dtype=torch.int8, device="cuda")[:, :d]
        s["scale"] = torch.empty(rows, device="cuda")
    else:
        s["a"], s["a_scale"] = _eight_bits(case["rows"], case["k"], gen)
        s["b"], s["b_scale"] = _eight_bits(case["cols"], case["k"], gen)
        t = torch.float32 if case["out"] == "f32" else torch.bfloat16
        s["out"] = torch.empty(case["rows"], -(-case["cols"] // 8) * 8, dtype=t, device="cuda")[:, :case["cols"]]
    return s


def _plain_norm(grads):
    return torch.stack([g.double().square().sum() for g in grads]).sum().sqrt()


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2101_06983_b200 import binding as gc
        if op == "norm":
            gc.gc_grad_norm(state["list"], state["norm"], ws=state["ws"])
            return state["norm"]
        if op == "clip":
            gc.gc_grad_clip(state["list"], state["max_norm"], state["norm"], ws=state["ws"])
            return [state["norm"], *state["kept"]]
        if op == "quantize":
            gc.gc_quantize_rows(state["x"], state["q"], state["scale"])
            return [state["q"], state["scale"]]
        gc.gc_matmul_i8(state["a"], state["a_scale"], state["b"], state["b_scale"], state["out"])
        return state["out"]
    if op == "norm":
        return _plain_norm(state["grads"]).float().reshape(1)
    if op == "clip":
        norm = _plain_norm(state["grads"])
        factor = (state["max_norm"] / (norm + EPS)).clamp(max=1.0).float()
        [o.copy_(g.float() * factor) for g, o in zip(state["grads"], state["out"])]
        return [norm.float().reshape(1), *state["kept"]]
    if op == "quantize":
        x = state["x"].float()
        scale = x.abs().amax(dim=1) / 127
        # next to a border between two integers the quotient's last bits decide: formed in 64 bits
        q = torch.round(x.double() / scale.double()[:, None]).clamp(-127, 127).to(torch.int8)
        return [q, scale]
    # 1024 products of 7 bits by 7 bits and their sum are exact in the 24 bits of a float
    a, b = state["a"].float(), state["b"].float()
    total = sum(x @ y.T for x, y in zip(a.split(1024, dim=1), b.split(1024, dim=1)))
    return (total * state["a_scale"][:, None] * state["b_scale"]).to(state["out"].dtype)


def work(case):
    if case["op"] in ("norm", "clip"):
        places, _ = _places(case)
        read = sum(math.prod(shape) * t.itemsize for t, _, shape in places)
        values = sum(math.prod(shape) for _, _, shape in places)
        written = read if case.get("over") else 0
        return {"bytes": read + written + 4, "flops": (3 if written else 2) * values}
    if case["op"] == "quantize":
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": case["rows"] * (case["d"] * (size + 1) + 4), "flops": 3 * case["rows"] * case["d"]}
    m, n, k = case["rows"], case["cols"], case["k"]
    return {"bytes": (m + n) * (k + 4) + m * n * (4 if case["out"] == "f32" else 2), "flops": 2 * m * n * k}


def exact(case, seed):
    """The definitions in 64 bits, on inputs made again from the seed.  An 8-bit integer is a choice of the
    nearest one, not a computed number: it has no value here."""
    s = prepare(case, seed)
    if case["op"] in ("norm", "clip"):
        total = math.sqrt(math.fsum(torch.linalg.vector_norm(g, dtype=torch.float64).item() ** 2 for g in s["grads"]))
        norm = torch.tensor([total], dtype=torch.float64)
        if case["op"] == "norm":
            return norm
        places, ends = _places(case)
        factor = min(1.0, s["max_norm"] / (total + EPS))
        wide = {t: torch.zeros(n, dtype=torch.float64, device="cuda") for t, n in ends.items()}
        for (t, a, shape), g in zip(places, s["grads"]):
            wide[t][a:a + math.prod(shape)] = torch.mul(g.to(torch.float64), factor).flatten()
        return [norm, *(wide[t] for t in sorted(wide, key=str))]
    if case["op"] == "quantize":
        return [None, torch.linalg.vector_norm(s["x"], ord=math.inf, dim=1, dtype=torch.float64) / 127]
    a = s["a"].to(torch.float64) * s["a_scale"].to(torch.float64).unsqueeze(1)
    b = s["b"].to(torch.float64) * s["b_scale"].to(torch.float64).unsqueeze(1)
    return torch.cat([torch.mm(a, part.t()) for part in b.split(1 << 15)], dim=1)
