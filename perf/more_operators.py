"""Performance cases of the operators on either side of a training step's output
head, as a training or serving job calls them through the Python entry points:
the root-mean-square norm in front of the head (with the residual's addition,
to 16 or 8 bits) and its gradient, the norm of all gradients of a chunk table,
and the committed step that clips them by it.

A case is a dict with an "op" and that operator's fields:

norm      rows, cols   the activations
          dtype        "bf16", "f16" or "f32" activations
          weight       type of the weight
          residual     a residual is added first, and the sum returned
          out          "same" (the activations' type), "e4m3" or "e5m2": 8 bits with a power-of-two
                       scale for every 128 values of a row
          transposed   the transpose is quantized too, with blocks along its own rows
          eps
norm_grad rows, cols, dtype, weight
          residual     the residual's own gradient is added
grad_norm n, tensors   elements in all, entries of the table
          spread       natural logarithm of the largest entry's size over the smallest's
          unit         every entry's size is a multiple of this
          packed       gradients lie back to back in their allocation, else each at a 256-byte boundary
          dtype
commit    n, tensors, spread, unit
          packed       the state lies back to back, gradients and working copies at boundaries of their own
          layout       "f32" (fp32 master and moments, bf16 gradient and working copy) or "bf16" (all bf16)
          goff         index of the first element in the flat model
          step         the optimizer step
          ratio        the gradients' norm over the largest one allowed
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
# largest value; bits of the fraction; exponent of the smallest normal number
FORMAT = {"e4m3": (448.0, 3, -6), "e5m2": (57344.0, 2, -14)}
BLOCK = 128
ALIGN = 128  # elements: a 256-byte boundary for 16-bit types
LR, B1, B2, EPS, WD = 3e-4, 0.9, 0.95, 1e-8, 0.1  # the package's DEFAULT_HPARAMS
MAX_NORM = 1.0


def _norm(rows, cols, dtype="bf16", weight="bf16", residual=True, out="same", transposed=False, eps=1e-5, **name):
    return dict(op="norm", rows=rows, cols=cols, dtype=dtype, weight=weight, residual=residual, out=out,
                transposed=transposed, eps=eps, **name)


def _norm_grad(rows, cols, dtype="bf16", weight="bf16", residual=True, **name):
    return dict(op="norm_grad", rows=rows, cols=cols, dtype=dtype, weight=weight, residual=residual, eps=1e-5, **name)


def _grad_norm(n, tensors=1, spread=0.0, unit=1, packed=False, dtype="bf16", **name):
    return dict(op="grad_norm", n=n, tensors=tensors, spread=spread, unit=unit, packed=packed, dtype=dtype, **name)


def _commit(n, tensors=1, layout="f32", spread=0.0, unit=1, packed=False, goff=0, step=18, ratio=2.7, **name):
    return dict(op="commit", n=n, tensors=tensors, layout=layout, spread=spread, unit=unit, packed=packed, goff=goff,
                step=step, ratio=ratio, **name)


def listed():
    return [
        # One token in front of an 8-bit head: latency.
        _norm(1, 4096, out="e4m3", name="norm_token"),
        # Sizes that are no multiple of anything, rows at any 2-byte boundary, no residual.
        _norm(777, 5001, dtype="f16", weight="f32", residual=False, eps=1e-6, name="norm_ragged"),
        # A training batch on its way into the head's product: rows for the
        # forward product, the transpose for the weight gradient.
        _norm(8192, 4096, out="e4m3", transposed=True, name="norm_train"),
        # A few positions (a short answer): fewer rows than SMs.
        _norm_grad(4, 4096, name="norm_grad_few"),
        # fp32 activations, odd sizes, a norm without a residual.
        _norm_grad(1021, 5003, dtype="f32", weight="f32", residual=False, name="norm_grad_odd"),
        # A training batch's backward pass.
        _norm_grad(8192, 4096, name="norm_grad_train"),
        # A table of many small tensors (norms, biases, adapters).
        _grad_norm(4_500_000, 1100, spread=5.0, name="grad_norm_many_small"),
        # Gradients of odd sizes, back to back: entries begin at any 2-byte boundary.
        _grad_norm(60_000_000, 291, spread=6.0, packed=True, name="grad_norm_packed_odd"),
        # An ordinary model as a table of matrices and norms.
        _grad_norm(152_000_000, 146, spread=8.6, unit=128, name="grad_norm_152m_table"),
        # The smallest step: one short ragged shard across index 2^32.
        _commit(100_003, goff=(1 << 32) - 50_000, step=3, name="commit_clip_short_shard"),
        # The same model's step with its gradients clipped.
        _commit(152_000_000, 146, spread=8.6, unit=128, step=10, name="commit_clip_152m_table"),
        # A rank of 16 of a large model, everything in bf16.
        _commit(453_001_472, 21, layout="bf16", spread=3.0, unit=128, goff=4_077_013_248, step=5,
                name="commit_clip_bf16_rank_shard"),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "grad_norm", "commit"])
    if op in ("norm", "norm_grad"):
        cols = _log(rng, 16, 16384)
        if rng.random() < 0.5:
            cols = -(-cols // 64) * 64
        rows = _log(rng, 1, max(1, min(16384, 20_000_000 // cols)))
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        weight = rng.choice([dtype, "f32"])
        if op == "norm_grad":
            return _norm_grad(rows, cols, dtype, weight, rng.random() < 0.7)
        out = rng.choice(["same", "e4m3", "e4m3", "e5m2"])
        return _norm(rows, cols, dtype, weight, rng.random() < 0.7, out, out != "same" and rng.random() < 0.5,
                     rng.choice([1e-5, 1e-6]))
    packed = rng.random() < 0.3
    n = _log(rng, 20_000, 60_000_000 if packed else 150_000_000)
    tensors = max(1, min(_log(rng, 1, 1200), n // 256))
    spread, unit = rng.uniform(0.5, 6.0), 1 if packed else rng.choice([1, 8, 128])
    if op == "grad_norm":
        return _grad_norm(n, tensors, spread, unit, packed, rng.choice(["bf16", "bf16", "f16", "f32"]))
    return _commit(n, tensors, rng.choice(["f32", "f32", "bf16"]), spread, unit, packed, rng.randrange(1 << 33),
                   rng.randrange(1, 2000), rng.choice([0.6, rng.uniform(1.0, 20.0)]))


def _blocks(n):
    return -(-n // BLOCK)


def _power(e):
    """2^e, exactly: fp32 for e of 32 bits, fp64 for 64."""
    if e.dtype == torch.int32:
        return ((e + 127) << 23).view(torch.float32)
    return ((e + 1023) << 52).view(torch.float64)


def _scales(x, fmt):
    """The scale of every 128 values of a row of x (fp32): the smallest power of
    two 2^e, with e >= -126, whose product with the format's largest value
    reaches the largest magnitude; 1 for zeros.  [column blocks, rows]."""
    r, c = x.shape
    a = torch.nn.functional.pad(x.abs(), (0, _blocks(c) * BLOCK - c)).view(r, _blocks(c), BLOCK).amax(2)
    top, exponent = torch.frexp(torch.tensor(FORMAT[fmt][0]))
    m, e = torch.frexp(a)
    e = (e - int(exponent) + (m > float(top))).clamp_(min=-126)
    return torch.where(a > 0, _power(e), 1.0).t().contiguous()


def _spread(s, cols):
    return s.t().repeat_interleave(BLOCK, 1)[:, :cols]


def _plain_quantize(x, fmt):
    s = _scales(x, fmt)
    return (x / _spread(s, x.shape[1])).to(FORMATS[fmt]), s


def _room(rows, cols, dtype, multiple):
    """A rows x cols matrix whose rows are a multiple of so many elements apart."""
    return torch.empty(rows, -(-cols // multiple) * multiple, dtype=dtype, device="cuda")[:, :cols]


def _quantized_room(rows, cols, fmt):
    return _room(rows, cols, FORMATS[fmt], 16), _room(_blocks(cols), rows, torch.float32, 4)


def _activations(rows, cols, gen):
    """Normal values with a few columns far larger than the others."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    x[:, torch.rand(cols, generator=gen, device="cuda") < 0.01] *= 20.0
    return x


def _prepare_norm(c, gen):
    r, n, dtype = c["rows"], c["cols"], DTYPES[c["dtype"]]
    s = {"x": _activations(r, n, gen).to(dtype), "residual": None, "sum": None}
    s["weight"] = torch.randn(n, generator=gen, device="cuda").mul_(0.1).add_(1.0).to(DTYPES[c["weight"]])
    if c["op"] == "norm":
        if c["residual"]:
            s["residual"] = _activations(r, n, gen).mul_(3.0).to(dtype)
            s["sum"] = torch.empty_like(s["x"])
        s["rstd"] = torch.empty(r, device="cuda")
        if c["out"] == "same":
            s["out"] = torch.empty_like(s["x"])
        else:
            s["out"] = _quantized_room(r, n, c["out"])
            if c["transposed"]:
                s["out"] += _quantized_room(n, r, c["out"])
        return s
    f = s["x"].float()
    s["rstd"] = 1.0 / (f.square().mean(1) + c["eps"]).sqrt()  # what the forward pass left
    d = torch.randn(r, n, generator=gen, device="cuda").mul_(1e-3)
    d[torch.arange(r, device="cuda") % 13 == 5] = 0.0  # positions that do not count
    s["dout"] = d.to(dtype)
    if c["residual"]:
        s["dresidual"] = torch.randn(r, n, generator=gen, device="cuda").mul_(2e-3).to(dtype)
    else:
        s["dresidual"] = None
    s["dx"] = torch.empty_like(s["x"])
    s["dweight"] = torch.empty_like(s["weight"])
    return s


def _sizes(c):
    """The table's entry sizes: a function of the case alone."""
    t, n, unit = c["tensors"], c["n"], c["unit"]
    r = random.Random("%d/%d/%g" % (n, t, c["spread"]))
    w = [math.exp(c["spread"] * r.random()) for _ in range(t)]
    total = sum(w)
    sizes = [max(unit, int(n * x / total) // unit * unit) for x in w]
    big = max(range(t), key=sizes.__getitem__)
    sizes[big] = max(1, n - (sum(sizes) - sizes[big]))
    return sizes


def _cut(sizes, packed, fill):
    """One buffer for the table, filled by fill(n), and its entries."""
    at, off = [], 0
    for s in sizes:
        at.append(off)
        off += s if packed else -(-s // ALIGN) * ALIGN
    flat = fill(off)
    return [flat[a:a + s] for a, s in zip(at, sizes)]


def _normal(n, sigma, gen, dtype):
    out = torch.empty(n, dtype=dtype, device="cuda")
    for a in range(0, n, 1 << 27):
        b = min(n, a + (1 << 27))
        out[a:b] = torch.randn(b - a, generator=gen, device="cuda").mul_(sigma)
    return out


def _gradients(n, gen, dtype):
    g = _normal(n, 1e-3, gen, dtype)
    g[::97] = 0.0  # exact zeros, as embeddings of absent tokens have
    return g


def _prepare_table(c, gen):
    sizes = _sizes(c)
    if own:
        import paper_2609_18178_gb300 as apc
    if c["op"] == "grad_norm":
        s = {"g": _cut(sizes, c["packed"], lambda n: _gradients(n, gen, DTYPES[c["dtype"]])),
             "out": torch.empty(1, device="cuda")}
        if own:
            s["table"] = apc.prepare_grads(s["g"])
        return s
    wide = c["layout"] == "f32"
    kind = torch.float32 if wide else torch.bfloat16
    s = {"p": _cut(sizes, c["packed"], lambda n: _normal(n, 0.02, gen, kind)),
         "m": _cut(sizes, c["packed"], lambda n: _normal(n, 1e-4, gen, kind)),
         "v": _cut(sizes, c["packed"], lambda n: _normal(n, 1e-3, gen, kind).square_()),
         "g": _cut(sizes, False, lambda n: _gradients(n, gen, torch.bfloat16))}
    if wide:
        s["w"] = _cut(sizes, False, lambda n: torch.zeros(n, dtype=torch.bfloat16, device="cuda"))
    s["goff"], at = [], c["goff"]
    for n in sizes:
        s["goff"].append(at)
        at += n
    s["norm"] = torch.full((1,), c["ratio"] * MAX_NORM, device="cuda")
    s["out"] = torch.empty(4 if wide else 3, dtype=torch.int64, device="cuda")
    if own:
        rows = zip(s["p"], s["m"], s["v"], s["g"], s["w"], s["goff"]) if wide else zip(s["p"], s["m"], s["v"], s["g"], s["goff"])
        s["table"] = apc.prepare_table([(apc.TensorEntry if wide else apc.TensorEntryBF16)(*r) for r in rows])
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 41)
    s = (_prepare_norm if case["op"] in ("norm", "norm_grad") else _prepare_table)(case, gen)
    s["case"] = case
    return s


def _plain_norm(s, c):
    h = s["x"].float()
    if c["residual"]:
        total = (h + s["residual"].float()).to(s["x"].dtype)
        h = total.float()
    # the mean in 64 bits and rounded once: a block's scale turns on the last bit of its largest value
    rstd = (1.0 / (h.double().square().mean(1) + c["eps"]).sqrt()).float()
    y = h * rstd[:, None] * s["weight"].float()
    out = {"rstd": rstd}
    if c["residual"]:
        out["sum"] = total
    if c["out"] == "same":
        out["out"] = y.to(s["x"].dtype)
    else:
        q = _plain_quantize(y, c["out"])
        out["out"] = q + _plain_quantize(y.t().contiguous(), c["out"]) if c["transposed"] else q
    return out


def _plain_norm_grad(s, c):
    z = s["x"].float() * s["rstd"][:, None]
    d = s["dout"].float()
    g = d * s["weight"].float()
    dx = (g - z * (g * z).mean(1, keepdim=True)) * s["rstd"][:, None]
    if c["residual"]:
        dx = dx + s["dresidual"].float()
    return {"dx": dx.to(s["x"].dtype), "dweight": (d * z).sum(0).to(s["weight"].dtype)}


def _signed(x):
    return x - (1 << 64) if x >> 63 else x


def _logical(z, k):
    return (z >> k) & ((1 << (64 - k)) - 1)


def _digest(x, goff):
    """The state digest of one tensor: splitmix64 of (index mod 2^32, bits), summed mod 2^64."""
    bits = x.view(torch.int32 if x.element_size() == 4 else torch.int16).long() & ((1 << 8 * x.element_size()) - 1)
    at = torch.arange(x.numel(), device="cuda").add_(goff) & 0xFFFFFFFF
    z = (at << 32 | bits) + _signed(0x9E3779B97F4A7C15)
    z = (z ^ _logical(z, 30)) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ _logical(z, 27)) * _signed(0x94D049BB133111EB)
    return (z ^ _logical(z, 31)).sum()


def _scalars(c):
    return [torch.tensor(x, dtype=torch.float32).item() for x in (
        B1, 1 - B1, B2, 1 - B2, EPS, 1 - LR * WD, LR / (1 - B1 ** c["step"]), 1 / math.sqrt(1 - B2 ** c["step"]))]


def _plain_commit(s, c):
    """AdamW on the clipped gradient in the step's fixed order of 32-bit operations, state updated in place."""
    b1, c1, b2, c2, eps, decay, lr, rsb2 = _scalars(c)
    factor = torch.where(s["norm"] > MAX_NORM, torch.full_like(s["norm"], MAX_NORM) / s["norm"], 1.0)
    sums = []
    for i, goff in enumerate(s["goff"]):
        g = s["g"][i].float() * factor
        m = s["m"][i].float() * b1 + g * c1
        v = s["v"][i].float() * b2 + g * g * c2
        p = s["p"][i].float() * decay - m / (v.sqrt() * rsb2 + eps) * lr
        written = [s["p"][i].copy_(p), s["m"][i].copy_(m), s["v"][i].copy_(v)]
        if c["layout"] == "f32":
            written.append(s["w"][i].copy_(p))
        sums.append(torch.stack([_digest(x, goff) for x in written]))
    return {**{k: s[k] for k in ("p", "m", "v", "w") if k in s}, "digests": torch.stack(sums).sum(0)}


def _flat(out):
    """A table's outputs, buffer by buffer."""
    return {k: v[0]._base if isinstance(v, list) else v for k, v in out.items()}


def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2609_18178_gb300 as apc
    if c["op"] == "norm":
        if not own:
            return _plain_norm(s, c)
        given = dict(residual=s["residual"], eps=c["eps"], sum=s["sum"], rstd=s["rstd"], out=s["out"])
        if c["out"] == "same":
            out, total, rstd = apc.rms_norm(s["x"], s["weight"], **given)
        else:
            *out, total, rstd = apc.rms_norm_fp8(s["x"], s["weight"], dtype=FORMATS[c["out"]], transposed=c["transposed"],
                                                 **given)
            out = tuple(out)
        return {"out": out, "rstd": rstd, "sum": total} if c["residual"] else {"out": out, "rstd": rstd}
    if c["op"] == "norm_grad":
        if not own:
            return _plain_norm_grad(s, c)
        dx, dweight = apc.rms_norm_grad(s["dout"], s["x"], s["weight"], s["rstd"], dresidual=s["dresidual"], out=s["dx"],
                                        dweight=s["dweight"])
        return {"dx": dx, "dweight": dweight}
    if c["op"] == "grad_norm":
        if own:
            return apc.grad_norm(s["table"], out=s["out"])
        return torch.cat(s["g"]).float().square().sum(dtype=torch.float64).sqrt().float().reshape(1)
    if not own:
        return _flat(_plain_commit(s, c))
    step = apc.commit_step if c["layout"] == "f32" else apc.commit_step_bf16
    step(s["table"], c["step"], out=s["out"], grad_norm=s["norm"], max_norm=MAX_NORM)
    return _flat({**{k: s[k] for k in ("p", "m", "v", "w") if k in s}, "digests": s["out"]})


def work(case):
    """Each input read once, each output written once."""
    if case["op"] in ("norm", "norm_grad"):
        r, c, size = case["rows"], case["cols"], DTYPES[case["dtype"]].itemsize
        n = r * c * size * (3 if case["residual"] else 1) + 4 * r + c * DTYPES[case["weight"]].itemsize
        if case["op"] == "norm_grad":  # dout, x, dx; the residual's gradient
            n += r * c * size * (1 if case["residual"] else 2) + c * DTYPES[case["weight"]].itemsize
            return {"bytes": n, "flops": 10 * r * c}
        if case["out"] == "same":
            return {"bytes": n + r * c * size, "flops": 4 * r * c}
        for a, b in ((r, c), (c, r))[:1 + case["transposed"]]:
            n += a * b + 4 * a * _blocks(b)
        return {"bytes": n, "flops": 5 * r * c}
    if case["op"] == "grad_norm":
        return {"bytes": case["n"] * DTYPES[case["dtype"]].itemsize, "flops": 2 * case["n"]}
    return {"bytes": case["n"] * (28 if case["layout"] == "f32" else 14), "flops": 16 * case["n"]}


def _exact_quantize(x, fmt):
    largest, bits, lowest = FORMAT[fmt]
    r, c = x.shape
    a = torch.zeros(r, _blocks(c) * BLOCK, dtype=torch.float64, device="cuda")
    a[:, :c] = x.abs()
    a = a.unflatten(1, (-1, BLOCK)).max(2).values.t()
    s = _power(torch.ceil(torch.log2(a / largest)).clamp(min=-126.0).long())
    s = torch.where(s * largest < a, 2 * s, s)
    s = torch.where((s * (largest / 2) >= a) & (s > 2.0 ** -126), s / 2, s)
    s = torch.where(a == 0, 1.0, s)
    y = x / s[torch.arange(c, device="cuda") // BLOCK].t()
    e = torch.frexp(y).exponent.long() - 1
    quantum = _power(torch.where(y == 0, lowest, e).clamp(min=lowest) - bits)
    return torch.round(y / quantum) * quantum, s


def _exact_norm(s, c):
    h, out = s["x"].double(), {}
    if c["residual"]:
        out["sum"] = h + s["residual"].double()
        h = out["sum"].to(s["x"].dtype).double()  # the sum goes on as it is stored
    rstd = torch.rsqrt(torch.linalg.vector_norm(h, dim=1) ** 2 / c["cols"] + c["eps"])
    y = torch.einsum("rc,r,c->rc", h, rstd, s["weight"].double())
    out["rstd"] = rstd
    if c["out"] == "same":
        out["out"] = y
    else:
        q = _exact_quantize(y, c["out"])
        out["out"] = q + _exact_quantize(y.t(), c["out"]) if c["transposed"] else q
    return out


def _exact_norm_grad(s, c):
    x, d, w, r = s["x"].double(), s["dout"].double(), s["weight"].double(), s["rstd"].double()
    inner = torch.einsum("rc,c,rc->r", d, w, x)
    dx = torch.einsum("rc,c,r->rc", d, w, r) - torch.einsum("rc,r->rc", x, r ** 3 * inner / c["cols"])
    if c["residual"]:
        dx += s["dresidual"].double()
    return {"dx": dx, "dweight": torch.einsum("rc,rc,r->c", d, x, r)}


def _exact_commit(s, c):
    """Decoupled-weight-decay AdamW with bias corrections, as the textbook has it."""
    t, factor = c["step"], min(1.0, MAX_NORM / s["norm"].item())
    whole = {k: s[k][0]._base.double() for k in ("p", "m", "v", "w") if k in s}
    for i, g in enumerate(s["g"]):
        at = {k: slice(s[k][i].storage_offset(), s[k][i].storage_offset() + g.numel()) for k in whole}
        p, m, v = (whole[k][at[k]] for k in ("p", "m", "v"))
        g = g.double() * factor
        m.lerp_(g, 1 - B1)
        v.lerp_(g.square(), 1 - B2)
        p.sub_(WD * p + (m / (1 - B1 ** t)) / ((v / (1 - B2 ** t)).sqrt() + EPS), alpha=LR)
        if "w" in whole:
            whole["w"][at["w"]] = p
    return {**whole, "digests": None}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s, case)
    if case["op"] == "norm_grad":
        return _exact_norm_grad(s, case)
    if case["op"] == "commit":
        return _exact_commit(s, case)
    total = sum(torch.dot(g, g) for g in (x.double() for x in s["g"]))
    return total.sqrt().reshape(1)
