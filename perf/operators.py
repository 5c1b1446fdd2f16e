"""The operators on the vectors themselves, as cases with sizes: looking vectors up by id and training that
table, the root-mean-square norm in front of a projection (with the residual's addition and an 8-bit result) and
its gradient, and products of 8-bit matrices with a scale for each block of 128, from one request to a training
batch.  Together they make the query vectors that the searches of perf/cases.py take, and score vectors kept in
8 bits.

run() computes an operator in its plain form (elementary torch operations in 32 bits, rounded once at the end);
with `own` it makes the calls of paper_1812_09162_amd.binding.  exact() gives the same outputs from the
definitions in 64 bits.

Sizes are the searches' own (96 to 256 dimensions, 65,536 cells, result lists of 100, batches of 1,000) and
generic powers of two with odd ones between; ids follow a log-uniform frequency (a few tokens make up most of a
batch) or are uniform, values are Gaussian with columns of unequal spread.
"""
import math

import torch

own = False

BLOCK = 128  # values that share a scale
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16,
         "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2, "e8m0": torch.float8_e8m0fnu}
LARGEST = {"e4m3": 448.0, "e5m2": 57344.0}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1, "e5m2": 1, "e8m0": 1}


# -------------------------------------------------------------------- cases --
def _lookup(name, **kw):
    return dict(dict(name=name, path="lookup", n=1, rows=65_536, d=1024, t="bf16", to="bf16", ids="i64", zipf=True, scale=1.0, missing=0.0), **kw)


def _lookup_grad(name, **kw):
    return dict(dict(name=name, path="lookup_grad", n=1, rows=65_536, d=256, t="bf16", to="f32", ids="i64", zipf=True, scale=1.0, missing=0.0), **kw)


def _norm(name, **kw):
    return dict(dict(name=name, path="norm", n=1, d=2048, t="bf16", w="bf16", residual=True, y=False, q="e4m3", s="e8m0"), **kw)


def _norm_grad(name, **kw):
    return dict(dict(name=name, path="norm_grad", n=16_384, d=2048, t="bf16", w="bf16", residual=True), **kw)


def _matmul(name, **kw):
    return dict(dict(name=name, path="matmul", m=1, n=4096, k=2048, a="e4m3", b="e4m3", s="e8m0", to="bf16"), **kw)


def _weight_grad(name, **kw):
    return dict(dict(name=name, path="weight_grad", n=32_768, m=1024, k=2048, t="bf16", a="e5m2", b="e4m3", s="f32", to="f32"), **kw)


def listed():
    return [
        # the vectors behind one search result of R = 100 (the last ids are the search's padding), for re-ranking
        _lookup("lookup_result", n=100, rows=1_000_003, d=96, t="f32", to="f32", ids="i32", zipf=False, missing=0.05),
        # the first layer of a training batch: 512 sequences of 128 tokens, scaled by sqrt(d)
        _lookup("lookup_tokens", n=65_536, scale=32.0),
        # the gradient of a small batch: nearly all of the table has no token
        _lookup_grad("lookup_grad_small", n=2048),
        # the gradient of a long batch, an odd vocabulary; the commonest token has thousands of rows
        _lookup_grad("lookup_grad_long", n=262_144, rows=100_003, d=512, to="bf16", scale=22.5),
        # one request through the norm in front of an 8-bit projection
        _norm("norm_request"),
        # a batch through the same
        _norm("norm_batch", n=16_384),
        # gradients of an odd width, fp16, no second gradient into the residual stream
        _norm_grad("norm_grad_odd", n=10_000, d=1001, t="f16", w="f32", residual=False),
        _norm_grad("norm_grad_batch"),
        # one request through a projection: the weights have to be read once
        _matmul("matmul_request"),
        # scores of 1,000 queries against 65,536 vectors of 96 dimensions kept in 8 bits (less than one block)
        _matmul("matmul_scores", m=1000, n=65_536, k=96, to="f32"),
        # a layer on a long batch
        _matmul("matmul_batch", m=16_384, n=4096, k=4096),
        # the gradient of a layer's weights: both factors brought to 8 bits along the tokens, then multiplied
        _weight_grad("weight_grad_batch"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, most):
    """A size of [lo, hi], at most `most`: a multiple of 128 or 16 half of the time, else whatever comes."""
    v = _log_int(rng, lo, max(lo, min(hi, most)))
    step = rng.choice([128, 16, 1, 1])
    return v // step * step if v >= 2 * step else v


def draw(rng):
    path = rng.choice(["lookup", "lookup", "lookup_grad", "lookup_grad", "norm", "norm", "norm_grad", "norm_grad", "matmul", "matmul", "matmul", "weight_grad"])
    t = rng.choice(["bf16", "bf16", "f16", "f32"])
    s = rng.choice(["e8m0", "e8m0", "f32"])
    if path in ("lookup", "lookup_grad"):
        d = _size(rng, 16, 4096, 4096)
        rows = _log_int(rng, 500, min(1_000_000, 100_000_000 // d))
        n = _log_int(rng, 1, min(262_144, 134_000_000 // d))
        return dict(path=path, n=n, rows=rows, d=d, t=t, to=rng.choice([t, "f32"]), ids=rng.choice(["i32", "i64"]),
                    zipf=rng.random() < 0.6, scale=rng.choice([1.0, math.sqrt(d)]), missing=rng.choice([0.0, 0.0, 0.1]))
    if path in ("norm", "norm_grad"):
        d = _size(rng, 32, 8192, 8192)
        n = _log_int(rng, 1, min(32_768, 33_000_000 // d))
        base = dict(path=path, n=n, d=d, t=t, w=rng.choice([t, "f32"]), residual=rng.random() < 0.7)
        if path == "norm":
            q = rng.choice(["e4m3", "e4m3", ""])
            base.update(y=not q or rng.random() < 0.3, q=q, s=s if q else "")
        return base
    to = rng.choice(["bf16", "bf16", "f16", "f32"])
    if path == "weight_grad":
        m, k = _size(rng, 64, 2048, 2048), _size(rng, 64, 2048, 2048)
        return dict(path=path, n=_size(rng, 128, 32_768, 32_768), m=m, k=k, t=rng.choice(["bf16", "f16"]), a="e5m2", b="e4m3", s=s, to=rng.choice(["f32", "bf16"]))
    k = _size(rng, 32, 8192, 8192)
    m = rng.choice([1, _log_int(rng, 2, 128), _size(rng, 16, 16_384, 16_384)])
    n = _size(rng, 64, 65_536, min(100_000_000 // m, 250_000_000_000 // (m * k)))
    return dict(path=path, m=m, n=n, k=k, a="e4m3", b=rng.choice(["e4m3", "e4m3", "e5m2"]), s=s, to=to)


# ------------------------------------------------------------------- inputs --
def _dev():
    return torch.device("cuda", torch.cuda.current_device())


def _gen(seed, stream):
    g = torch.Generator(device=_dev())
    g.manual_seed((seed * 1000003 + stream * 7919 + 54321) & 0x7FFFFFFFFFFFFFFF)
    return g


def _values(n, d, seed, stream, t, spread=1.0):
    """Gaussian, every column with a spread of its own (log-normal), as the activations of a trained layer have."""
    x = torch.randn((n, d), generator=_gen(seed, stream), device=_dev(), dtype=torch.float32)
    x.mul_(torch.exp(0.5 * torch.randn((d,), generator=_gen(seed, stream + 1), device=_dev())).mul_(spread))
    return x.to(TYPES[t])


def _ids(case, seed):
    n, rows = case["n"], case["rows"]
    u = torch.rand((n,), generator=_gen(seed, 2), device=_dev(), dtype=torch.float64)
    i = (torch.pow(float(rows), u) - 1.0 if case["zipf"] else u * rows).to(torch.int64).clamp_(0, rows - 1)
    if case["missing"]:  # what a search pads its result with
        i[n - int(n * case["missing"]):] = -1
    return i.to(torch.int32 if case["ids"] == "i32" else torch.int64)


def _padded(x, step, t):
    """x as t, the rows a multiple of `step` elements apart (what the block quantizer hands out)."""
    n, d = x.shape
    out = torch.zeros((n, -(-d // step) * step), device=x.device, dtype=torch.uint8 if BYTES[t] == 1 else TYPES[t])
    out = out.view(TYPES[t])[:, :d]
    out.view(torch.uint8 if BYTES[t] == 1 else TYPES[t]).copy_(x.to(TYPES[t]).view(torch.uint8) if BYTES[t] == 1 else x)
    return out


def _eight_bits(n, d, seed, stream, t, s):
    q, scale = _quantize(_values(n, d, seed, stream, "f32"), t, s)
    return _padded(q, 16, t), _padded(scale, 4, s)


def prepare(case, seed):
    path, state = case["path"], dict(case)
    if path == "lookup":
        state.update(table=_values(case["rows"], case["d"], seed, 10, case["t"], 0.05), index=_ids(case, seed))
    elif path == "lookup_grad":
        state.update(grad=_values(case["n"], case["d"], seed, 10, case["t"], 0.01), index=_ids(case, seed))
    elif path in ("norm", "norm_grad"):
        n, d, t = case["n"], case["d"], case["t"]
        state.update(x=_values(n, d, seed, 10, t), weight=(1.0 + 0.2 * _values(1, d, seed, 20, "f32")[0]).to(TYPES[case["w"]]), eps=1e-6)
        if case["residual"]:
            state.update(r=_values(n, d, seed, 30, t, 2.0))
        if path == "norm_grad":
            state.update(dy=_values(n, d, seed, 40, t, 0.01))
    elif path == "matmul":
        state["qa"], state["sa"] = _eight_bits(case["m"], case["k"], seed, 10, case["a"], case["s"])
        state["qb"], state["sb"] = _eight_bits(case["n"], case["k"], seed, 20, case["b"], case["s"])
    else:
        state.update(dy=_values(case["n"], case["m"], seed, 10, case["t"], 0.01), x=_values(case["n"], case["k"], seed, 20, case["t"]))
    return state


# -------------------------------------------------------------- plain forms --
def _blocks(x):
    """[n, d] as [n, blocks, 128], padded with zeros."""
    n, d = x.shape
    return torch.nn.functional.pad(x, (0, -d % BLOCK)).reshape(n, -1, BLOCK)


def _quantize(x, t, s):
    """[n, d] float32 -> 8-bit values and a scale for each 128 of a row: the smallest power of two (e8m0) that brings the
    largest magnitude within the type's range, or their quotient (float32); 1 where all are zero."""
    n, d = x.shape
    b = _blocks(x)
    top = b.abs().amax(dim=2)
    if s == "e8m0":
        fraction, exponent = torch.frexp(top)
        fraction8, exponent8 = math.frexp(LARGEST[t])
        power = (exponent - exponent8 + (fraction > fraction8)).clamp(-127, 127).masked_fill(top == 0, 0)
        scale = (power + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
    else:
        scale = torch.where(top == 0, 1.0, top / torch.full_like(top, LARGEST[t]))  # (a number as divisor would be multiplied by its reciprocal)
    q = b / scale.float().unsqueeze(2)
    return q.reshape(n, -1)[:, :d].to(TYPES[t]), scale


def _restore(q, scale):
    return q.float() * scale.float().repeat_interleave(BLOCK, dim=1)[:, :q.shape[1]]


def _plain_lookup(state):
    index, table = state["index"].long(), state["table"]
    rows = table[index.clamp(min=0)].float() * state["scale"]
    return torch.where((index >= 0).unsqueeze(1), rows, 0.0).to(TYPES[state["to"]])


def _plain_lookup_grad(state):
    index = state["index"].long()
    g = torch.where((index >= 0).unsqueeze(1), state["grad"].float() * state["scale"], 0.0)
    out = torch.zeros((state["rows"], state["d"]), dtype=torch.float32, device=g.device)
    return out.index_add_(0, index.clamp(min=0), g).to(TYPES[state["to"]])


def _plain_norm(state):
    x, out = state["x"], {}
    if state["residual"]:
        x = out["h"] = (x.float() + state["r"].float()).to(x.dtype)
    h = x.float()
    y = h * torch.rsqrt(h.square().mean(dim=1, keepdim=True) + state["eps"]) * state["weight"].float()
    if state["y"]:
        out["y"] = y.to(x.dtype)
    if state["q"]:
        out["q"], out["scales"] = _quantize(y, state["q"], state["s"])
    return out


def _plain_norm_grad(state):
    h, dy = state["x"].float(), state["dy"].float()
    r = torch.rsqrt(h.square().mean(dim=1, keepdim=True) + state["eps"])
    u = dy * state["weight"].float()
    dx = r * u - h * (r * r * r * (u * h).mean(dim=1, keepdim=True))
    if state["residual"]:
        dx = dx + state["r"].float()
    return {"dx": dx.to(state["x"].dtype), "dweight": (dy * h * r).sum(dim=0)}


def _plain_matmul(state):
    return (_restore(state["qa"], state["sa"]) @ _restore(state["qb"], state["sb"]).t()).to(TYPES[state["to"]])


def _plain_weight_grad(state):
    a, sa = _quantize(state["dy"].float().t().contiguous(), state["a"], state["s"])
    b, sb = _quantize(state["x"].float().t().contiguous(), state["b"], state["s"])
    return (_restore(a, sa) @ _restore(b, sb).t()).to(TYPES[state["to"]])


# ------------------------------------------------------ the framework's calls --
def _own(state):
    from paper_1812_09162_amd import binding as qb
    path = state["path"]
    if path == "lookup":
        return qb.vec_lookup(state["table"], state["index"], scale=state["scale"], dtype=TYPES[state["to"]])
    if path == "lookup_grad":
        return qb.vec_lookup_grad(state["grad"], state["index"], state["rows"], scale=state["scale"], dtype=TYPES[state["to"]])
    if path == "norm":
        y, h, q, scales = qb.vec_norm(state["x"], state["weight"], residual=state.get("r"), eps=state["eps"], want_y=state["y"],
                                      quant=TYPES[state["q"]] if state["q"] else None, scale_dtype=TYPES[state["s"]] if state["q"] else None)
        return {k: v for k, v in (("h", h), ("y", y), ("q", q), ("scales", scales)) if v is not None}
    if path == "norm_grad":
        dx, dweight = qb.vec_norm_grad(state["dy"], state["x"], state["weight"], dh=state.get("r"), eps=state["eps"])
        return {"dx": dx, "dweight": dweight}
    to = TYPES[state["to"]]
    if path == "matmul":
        return qb.vec_matmul_blocks(state["qa"], state["sa"], state["qb"], state["sb"], dtype=to)
    a, sa = qb.vec_quantize_blocks(state["dy"], dtype=TYPES[state["a"]], scale_dtype=TYPES[state["s"]], transposed=True)
    b, sb = qb.vec_quantize_blocks(state["x"], dtype=TYPES[state["b"]], scale_dtype=TYPES[state["s"]], transposed=True)
    return qb.vec_matmul_blocks(a, sa, b, sb, dtype=to)


def run(state):
    if own:
        return _own(state)
    return {"lookup": _plain_lookup, "lookup_grad": _plain_lookup_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad,
            "matmul": _plain_matmul, "weight_grad": _plain_weight_grad}[state["path"]](state)


# --------------------------------------------------------------- definitions --
def _scale64(top, t, s):
    if s == "f32":
        return torch.where(top == 0, torch.ones_like(top), (top / LARGEST[t]).float().double())
    power = torch.ceil(torch.log2(torch.where(top == 0, torch.full_like(top, LARGEST[t]), top) / LARGEST[t]))
    power = power + (top > LARGEST[t] * torch.exp2(power)) - (top <= LARGEST[t] * torch.exp2(power - 1)).double() * (top != 0)
    return torch.exp2(power.clamp(-127, 127))


def _scaled64(y, t, s):
    """y / scale, not rounded, and the scales."""
    n, d = y.shape
    groups = [y[:, at:at + BLOCK] for at in range(0, d, BLOCK)]
    scale = torch.stack([_scale64(g.abs().amax(dim=1), t, s) for g in groups], dim=1)
    return torch.cat([g / scale[:, i:i + 1] for i, g in enumerate(groups)], dim=1), scale


def _round8(v, t):
    """To the nearest value with 3 (e4m3) or 2 (e5m2) bits behind the point, ties to even."""
    bits, least = {"e4m3": (3, -6), "e5m2": (2, -14)}[t]
    power = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** (least - 1)))).clamp(min=least)
    power = power + (v.abs() >= torch.exp2(power + 1)) - (v.abs() < torch.exp2(power)).double() * (power > least)
    step = torch.exp2(power - bits)
    return torch.round(v / step) * step


def exact(case, seed):
    state, path = prepare(case, seed), case["path"]
    if path == "lookup":
        out = torch.zeros((case["n"], case["d"]), dtype=torch.float64, device=_dev())
        known = (state["index"] >= 0).nonzero()[:, 0]
        out[known] = state["table"][state["index"][known].long()].double() * state["scale"]
        return out
    if path == "lookup_grad":
        order = torch.argsort(state["index"].long(), stable=True)
        ids = state["index"].long()[order]
        out = torch.zeros((case["rows"], case["d"]), dtype=torch.float64, device=_dev())
        start = torch.searchsorted(ids, torch.arange(case["rows"] + 1, device=_dev()))
        for lo in range(0, case["d"], 64):  # differences of running sums in 64 bits, 64 columns at a time
            run_sum = torch.nn.functional.pad(state["grad"][:, lo:lo + 64][order].double().cumsum(0), (0, 0, 1, 0))
            out[:, lo:lo + 64] = (run_sum[start[1:]] - run_sum[start[:-1]]) * state["scale"]
        return out
    if path == "norm":
        h, out = state["x"].double(), {}
        if case["residual"]:
            out["h"] = h + state["r"].double()
            h = out["h"].to(state["x"].dtype).double()
        y = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["d"] + state["eps"]) * state["weight"].double()
        if case["y"]:
            out["y"] = y
        if case["q"]:
            out["q"], out["scales"] = _scaled64(y, case["q"], case["s"])
        return out
    if path == "norm_grad":
        h, dy, d = state["x"].double(), state["dy"].double(), case["d"]
        rms = torch.sqrt((h * h).sum(1, keepdim=True) / d + state["eps"])
        u = dy * state["weight"].double()
        dx = u / rms - h * (u * h).sum(1, keepdim=True) / (d * rms ** 3)
        return {"dx": dx + state["r"].double() if case["residual"] else dx, "dweight": (dy * h / rms).sum(0)}
    if path == "matmul":
        a, b = ((state[q].double().t() * torch.repeat_interleave(state[s].double().t(), BLOCK, dim=0)[:case["k"]]).t() for q, s in (("qa", "sa"), ("qb", "sb")))
        return a @ b.t().contiguous()
    factors = []
    for v, t in ((state["dy"], case["a"]), (state["x"], case["b"])):
        q, scale = _scaled64(v.double().t(), t, case["s"])
        if case["s"] == "f32":  # by definition the quotient is a float32 before it becomes 8 bits (many are halfway cases)
            q = q.float().double()
        factors.append(_round8(q, t) * torch.repeat_interleave(scale, BLOCK, dim=1)[:, :case["n"]])
    return factors[0] @ factors[1].t().contiguous()


# ---------------------------------------------------------------------- work --
def work(case):
    path, size = case["path"], BYTES
    if path in ("lookup", "lookup_grad"):
        n, rows, d = case["n"], case["rows"], case["d"]
        moved = (min(n, rows) if path == "lookup" else n) * d * size[case["t"]] + (n if path == "lookup" else rows) * d * size[case["to"]]
        return {"bytes": moved + n * (4 if case["ids"] == "i32" else 8), "flops": n * d}
    if path == "norm":
        values, t = case["n"] * case["d"], size[case["t"]]
        out = (t if case["residual"] else 0) + (t if case["y"] else 0) + (1 if case["q"] else 0)
        scales = case["n"] * -(-case["d"] // BLOCK) * size[case["s"]] if case["q"] else 0
        return {"bytes": values * (t + (t if case["residual"] else 0) + out) + scales + case["d"] * size[case["w"]], "flops": 6 * values}
    if path == "norm_grad":
        values = case["n"] * case["d"]
        return {"bytes": values * size[case["t"]] * (4 if case["residual"] else 3) + case["d"] * (4 + size[case["w"]]), "flops": 10 * values}
    m, n, k = case["m"], case["n"], case["k"]
    if path == "matmul":
        return {"bytes": (m + n) * (k + -(-k // BLOCK) * size[case["s"]]) + m * n * size[case["to"]], "flops": 2 * m * n * k}
    return {"bytes": n * (m + k) * size[case["t"]] + m * k * size[case["to"]], "flops": 2 * m * n * k}
