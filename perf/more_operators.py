"""Dropout and low-rank adapters, as cases with sizes: dropout from a counter-based generator (its mask is made from a seed,
a step and a layer wherever it is needed, and never stored), by itself with the residual's addition; and low-rank adapters of
many requests beside a shared projection, with dropout of their input, from one token to a training batch, and their gradient.
They train the towers whose vectors the searches of perf/cases.py take, and serve many of them over one projection.

run() computes an operator in its plain form (elementary torch operations in 32 bits, rounded once at the end);
with `own` it makes the calls of paper_1812_09162_amd.binding.  exact() gives the same outputs from the
definitions in 64 bits.

Sizes are the query tower's own (256 columns, batches of 1,024, vectors of 96) and generic powers of two with odd ones
between.  Requests come as runs of neighbouring rows (sequences) or mixed (one token of each); the adapters' frequencies are
log-uniform, some rows have none.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# -------------------------------------------------------------------- cases --
def _dropout(name, **kw):
    return dict(dict(name=name, path="dropout", n=16_384, d=2048, t="bf16", p=0.1, residual=True), **kw)


def _adapter(name, **kw):
    return dict(dict(name=name, path="adapter", n=1, din=4096, dout=4096, r=16, adapters=64, t="bf16", to="bf16", ids="i64", runs=1,
                     missing=0.0, p=0.0, base=True, keep_t=False), **kw)


def _adapter_grad(name, **kw):
    return dict(dict(name=name, path="adapter_grad", n=16_384, din=4096, dout=4096, r=16, adapters=8, t="bf16", to="f32", ids="i64", runs=32,
                     missing=0.0, p=0.05, base=True), **kw)


def listed():
    return [
        # a training step of the query tower: its batch in float32
        _dropout("dropout_step", n=1024, d=256, t="f32", residual=False),
        # the residual stream of a training batch
        _dropout("dropout_batch"),
        # an odd width, fp16, a high rate
        _dropout("dropout_odd", n=10_000, d=1001, t="f16", p=0.25, residual=False),
        # one request's token beside a projection
        _adapter("adapter_request"),
        # one token of each of 64 requests, nearly every one with an adapter of its own; some have none
        _adapter("adapter_tokens", n=64, adapters=128, ids="i32", runs=0, missing=0.1),
        # sixteen requests' sequences in one batch
        _adapter("adapter_prefill", n=16_384, runs=16),
        # rows of many requests mixed, odd widths, fp16
        _adapter("adapter_mixed", n=8192, din=1000, dout=1001, r=8, adapters=500, t="f16", to="f16", runs=0, missing=0.05),
        # a wider projection and a high rank, the result in float32
        _adapter("adapter_rank", n=4096, din=2048, dout=8192, r=64, adapters=4, to="f32", runs=8),
        # the forward pass of training one adapter: dropout of its input, what the gradient reads kept
        _adapter("adapter_train", n=16_384, din=2048, dout=2048, r=32, adapters=1, p=0.05, keep_t=True),
        # the gradient of a training step of four small towers
        _adapter_grad("adapter_grad_step", n=1024, din=256, dout=96, r=8, adapters=4, t="f32", runs=0, p=0.1, base=False),
        # the gradient of a training batch of eight adapters
        _adapter_grad("adapter_grad_batch"),
        # the gradient of many adapters, few rows each, odd widths, fp16
        _adapter_grad("adapter_grad_many", n=10_000, din=1001, dout=700, r=12, adapters=200, t="f16", to="f16", runs=0, missing=0.05, p=0.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _size(rng, lo, hi):
    """A size of [lo, hi]: a multiple of 128 or 16 half of the time, else whatever comes."""
    v = _log_int(rng, lo, hi)
    step = rng.choice([128, 16, 1, 1])
    return v // step * step if v >= 2 * step else v


def draw(rng):
    path = rng.choice(["dropout", "adapter", "adapter", "adapter_grad", "adapter_grad"])
    t = rng.choice(["bf16", "bf16", "f16", "f32"])
    if path == "dropout":
        d = _size(rng, 16, 8192)
        return dict(path=path, n=_log_int(rng, 1, min(65_536, 33_000_000 // d)), d=d, t=t, p=rng.choice([0.05, 0.1, 0.5]), residual=rng.random() < 0.6)
    din, dout = _size(rng, 64, 8192), _size(rng, 64, 8192)
    r = rng.choice([4, 8, 8, 16, 16, 16, 32, 64, 128, rng.randint(1, 64)])
    adapters = _log_int(rng, 1, min(1000, 20_000_000 // (r * (din + dout))))
    values = 200_000_000 // (2 if t == "f32" else 1)  # read and written, by the largest
    most = min(32_768, values // (3 * din + 2 * dout), 1_300_000_000 // (r * (din + dout)), 400_000_000 // (adapters * r))
    base = dict(path=path, din=din, dout=dout, r=r, adapters=adapters, t=t, to=rng.choice([t, "f32"]), ids=rng.choice(["i32", "i64"]),
                missing=0.0, base=rng.random() < 0.8)
    if path == "adapter":
        p, n = rng.choice([0.0, 0.0, 0.1]), rng.choice([1, _log_int(rng, 2, min(most, 256)), _log_int(rng, 1, most)])
        base.update(keep_t=p > 0)
    else:
        p, n = rng.choice([0.0, 0.05, 0.1]), _log_int(rng, 1, most)
    base.update(n=n, p=p, runs=rng.choice([0, _log_int(rng, 1, min(n, 64))]))
    if (base["runs"] or n) >= 16:
        base.update(missing=rng.choice([0.0, 0.1]))
    return base


# ------------------------------------------------------------------- inputs --
def _dev():
    return torch.device("cuda", torch.cuda.current_device())


def _gen(seed, stream):
    g = torch.Generator(device=_dev())
    g.manual_seed((seed * 1000003 + stream * 7919 + 98765) & 0x7FFFFFFFFFFFFFFF)
    return g


def _values(n, d, seed, stream, t, spread=1.0):
    """Gaussian, every column with a spread of its own (log-normal), as the activations of a trained layer have."""
    x = torch.randn((n, d), generator=_gen(seed, stream), device=_dev(), dtype=torch.float32)
    x.mul_(torch.exp(0.5 * torch.randn((d,), generator=_gen(seed, stream + 1), device=_dev())).mul_(spread))
    return x.to(TYPES[t])


def _ids(case, seed):
    """An adapter for each row: of log-uniform frequency, for each row by itself or for each of `runs` sequences."""
    n, count = case["n"], case["runs"] or case["n"]
    u = torch.rand((2, count), generator=_gen(seed, 2), device=_dev(), dtype=torch.float64)
    i = (torch.pow(float(case["adapters"] + 1), u[0]) - 1.0).to(torch.int64).clamp_(0, case["adapters"] - 1)
    i[u[1] < case["missing"]] = -1
    if case["runs"]:
        cuts = torch.sort(torch.rand((count - 1,), generator=_gen(seed, 3), device=_dev(), dtype=torch.float64) * n)[0]
        i = i[torch.searchsorted(cuts, torch.arange(n, device=_dev(), dtype=torch.float64), right=True)]
    return i.to(torch.int32 if case["ids"] == "i32" else torch.int64).contiguous()


def prepare(case, seed):
    path, state, t = case["path"], dict(case), case["t"]
    if case["p"]:  # the generator's seed and the step of training
        state.update(state=torch.tensor([seed * 0x9E3779B97F4A7C15 % (1 << 63), 1000 + seed], device=_dev()), layer=5)
    if path == "dropout":
        state.update(x=_values(case["n"], case["d"], seed, 10, t))
        if case["residual"]:
            state.update(res=_values(case["n"], case["d"], seed, 20, t, 2.0))
        return state
    n, din, dout, r, count = (case[k] for k in ("n", "din", "dout", "r", "adapters"))
    state.update(index=_ids(case, seed), x=_values(n, din, seed, 10, t),
                 a=_values(count * r, din, seed, 30, t, din ** -0.5).view(count, r, din), b=_values(count * r, dout, seed, 40, t, 0.5).view(count, r, dout),
                 scales=torch.exp2(torch.randint(-2, 3, (count,), generator=_gen(seed, 4), device=_dev()).float()) * 0.7)
    if path == "adapter":
        if case["base"]:
            state.update(y0=_values(n, dout, seed, 50, case["to"], 2.0))
    else:
        state.update(dy=_values(n, dout, seed, 50, t, 0.1), kept=_values(n, r, seed, 60, "f32"))
        state["kept"][state["index"] < 0] = 0.0
        if case["base"]:
            state.update(dx0=_values(n, din, seed, 70, t, 0.2))
    return state


# -------------------------------------------------------------- plain forms --
LOW = 0xFFFFFFFF


def _round_of(c0, c1, c2, c3, k0, k1):
    p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # (64 bits, which wrap around; the halves are right)
    return (p1 >> 32 & LOW) ^ c1 ^ k0, p1 & LOW, (p0 >> 32 & LOW) ^ c3 ^ k1, p0 & LOW


def _threshold(p):
    return int(round(65536 * p))


def _factor(p):
    return 65536.0 / (65536 - _threshold(p))


def _kept(state, n, d):
    """The mask [n, d]: sixteen bits for each element from ten rounds of the generator Philox4x32 (Salmon et al., 2011), eight elements a call."""
    blocks = -(-d // 8)
    seed, step = state["state"][0], state["state"][1] & LOW
    k0, k1 = seed & LOW, seed >> 32 & LOW
    c = (torch.arange(blocks, device=_dev()).expand(n, blocks), torch.arange(n, device=_dev()).unsqueeze(1).expand(n, blocks), step.expand(n, blocks),
         torch.full((), state["layer"], device=_dev()).expand(n, blocks))
    one = lambda c, i: _round_of(*c, k0 + i * 0x9E3779B9 & LOW, k1 + i * 0xBB67AE85 & LOW)  # noqa: E731
    c = one(one(one(one(one(one(one(one(one(one(c, 0), 1), 2), 3), 4), 5), 6), 7), 8), 9)
    words = torch.stack(c, dim=2)
    halves = torch.stack([words & 0xFFFF, words >> 16], dim=3)
    return halves.reshape(n, blocks * 8)[:, :d] >= _threshold(state["p"])


def _plain_dropout(state):
    x = state["x"].float()
    y = torch.where(_kept(state, *x.shape), x * _factor(state["p"]), 0.0)
    if state["residual"]:
        y = y + state["res"].float()
    return y.to(state["x"].dtype)


def _of_adapters(state):
    """[n, adapters]: which adapter a row has."""
    return state["index"].long().unsqueeze(1) == torch.arange(state["adapters"], device=_dev())


def _dropped(state):
    """x with zeros where it is dropped, the mask, and the factor of the rest with the adapters' scales: [n, 1], zero without one."""
    x, index = state["x"].float(), state["index"].long()
    s = torch.where(index >= 0, state["scales"][index.clamp(min=0)], 0.0).unsqueeze(1)
    if state["p"]:
        mask = _kept(state, *x.shape)
        return torch.where(mask, x, 0.0), mask, s * _factor(state["p"])
    return x, None, s


def _plain_adapter(state):
    n, r, count, dout = state["n"], state["r"], state["adapters"], state["dout"]
    x, _, s = _dropped(state)
    if n <= count:  # every row its own weights
        of = state["index"].long().clamp(min=0)
        t = (state["a"][of].float() @ x.unsqueeze(2)).squeeze(2) * s
        y = (t.unsqueeze(1) @ state["b"][of].float()).squeeze(1)
    else:  # all adapters' products, of which a row keeps its own
        t = torch.where(_of_adapters(state).unsqueeze(2), (x @ state["a"].float().view(count * r, -1).t()).view(n, count, r), 0.0) * s.unsqueeze(2)
        y = t.view(n, count * r) @ state["b"].float().view(count * r, dout)
        t = t.sum(dim=1)
    if state["base"]:
        y = y + state["y0"].float()
    out = {"y": y.to(TYPES[state["to"]])}
    return dict(out, t=t) if state["keep_t"] else out


def _plain_adapter_grad(state):
    n, r, count, dout = state["n"], state["r"], state["adapters"], state["dout"]
    x, mask, s = _dropped(state)
    dy, its = state["dy"].float(), _of_adapters(state).unsqueeze(2)
    a, b = state["a"].float().view(count * r, -1), state["b"].float().view(count * r, dout)
    u = (torch.where(its, (dy @ b.t()).view(n, count, r), 0.0) * s.unsqueeze(2)).view(n, count * r)
    t = torch.where(its, state["kept"].unsqueeze(1), 0.0).view(n, count * r)
    dx = u @ a
    if state["p"]:
        dx = torch.where(mask, dx, 0.0)
    if state["base"]:
        dx = dx + state["dx0"].float()
    da, db = (u.t() @ x).view(count, r, -1), (t.t() @ dy).view(count, r, dout)
    return {"dx": dx.to(TYPES[state["t"]]), "da": da.to(TYPES[state["to"]]), "db": db.to(TYPES[state["to"]])}


# ------------------------------------------------------ the framework's calls --
def _own(state):
    from paper_1812_09162_amd import binding as qb
    path, drop = state["path"], dict(p=state["p"], state=state.get("state"), layer=state.get("layer", 0))
    if path == "dropout":
        return qb.vec_dropout(state["x"], residual=state.get("res"), **drop)
    if path == "adapter":
        y, t = qb.vec_adapter(state["x"], state["a"], state["b"], state["index"], scales=state["scales"], base=state.get("y0"), want_t=state["keep_t"],
                              dtype=TYPES[state["to"]], **drop)
        return {"y": y, "t": t} if state["keep_t"] else {"y": y}
    dx, da, db = qb.vec_adapter_grad(state["dy"], state["x"], state["kept"], state["a"], state["b"], state["index"], scales=state["scales"],
                                     dx_base=state.get("dx0"), dtype=TYPES[state["to"]], **drop)
    return {"dx": dx, "da": da, "db": db}


def run(state):
    if own:
        return _own(state)
    return {"dropout": _plain_dropout, "adapter": _plain_adapter, "adapter_grad": _plain_adapter_grad}[state["path"]](state)


# --------------------------------------------------------------- definitions --
def _mask64(state, n, d):
    """The mask by the generator's definition, in unsigned numbers on the host."""
    seed, step = (int(v) for v in state["state"].cpu())
    key = [np.uint64(seed & LOW), np.uint64(seed >> 32 & LOW)]
    shape, shift, low = (n, -(-d // 8)), np.uint64(32), np.uint64(LOW)
    c = [np.broadcast_to(np.arange(shape[1], dtype=np.uint64)[None, :], shape), np.broadcast_to(np.arange(n, dtype=np.uint64)[:, None], shape),
         np.broadcast_to(np.uint64(step & LOW), shape), np.broadcast_to(np.uint64(state["layer"]), shape)]
    for _ in range(10):
        left, right = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(right >> shift) ^ c[1] ^ key[0], right & low, (left >> shift) ^ c[3] ^ key[1], left & low]
        key = [(key[0] + np.uint64(0x9E3779B9)) & low, (key[1] + np.uint64(0xBB67AE85)) & low]
    numbers = np.empty(shape + (8,), dtype=np.uint16)
    for w in range(4):
        numbers[:, :, 2 * w] = (c[w] & np.uint64(0xFFFF)).astype(np.uint16)
        numbers[:, :, 2 * w + 1] = (c[w] >> np.uint64(16)).astype(np.uint16)
    kept = numbers.reshape(n, -1)[:, :d].astype(np.int64) >= int(round(65536 * state["p"]))
    return torch.from_numpy(kept).to(_dev())


def exact(case, seed):
    state, path = prepare(case, seed), case["path"]
    x = state["x"].double()
    n = x.shape[0]
    mask, factor = None, 1.0
    if case["p"]:
        mask, factor = _mask64(state, n, x.shape[1]), 1.0 / (1.0 - round(65536 * case["p"]) / 65536.0)
        x = x * mask * factor
    if path == "dropout":
        return x + state["res"].double() if case["residual"] else x
    index = state["index"].long()
    rows = {e: (index == e).nonzero()[:, 0] for e in torch.unique(index).tolist() if e >= 0}
    if path == "adapter":
        y = state["y0"].double() if case["base"] else torch.zeros((n, case["dout"]), dtype=torch.float64, device=_dev())
        t = torch.zeros((n, case["r"]), dtype=torch.float64, device=_dev())
        for e, at in rows.items():
            t[at] = (x[at] @ state["a"][e].double().t()) * state["scales"][e].double()
            y[at] += t[at] @ state["b"][e].double()
        return {"y": y, "t": t} if case["keep_t"] else {"y": y}
    dx = state["dx0"].double() if case["base"] else torch.zeros_like(x)
    da, db = torch.zeros(state["a"].shape, dtype=torch.float64, device=_dev()), torch.zeros(state["b"].shape, dtype=torch.float64, device=_dev())
    for e, at in rows.items():
        dy = state["dy"][at].double()
        u = (dy @ state["b"][e].double().t()) * state["scales"][e].double()
        part = u @ state["a"][e].double()
        dx[at] += part * mask[at] * factor if case["p"] else part
        da[e] = u.t() @ x[at]
        db[e] = state["kept"][at].double().t() @ dy
    return {"dx": dx, "da": da, "db": db}


# ---------------------------------------------------------------------- work --
def work(case):
    n, t = case["n"], BYTES[case["t"]]
    if case["path"] == "dropout":
        values = n * case["d"]
        return {"bytes": values * t * (3 if case["residual"] else 2), "flops": 3 * values}
    din, dout, r, to = case["din"], case["dout"], case["r"], BYTES[case["to"]]
    named = min(case["adapters"], case["runs"] or n)
    moved = n * (4 if case["ids"] == "i32" else 8) + named * r * (din + dout) * t
    if case["path"] == "adapter":
        moved += n * din * t + n * dout * to * (2 if case["base"] else 1) + (n * r * 4 if case["keep_t"] else 0)
        return {"bytes": moved, "flops": 2 * n * r * (din + dout)}
    moved += n * (din + dout + din * (2 if case["base"] else 1)) * t + n * r * 4 + case["adapters"] * r * (din + dout) * to
    return {"bytes": moved, "flops": 4 * n * r * (din + dout)}
