"""vec_adapter and vec_adapter_grad against their definitions in 64 bits.  Tolerances count roundings: half a step of the result's type for the last,
and for sums of N float32 terms N steps of 2^-24 of the sum of magnitudes (whatever their order); products of bfloat16 and fp16 values are exact, and
a factor split into three bfloat16 numbers loses at most 2^-23 of each product."""
import math

import pytest
import torch

from philox import factor, kept
from test_gpu_vec import BF16, F16, F32, U, WIDE, close, dev, framed, half_step, rnd, untouched

pytestmark = pytest.mark.gpu
SEED, STEP, LAYER = 0x0BAD_5EED_0123_4567, 12, 3


@pytest.fixture(scope="module")
def qb():
    from paper_1812_09162_amd import binding
    binding.load()
    return binding


def state(step=STEP):
    return torch.tensor([SEED, step], device=dev())


def make_ids(n, adapters, kind, seed=5, dtype=torch.int64):
    g = torch.Generator().manual_seed(seed + n)
    u = torch.rand((n,), generator=g, dtype=torch.float64)
    even = (u * adapters).long().clamp(max=max(adapters - 1, 0))
    skew = ((adapters + 1) ** u - 1).long().clamp(0, max(adapters - 1, 0))
    ids = {"even": even, "skew": skew, "none": torch.full((n,), -1), "one": torch.full((n,), adapters - 1), "some": torch.where(u < 0.3, -1, skew),
           "outside": torch.where(u < 0.2, -7, torch.where(u < 0.4, adapters + (u * 100).long(), even)),
           "runs": (torch.arange(n) * 7 // max(n, 1) * 5) % max(adapters, 1),
           "alternate": torch.arange(n) % max(adapters, 1)}[kind]
    return ids.to(dtype).to(dev())


def weights(adapters, r, din, dout, t, seed=30):
    return (rnd((adapters * r, din), seed, t, din ** -0.5).view(adapters, r, din), rnd((adapters * r, dout), seed + 1, t, 0.5).view(adapters, r, dout),
            torch.exp2(torch.arange(adapters, device=dev()).float() % 5 - 2) * 0.7)


def terms(x, a, b, ids, scales, p, step=STEP):
    """Rows with their adapters; x after dropout without the factor, the mask, scale times factor per row (all of 64 bits)."""
    n, din = x.shape
    m = kept(range(n), din, p, SEED, step, LAYER).to(dev()) if p else torch.ones((n, din), dtype=torch.bool, device=dev())
    of = {e: (ids.long() == e).nonzero()[:, 0] for e in torch.unique(ids.long()).tolist() if 0 <= e < a.shape[0]}
    s = torch.zeros((n, 1), dtype=torch.float64, device=dev())
    for e, at in of.items():
        s[at] = float((scales[e] if scales is not None else 1.0)) * (factor(p) if p else 1.0)
    return of, torch.where(m, x.double(), 0.0), m, s


def forward64(x, a, b, ids, scales, base, p, step=STEP):
    """y, t and what they may be off by before y's own rounding."""
    n, din = x.shape
    r, dout = a.shape[1], b.shape[2]
    of, xd, m, s = terms(x, a, b, ids, scales, p, step)
    y = torch.zeros((n, dout), dtype=torch.float64, device=dev()) if base is None else base.double()
    ty, t, tt = y.abs() * 2 * U, torch.zeros((n, r), dtype=torch.float64, device=dev()), torch.zeros((n, r), dtype=torch.float64, device=dev())
    for e, at in of.items():
        t[at] = xd[at] @ a[e].double().t() * s[at]
        tt[at] = (xd[at].abs() @ a[e].double().abs().t()) * s[at].abs() * U * (din + 8)
        y[at] = y[at] + t[at] @ b[e].double()
        ty[at] += (tt[at] + t[at].abs() * U * (r + 8)) @ b[e].double().abs()
    return y, ty, t, tt


def check(qb, n, din, dout, r, adapters, kind, t, to, p=0.0, base=True, scales=True, keep=True, idt=torch.int64):
    x, xs = framed(rnd((n, din), 1, t))
    a, b, sc = weights(adapters, r, din, dout, t)
    if not scales:
        sc = None
    ids = make_ids(n, adapters, kind, dtype=idt)
    b0 = framed(rnd((n, dout), 4, to, 2.0))[0] if base else None
    y64, ty, t64, tt = forward64(x, a, b, ids, sc, b0, p)
    call = dict(scales=sc, base=b0, p=p, state=state() if p else None, layer=LAYER, dtype=to)
    y, kept_t = qb.vec_adapter(x, a, b, ids, want_t=keep, **call)
    close(y, y64, ty + half_step(y64, to))
    assert (kept_t is not None) == keep
    if keep:
        close(kept_t, t64, tt + half_step(t64, F32))
    out, store = framed(torch.zeros((n, dout), dtype=to, device=dev()))
    was = store.clone()
    qb.vec_adapter(x, a, b, ids, out=(out, None), **call)
    assert torch.equal(out, y) and untouched(out, store, was)
    if base:
        out, store = framed(b0)
        was = store.clone()
        qb.vec_adapter(x, a, b, ids, out=(out, None), **dict(call, base=out))
        assert torch.equal(out, y) and untouched(out, store, was)


TYPES = [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32), (F32, F32)]


@pytest.mark.parametrize("t,to", TYPES)
@pytest.mark.parametrize("n,din,dout,r,adapters,kind,p", [
    (1, 1, 1, 1, 1, "one", 0.0), (1, 256, 512, 16, 5, "one", 0.0), (3, 100, 77, 7, 3, "even", 0.5), (17, 129, 1000, 8, 40, "even", 0.0), (64, 1024, 520, 16, 100, "some", 0.0),
    (512, 96, 200, 4, 9, "skew", 0.1), (513, 96, 200, 4, 9, "skew", 0.1), (700, 1001, 333, 17, 30, "outside", 0.0), (1500, 300, 513, 32, 3, "runs", 0.25),
    (1100, 256, 96, 33, 20, "skew", 0.0), (2000, 160, 264, 64, 7, "alternate", 0.0), (1030, 137, 140, 100, 2, "even", 0.1), (1300, 264, 136, 128, 3, "skew", 0.0), (90, 500, 60, 256, 4, "even", 0.0),
    (1200, 130, 70, 200, 4, "even", 0.5), (5000, 64, 72, 12, 1, "some", 0.1), (3000, 40, 33, 5, 2000, "even", 0.0), (2500, 31, 9, 3, 1023, "skew", 0.0)])
def test_adapter(qb, n, din, dout, r, adapters, kind, p, t, to):
    check(qb, n, din, dout, r, adapters, kind, t, to, p)


@pytest.mark.parametrize("kind", ["none", "one", "outside", "runs"])
@pytest.mark.parametrize("n", [1, 40, 600, 1025])
def test_adapter_variants(qb, n, kind):
    check(qb, n, 200, 136, 16, 6, kind, BF16, BF16, base=False, scales=False, keep=True, idt=torch.int32)
    check(qb, n, 200, 136, 16, 6, kind, F16, F32, p=0.1, base=False, keep=False)
    check(qb, n, 200, 136, 40, 1, kind, F32, F32, base=True, scales=False, idt=torch.int32)


def test_large_products(qb):
    check(qb, 4097, 4096, 4104, 16, 9, "runs", BF16, BF16)
    check(qb, 2000, 8192, 1000, 48, 300, "skew", F16, F16, p=0.1)
    check(qb, 2, 16_384, 20_000, 8, 2, "even", BF16, F32)


def test_ids_far_outside(qb):
    """Numbers whose low 32 bits would name an adapter name none."""
    x, (a, b, s) = rnd((6, 64), 1), weights(3, 4, 64, 32, F32)
    base = rnd((6, 32), 2)
    ids = torch.tensor([1 << 32, (1 << 32) + 1, -(1 << 32), -(1 << 63), (1 << 63) - 1, 3], device=dev())
    y, t = qb.vec_adapter(x, a, b, ids, scales=s, base=base, want_t=True)
    assert torch.equal(y, base) and not bool(t.any())
    for da in qb.vec_adapter_grad(base, x, t, a, b, ids, scales=s)[1:]:
        assert not bool(da.any())


def test_no_adapters_and_no_rows(qb):
    x, (a, b, _) = rnd((5, 16), 1, BF16), weights(2, 4, 16, 24, BF16)
    base = rnd((5, 24), 2, BF16)
    ids = torch.zeros(5, dtype=torch.int32, device=dev())
    y, t = qb.vec_adapter(x, a[:0], b[:0], ids, base=base, want_t=True)
    assert torch.equal(y, base) and not bool(t.any())
    y, t = qb.vec_adapter(x[:0], a, b, ids[:0], want_t=True)
    assert y.shape == (0, 24) and t.shape == (0, 4)
    dx, da, db = qb.vec_adapter_grad(base, x, torch.zeros((5, 4), device=dev()), a[:0], b[:0], ids, dx_base=x)
    assert torch.equal(dx, x) and da.shape == (0, 4, 16) and db.shape == (0, 4, 24)
    dx, da, db = qb.vec_adapter_grad(base[:0], x[:0], torch.zeros((0, 4), device=dev()), a, b, ids[:0])
    assert dx.shape == (0, 16) and not bool(da.any()) and not bool(db.any())
    old = torch.ones_like(da)
    qb.vec_adapter_grad(base[:0], x[:0], torch.zeros((0, 4), device=dev()), a, b, ids[:0], out=(None, old, db), accumulate=True)
    assert bool((old == 1).all())


def test_factors_of_other_layouts(qb):
    """Rows and adapters apart, one adapter's weights for all ids, weights of a slice of the ranks."""
    n, din, dout, r = 700, 130, 90, 6
    x, ids = rnd((n, din), 1, BF16), make_ids(n, 4, "even")
    big_a, big_b = rnd((8, 9, din + 7), 2, BF16, 0.1), rnd((8, 9, dout + 5), 3, BF16)
    for a, b in ((big_a[::2, 1:1 + r, 3:3 + din], big_b[4:, :r, 1:1 + dout]), (big_a[3:4, :r, :din].expand(4, r, din), big_b[:1, :r, :dout].expand(4, r, dout)),
                 (big_a[:4, ::2, :din][:, :4], big_b[:4, 1::2, :dout])):
        y, t = qb.vec_adapter(x, a, b, ids, want_t=True)
        y2, t2 = qb.vec_adapter(x, a.contiguous(), b.contiguous(), ids, want_t=True)
        assert torch.equal(y, y2) and torch.equal(t, t2)
        dy = rnd((n, dout), 4, BF16)
        for u, v in zip(qb.vec_adapter_grad(dy, x, t, a, b, ids), qb.vec_adapter_grad(dy, x, t, a.contiguous(), b.contiguous(), ids)):
            assert torch.equal(u, v)


@pytest.mark.parametrize("n", [30, 1300])
@pytest.mark.parametrize("t", WIDE)
def test_what_takes_no_part_is_not_read(qb, n, t):
    """NaN in rows without an adapter, in adapters without a row, in dropped elements; an infinity stays in its row."""
    adapters, din, dout, r, p = 5, 150, 70, 10, 0.5
    x, (a, b, s) = rnd((n, din), 1, t), weights(adapters, r, din, dout, t)
    ids = make_ids(n, adapters, "some")
    ids[ids == 3] = 2
    base, dy = rnd((n, dout), 2, t), rnd((n, dout), 3, t)
    call = dict(scales=s, p=p, state=state(), layer=LAYER)
    y, kt = qb.vec_adapter(x, a, b, ids, base=base, want_t=True, **call)
    grads = qb.vec_adapter_grad(dy, x, kt, a, b, ids, **call)
    m = kept(range(n), din, p, SEED, STEP, LAYER).to(dev())
    bad = x.clone()
    bad[~m] = math.nan
    bad[ids < 0] = math.nan
    a[3], b[3], s[3] = math.nan, math.inf, math.nan
    y2, kt2 = qb.vec_adapter(bad, a, b, ids, base=base, want_t=True, **call)
    dy2, kt3 = dy.clone(), kt2.clone()
    dy2[ids < 0], kt3[ids < 0] = math.nan, math.inf
    assert torch.equal(y, y2) and torch.equal(kt, kt2)
    for u, v in zip(grads, qb.vec_adapter_grad(dy2, bad, kt3, a, b, ids, **call)):
        assert torch.equal(u, v)
    row = int((ids >= 0).nonzero()[n // 4, 0])
    col = int(m[row].nonzero()[5, 0])
    bad[row, col] = math.inf
    y3, _ = qb.vec_adapter(bad, a, b, ids, base=base, **call)
    others = torch.arange(n, device=dev()) != row
    assert torch.equal(y3[others], y[others]) and not bool(y3[row].isfinite().any())
    dx, da, db = qb.vec_adapter_grad(dy, bad, kt, a, b, ids, **call)
    assert torch.equal(dx, grads[0]) and torch.equal(db, grads[2])
    e, cols = int(ids[row]), torch.arange(din, device=dev()) != col
    assert torch.equal(da[:, :, cols], grads[1][:, :, cols]) and not bool(da[e, :, col].isfinite().any())


def test_small_and_large_values(qb):
    """fp16 numbers below its normal range, t far outside it: t is not rounded to 16 bits."""
    n, din, dout, r = 40, 64, 48, 8
    ids = torch.zeros(n, dtype=torch.int64, device=dev())
    for sx, sb, ss in ((2.0 ** -20, 1.0, 2.0 ** 12), (100.0, 2.0 ** -14, 1.0), (1.0, 1.0, 2.0 ** -30)):
        x, a, b = rnd((n, din), 1, F16, sx), rnd((1, r, din), 2, F16), rnd((1, r, dout), 3, F16, sb)
        s = torch.full((1,), ss, device=dev())
        y64, ty, t64, tt = forward64(x, a, b, ids, s, None, 0.0)
        y, t = qb.vec_adapter(x, a, b, ids, scales=s, dtype=F32, want_t=True)
        close(t, t64, tt + half_step(t64, F32))
        close(y, y64, ty + half_step(y64, F32))


def test_dropout_is_that_of_the_other_call(qb):
    """p = 1/2, whose factor is exact: the same bits as the adapters on what vec_dropout returns."""
    n, din, dout, r = 900, 520, 130, 12
    x, ids = rnd((n, din), 1, F16), make_ids(n, 6, "some")
    a, b, s = weights(6, r, din, dout, F16)
    y, t = qb.vec_adapter(x, a, b, ids, scales=s, p=0.5, state=state(), layer=LAYER, want_t=True)
    y2, t2 = qb.vec_adapter(qb.vec_dropout(x, 0.5, state(), LAYER), a, b, ids, scales=s, want_t=True)
    assert torch.equal(t, t2) and torch.equal(y, y2)


# --------------------------------------------------------------- gradient --
def gradient64(dy, x, t, a, b, ids, scales, dx_base, p, step=STEP):
    n, din = x.shape
    r, dout = a.shape[1], b.shape[2]
    of, xd, m, s = terms(x, a, b, ids, scales, p, step)
    d, td = dy.double(), t.double()
    zero = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=dev())  # noqa: E731
    dx = zero(n, din) if dx_base is None else dx_base.double()
    tx, da, ta, db, tb = dx.abs() * 2 * U, zero(*a.shape), zero(*a.shape), zero(*b.shape), zero(*b.shape)
    for e, at in of.items():
        u = d[at] @ b[e].double().t() * s[at]
        tu = (d[at].abs() @ b[e].double().abs().t()) * s[at].abs() * U * (dout + 8)
        dx[at] += torch.where(m[at], u @ a[e].double(), 0.0)
        tx[at] += (tu + u.abs() * U * (r + 8)) @ a[e].double().abs()
        da[e] = u.t() @ xd[at]
        ta[e] = tu.t() @ xd[at].abs() + (u.abs().t() @ xd[at].abs()) * U * (len(at) + 8)
        db[e] = td[at].t() @ d[at]
        tb[e] = (td[at].abs().t() @ d[at].abs()) * U * (len(at) + 8)
    return (dx, tx), (da, ta), (db, tb)


def check_grad(qb, n, din, dout, r, adapters, kind, t, to, p=0.0, base=True, scales=True, idt=torch.int64):
    x, _ = framed(rnd((n, din), 1, t))
    dy, _ = framed(rnd((n, dout), 2, t, 0.3))
    a, b, sc = weights(adapters, r, din, dout, t)
    if not scales:
        sc = None
    ids = make_ids(n, adapters, kind, dtype=idt)
    kt = rnd((n, r), 3, F32)
    dx0 = framed(rnd((n, din), 4, t))[0] if base else None
    want = gradient64(dy, x, kt, a, b, ids, sc, dx0, p)
    call = dict(scales=sc, p=p, state=state() if p else None, layer=LAYER)
    got = qb.vec_adapter_grad(dy, x, kt, a, b, ids, dx_base=dx0, dtype=to, **call)
    for g, (ref, tol), ty in zip(got, want, (t, to, to)):
        assert g.dtype == ty
        close(g, ref, tol + half_step(ref, ty))
    # into views, dx in place of dx_base, sums added to what is there
    dx, xs = framed(dx0 if base else torch.zeros((n, din), dtype=t, device=dev()))
    wx = xs.clone()
    da0, db0 = rnd((adapters * r, din), 5, to), rnd((adapters * r, dout), 6, to)
    (da, sa), (db, sb) = framed(da0), framed(db0)
    wa, wb = sa.clone(), sb.clone()
    v = lambda m, d: m.as_strided((adapters, r, d), (r * m.stride(0), m.stride(0), 1), m.storage_offset())  # noqa: E731
    qb.vec_adapter_grad(dy, x, kt, a, b, ids, dx_base=dx if base else None, out=(dx, v(da, din), v(db, dout)), accumulate=True, **call)
    assert torch.equal(dx, got[0]) and untouched(dx, xs, wx) and untouched(da, sa, wa) and untouched(db, sb, wb)
    for g, g0, (ref, tol) in ((da, da0, want[1]), (db, db0, want[2])):
        ref, tol = ref.view(g.shape) + g0.double(), tol.view(g.shape)
        close(g, ref, tol + U * (ref.abs() + g0.double().abs()) + half_step(ref, to))
    again = qb.vec_adapter_grad(dy, x, kt, a, b, ids, want_dx=False, dtype=to, **call)
    assert again[0] is None and torch.equal(again[1], got[1]) and torch.equal(again[2], got[2])


@pytest.mark.parametrize("t,to", TYPES)
@pytest.mark.parametrize("n,din,dout,r,adapters,kind,p", [
    (1, 1, 1, 1, 1, "one", 0.0), (1, 256, 96, 8, 3, "one", 0.1), (5, 33, 600, 16, 2, "even", 0.0), (127, 100, 40, 7, 1, "one", 0.0), (129, 136, 77, 16, 4, "some", 0.5),
    (700, 96, 200, 4, 9, "skew", 0.1), (1024, 256, 96, 8, 4, "alternate", 0.1), (1300, 1001, 333, 17, 30, "outside", 0.0), (2049, 300, 513, 32, 3, "runs", 0.25),
    (1100, 256, 96, 33, 20, "skew", 0.0), (3000, 160, 264, 64, 2, "even", 0.0), (1030, 137, 140, 100, 2, "even", 0.1), (300, 500, 60, 256, 4, "even", 0.0),
    (9000, 64, 72, 12, 1, "some", 0.1), (3000, 40, 33, 5, 2000, "even", 0.0), (2500, 31, 9, 3, 1023, "none", 0.0)])
def test_adapter_grad(qb, n, din, dout, r, adapters, kind, p, t, to):
    check_grad(qb, n, din, dout, r, adapters, kind, t, to, p)


def test_adapter_grad_variants(qb):
    check_grad(qb, 1500, 200, 136, 16, 6, "one", BF16, F32, base=False, scales=False, idt=torch.int32)
    check_grad(qb, 700, 200, 136, 16, 6, "runs", F16, F16, p=0.1, base=False, idt=torch.int32)
    check_grad(qb, 20_000, 520, 1032, 16, 5, "runs", BF16, F32, p=0.05)
    check_grad(qb, 6000, 4096, 2056, 24, 40, "skew", BF16, BF16)


def test_adapter_grad_against_differences(qb):
    """Central differences of the forward pass in float32, whose error is bounded by the roundings of y and the second-order term, which is zero: y is
    linear in x, a and b each."""
    n, din, dout, r, adapters, p = 60, 48, 40, 5, 3, 0.25
    x, (a, b, s), ids = rnd((n, din), 1), weights(adapters, r, din, dout, F32), make_ids(n, adapters, "some")
    dy = rnd((n, dout), 2)
    call = dict(scales=s, p=p, state=state(), layer=LAYER)
    y, t = qb.vec_adapter(x, a, b, ids, want_t=True, **call)
    dx, da, db = qb.vec_adapter_grad(dy, x, t, a, b, ids, **call)
    for which, grad in ((0, dx), (1, da), (2, db)):
        v = [torch.zeros_like(x), torch.zeros_like(a), torch.zeros_like(b)]
        v[which] = rnd(tuple(grad.shape), 7 + which)
        f = [(dy.double() * qb.vec_adapter(x + h * v[0], a + h * v[1], b + h * v[2], ids, **call)[0].double()).sum() for h in (1.0, -1.0)]
        tol = 0.0
        for h in (1.0, -1.0):
            y64, ty, _, _ = forward64(x + h * v[0], a + h * v[1], b + h * v[2], ids, s, None, p)
            tol += float((dy.double().abs() * (ty + U * y64.abs())).sum()) / 2
            # x + h v, a + h v and b + h v are rounded themselves
            tol += float((dy.double().abs() * forward64(x.abs() + v[0].abs(), a.abs() + v[1].abs(), b.abs() + v[2].abs(), ids, s, None, p)[0]).sum()) * 2 * U
        got = (grad.double() * v[which].double()).sum()
        (dx64, tx), (da64, ta), (db64, tb) = gradient64(dy, x, t, a, b, ids, s, None, p)
        tol += float(((tx, ta, tb)[which] * v[which].double().abs()).sum()) + 2 * U * float((grad.double().abs() * v[which].double().abs()).sum()) + 4 * U * float(
            (dy.double().abs() * y.double().abs()).sum())
        assert abs(float((f[0] - f[1]) / 2 - got)) <= tol


# ------------------------------------------------- calls beside each other --
def test_same_bits_twice_and_on_another_stream(qb):
    n, din, dout, r, adapters = 3000, 264, 520, 16, 11
    x, (a, b, s), ids = rnd((n, din), 1, BF16), weights(adapters, r, din, dout, BF16), make_ids(n, adapters, "skew")
    dy, base = rnd((n, dout), 2, BF16), rnd((n, dout), 3, BF16)
    call = dict(scales=s, p=0.1, state=state(), layer=LAYER)
    y, t = qb.vec_adapter(x, a, b, ids, base=base, want_t=True, **call)
    first = (y, t, *qb.vec_adapter_grad(dy, x, t, a, b, ids, **call))
    torch.cuda.synchronize()
    for stream in (None, torch.cuda.Stream()):
        y, t2 = qb.vec_adapter(x, a, b, ids, base=base, want_t=True, stream=stream, **call)
        got = (y, t2, *qb.vec_adapter_grad(dy, x, t, a, b, ids, stream=stream, **call))
        torch.cuda.synchronize()
        for u, v in zip(first, got):
            assert torch.equal(u, v)


@pytest.mark.parametrize("n", [3, 300, 2000])
def test_graphs_that_share_a_workspace(qb, n):
    """Forward and gradient recorded in two graphs over one workspace, replayed in turn with eager work between, under steps that move on."""
    din, dout, r, adapters = 200, 264, 12, 7
    x, (a, b, s), ids = rnd((n, din), 1, F16), weights(adapters, r, din, dout, F16), make_ids(n, adapters, "some")
    dy, base, st = rnd((n, dout), 2, F16), rnd((n, dout), 3, F16), state()
    ws = torch.empty(max(qb.vec_adapter_workspace_bytes(n, din, dout, r, adapters, F16), qb.vec_adapter_grad_workspace_bytes(n, din, dout, r, adapters, F16)),
                     dtype=torch.uint8, device=dev())
    y, t, dx = torch.empty_like(base), torch.empty((n, r), device=dev()), torch.empty_like(x)
    da, db = torch.empty((adapters, r, din), device=dev()), torch.empty((adapters, r, dout), device=dev())
    call = dict(scales=s, p=0.2, state=st, layer=LAYER, workspace=ws)
    fwd = lambda: qb.vec_adapter(x, a, b, ids, base=base, out=(y, t), **call)  # noqa: E731
    bwd = lambda: qb.vec_adapter_grad(dy, x, t, a, b, ids, out=(dx, da, db), **call)  # noqa: E731
    fwd(), bwd()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        fwd()
    with torch.cuda.graph(graphs[1]):
        bwd()
        st[1] += 1
    for i in range(4):
        for o in (y, t, dx, da, db):
            o.fill_(7.0)
        ws.fill_(255)
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        eager = dict(scales=s, p=0.2, state=state(STEP + i), layer=LAYER)
        y2, t2 = qb.vec_adapter(x, a, b, ids, base=base, want_t=True, **eager)
        for u, v in zip((y, t, dx, da, db), (y2, t2, *qb.vec_adapter_grad(dy, x, t2, a, b, ids, **eager))):
            assert torch.equal(u, v)


def test_rows_beyond_32_bits(qb):
    """Elements past 2^32 of x, y and the adapters."""
    n, d, r = 530_000, 8200, 4
    x = torch.ones((n, d), dtype=BF16, device=dev())
    a, b = rnd((3, r, d), 1, BF16, 0.1), rnd((3, r, d), 2, BF16)
    ids = make_ids(n, 3, "runs")
    rows = torch.tensor([0, 1, 262_144, 523_775, 523_776, 523_777, n - 1], device=dev())
    x[rows] = rnd((7, d), 3, BF16)
    y, _ = qb.vec_adapter(x, a, b, ids, out=(torch.empty_like(x), None))
    rest = torch.ones(n, dtype=torch.bool, device=dev())
    rest[rows] = False
    for at in [rows, *(((ids == e) & rest).nonzero()[::3000, 0] for e in range(3))]:  # (sums are within their roundings; other places may add up in another order)
        y64, ty, _, _ = forward64(x[at], a, b, ids[at], None, None, 0.0)
        close(y[at], y64, ty + half_step(y64, BF16))
    del y
    big = torch.zeros((70, 64, 1 << 20), dtype=BF16, device=dev())
    big[69, 63] = 1.0
    x = torch.ones((2, 1 << 20), dtype=BF16, device=dev())
    _, t = qb.vec_adapter(x, big, rnd((70, 64, 8), 4, BF16), torch.tensor([69, 0], device=dev()), want_t=True)
    assert float(t[0, 63]) == 2 ** 20 and not bool(t[0, :63].any()) and not bool(t[1].any())


def test_refusals(qb):
    x, (a, b, s), ids = rnd((6, 16), 1), weights(3, 4, 16, 24, F32), torch.zeros(6, dtype=torch.int64, device=dev())
    dy, t, st = rnd((6, 24), 2), rnd((6, 4), 3), state()
    ok = dict(x=x, a=a, b=b, ids=ids, scales=s)
    bad = [dict(a=a[0]), dict(a=a.half()), dict(b=b[:2]), dict(b=b[:, :3]), dict(a=a[:, :, :8]), dict(ids=ids[:5]), dict(ids=ids.short()), dict(ids=ids.cpu()),
           dict(scales=s[:2]), dict(scales=s.double()), dict(a=a.transpose(1, 2).contiguous().transpose(1, 2)), dict(p=0.5), dict(p=1.0, state=st),
           dict(workspace=torch.empty(256, dtype=torch.uint8, device=dev())), dict(x=x.double())]
    for kw in bad + [dict(base=dy[:5]), dict(base=dy.half()), dict(dtype=BF16), dict(out=(dy.half(), None)), dict(out=(dy, t[:, :3])), dict(out=(dy, rnd((6, 5), 1)[:, :4]))]:
        with pytest.raises(qb.QadcError):
            qb.vec_adapter(**dict(ok, **kw))
    ok.update(dy=dy, t=t)
    for kw in bad + [dict(dy=dy[:5]), dict(t=t[:, :3]), dict(t=t.half()), dict(dx_base=x.half()), dict(dtype=F16), dict(accumulate=True), dict(want_dx=False, dx_base=x),
                     dict(out=(None, a.clone(), a.clone())), dict(out=(None, a.new_zeros(4, 16).expand(3, 4, 16), b.clone()))]:
        with pytest.raises(qb.QadcError):
            qb.vec_adapter_grad(**dict(ok, **kw))
