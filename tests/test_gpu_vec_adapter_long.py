"""The adapters' forms that ordinary training batches take: sums over rows in pieces of several stages, dx with the kept bits of the mask at ranks above 32,
tiles of 32 rows at high ranks, and gradients of tensors whose elements pass 2^32.  Tolerances as in test_gpu_vec_adapter."""
import pytest
import torch

from philox import factor
from test_gpu_vec import BF16, F16, F32, WIDE, dev, rnd
from test_gpu_vec_adapter import LAYER, STEP, check, check_grad, gradient64, state, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qb():
    from paper_1812_09162_amd import binding
    binding.load()
    return binding


# ------------------------------------------------- pieces of several stages --
def pieces(total, n, din, dout, r, adapters):
    """Lengths of the pieces (of da's sums, of db's) and slabs that give a gradient's workspace of `total` bytes: the sorted keys and positions and where the adapters
    begin, parts of u of each slab, two slots of sums a piece, and a word of the mask for eight columns of four rows."""
    up = lambda v: -(-v // 256) * 256  # noqa: E731
    known = 2 * up(4 * n) + up(4 * (adapters + 1)) + (up(-(-n // 4) * (din // 8) * 4) if din % 8 == 0 and dout >= 4 else 0)
    sums = lambda d, k: up(-(-n // k) * 2 * r * (-(-d // 8) * 8) * 4)  # noqa: E731
    lengths = [16 << i for i in range(7)]
    return {(a, b) for s in range(1, 17) for a in lengths for b in lengths if known + up(s * n * (-(-r // 16) * 16) * 4) + sums(din, a) + sums(dout, b) == total}


# Runs whose borders lie at, before and behind a stage's (128 positions) and a piece's, at odd places, and that hold several pieces; adapters 5 and 9 have no row.
RUNS = [127, 2, 126, 1, 128, 0, 129, 383, 512, 0, 641, 1023, 1024, 1025, 2050, 3000, 6201]
MISSING = 128  # rows without an adapter

# (rows behind the last run, columns, ranks, types, dropout) and the lengths of the two sums' pieces
PIECES = [
    ((0, 2048, 2056, 16, F16, F16, 0.0), (256, 256)),
    ((0, 2056, 2048, 12, BF16, F32, 0.5), (256, 256)),
    ((0, 4100, 4104, 16, BF16, F32, 0.0), (512, 512)),
    ((0, 4104, 4100, 16, F16, F32, 0.75), (512, 512)),
    ((0, 4097, 520, 31, F32, F32, 0.5), (512, 64)),
    ((0, 6100, 72, 7, BF16, BF16, 0.0), (1024, 32)),
    ((0, 40, 6104, 16, F32, F32, 0.5), (32, 1024)),
    ((0, 3080, 3084, 128, F16, F16, 0.5), (1024, 1024)),
    ((0, 2056, 2052, 60, F32, F32, 0.5), (256, 256)),
    ((33_000, 3080, 1032, 16, BF16, F32, 0.5), (1024, 512)),
]


def sizes(case):
    more, din, dout, r, t, to, p = case
    return sum(RUNS) + MISSING + more, din, dout, r, len(RUNS) + (more > 0)


def whole(shape, seed, most, dtype):
    return torch.randint(-most, most + 1, shape, generator=torch.Generator().manual_seed(seed), dtype=torch.int8).to(dev()).to(dtype)


@pytest.mark.parametrize("case,lengths", PIECES)
def test_sums_over_pieces_of_several_stages(qb, case, lengths):
    """Bit for bit: values are small whole numbers, scales and the mask's factor powers of two, and all sums of magnitudes below 2^24 (asserted), so that float32 sums
    of any order are exact and only the results' own rounding is left."""
    more, din, dout, r, t, to, p = case
    n, _, _, _, adapters = sizes(case)
    assert pieces(qb.vec_adapter_grad_workspace_bytes(n, din, dout, r, adapters, t), n, din, dout, r, adapters) == {lengths}
    ids = torch.cat([torch.full((k,), e) for e, k in enumerate(RUNS + [more] * (more > 0))] + [torch.full((MISSING,), -1)])
    ids = ids[torch.randperm(n, generator=torch.Generator().manual_seed(3))].to(dev())
    x, dy, kt, dx0 = whole((n, din), 1, 1, t), whole((n, dout), 2, 1, t), whole((n, r), 3, 9, F32), whole((n, din), 4, 9, t)
    a, b = whole((adapters, r, din), 5, 1, t), whole((adapters, r, dout), 6, 1, t)
    s = torch.exp2(torch.arange(adapters, device=dev()).float() % 3)
    call = dict(scales=s, p=p, state=state() if p else None, layer=LAYER)
    got = qb.vec_adapter_grad(dy, x, kt, a, b, ids, dx_base=dx0, dtype=to, **call)
    want = [ref for ref, _ in gradient64(dy, x, kt, a, b, ids, s, dx0, p)]
    (most, _), _, (most_b, _) = gradient64(*(v.abs() for v in (dy, x, kt, a, b)), ids, s, dx0.abs(), p)
    assert float(most.max()) < 1 << 24 and float(most_b.max()) < 1 << 24  # of u and dx; of db
    for e in range(adapters):  # of da, whose factor x is at most 1
        u = dy[ids == e].double() @ b[e].double().t() * float(s[e]) * (factor(p) if p else 1.0)
        assert float(u.abs().sum(0).max()) < 1 << 24
    for v, ref, ty in zip(got, want, (t, to, to)):
        assert torch.equal(v, ref.to(ty))
    for v, ref, ty in zip(qb.vec_adapter_grad(dy, x, kt, a, b, ids, dtype=to, want_dx=False, **call)[1:], want[1:], (to, to)):
        assert torch.equal(v, ref.to(ty))


# ---------------------------------------------------------------- high ranks --
@pytest.mark.parametrize("t,to", [(BF16, F32), (BF16, BF16), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("n,din,dout,r,adapters,kind,p", [
    (2500, 2056, 2048, 33, 3, "some", 0.1),      # tiles of 32 rows (64 of them and more), the mask's bits kept
    (2500, 2048, 2056, 64, 5, "skew", 0.25), (2500, 2056, 2048, 100, 1, "some", 0.1), (2500, 2048, 2056, 128, 3, "even", 0.1), (2500, 2056, 2048, 256, 2, "some", 0.5),
    (2500, 2050, 2047, 64, 4, "runs", 0.1), (2500, 2050, 2047, 200, 2, "some", 0.1),  # of odd widths, where they are not
    (2500, 2056, 2048, 64, 4, "alternate", 0.0), (2500, 2048, 2056, 256, 1, "one", 0.0),
    (700, 264, 136, 33, 3, "some", 0.5), (700, 264, 136, 64, 9, "even", 0.1), (700, 136, 264, 100, 4, "some", 0.1), (300, 72, 40, 256, 3, "skew", 0.1),  # tiles of 16
    (700, 8, 4, 65, 3, "some", 0.5)])
def test_gradients_of_high_ranks(qb, n, din, dout, r, adapters, kind, p, t, to):
    check_grad(qb, n, din, dout, r, adapters, kind, t, to, p)


@pytest.mark.parametrize("t,to", [(BF16, F32), (BF16, BF16), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("n,din,dout,r,adapters,kind,p", [
    (2500, 2056, 2048, 64, 3, "some", 0.1), (2500, 2048, 2056, 65, 5, "skew", 0.0), (2500, 2056, 2048, 128, 1, "some", 0.1), (2500, 2048, 2056, 128, 3, "alternate", 0.0),
    (2500, 2056, 2048, 256, 2, "even", 0.1), (2500, 2050, 2047, 256, 1, "some", 0.0), (2500, 4100, 5, 256, 3, "some", 0.0), (2500, 5, 4100, 256, 3, "some", 0.5),
    (2500, 2047, 2050, 177, 4, "runs", 0.0)])
def test_tiles_of_high_ranks(qb, n, din, dout, r, adapters, kind, p, t, to):
    check(qb, n, din, dout, r, adapters, kind, t, to, p)


@pytest.mark.parametrize("t", WIDE)
@pytest.mark.parametrize("r", [40, 64, 130, 256])
def test_the_kept_mask_is_that_of_the_rows(qb, r, t):
    """dx of ranks above 32 with the bits that the sums leave: what is dropped is dx_base itself, and the rest the gradient without dropout (p = 1/2, whose factor is exact)."""
    n, din, dout = 2500, 2056, 2048
    x, dy, kt, dx0 = rnd((n, din), 1, t), rnd((n, dout), 2, t), rnd((n, r), 3), rnd((n, din), 4, t)
    a, b, s = weights(3, r, din, dout, t)
    ids = torch.randint(-1, 3, (n,), generator=torch.Generator().manual_seed(5)).to(dev())
    m = qb.vec_dropout(torch.ones_like(x), 0.5, state(), LAYER) != 0
    dx, da, _ = qb.vec_adapter_grad(dy, x, kt, a, b, ids, scales=s, dx_base=dx0, p=0.5, state=state(), layer=LAYER)
    dx2, da2, _ = qb.vec_adapter_grad(dy, torch.where(m, x, 0.0), kt, a, b, ids, scales=s * 2, dx_base=dx0)
    assert torch.equal(dx[~m], dx0[~m]) and torch.equal(dx[m], dx2[m]) and torch.equal(da, da2)


# ------------------------------------------------------------ beyond 32 bits --
def test_gradients_beyond_32_bits(qb):
    """Elements past 2^32 of x, dx and dy, with dropout.  All values are small whole numbers, and p is 1/2 with the factor 2, so that every product and every sum of them is
    one below 2^24 (asserted), which float32 holds: whatever their order, da and db are exact, and dx but for its own rounding."""
    n, din, dout, r, adapters, p = 530_000, 8200, 8104, 4, 3, 0.5
    assert n * din > 1 << 32 and n * dout > 1 << 32
    g = torch.Generator(device=dev()).manual_seed(8)
    whole = lambda lo, *shape: torch.randint(lo, 2, shape, generator=g, device=dev())  # noqa: E731
    x, dy, step = torch.empty((n, din), dtype=BF16, device=dev()), torch.empty((n, dout), dtype=BF16, device=dev()), 10_000
    for i in range(0, n, step):
        x[i:i + step] = (2 * whole(0, step, din) - 1).to(BF16)  # (no zeros, so that what is dropped can be told)
        dy[i:i + step] = whole(-1, step, dout).to(BF16)
    a, b, kt, ids = whole(-1, adapters, r, din).to(BF16), whole(-1, adapters, r, dout).to(BF16), whole(-1, n, r).float(), whole(-1, n) + whole(0, n)
    call = dict(p=p, state=state(STEP), layer=LAYER)
    dx, da, db = qb.vec_adapter_grad(dy, x, kt, a, b, ids, **call)
    dropped = qb.vec_dropout(x, p, state(STEP), LAYER)
    del x
    own = torch.nn.functional.one_hot(ids + 1, adapters + 1)[:, 1:].double().repeat_interleave(r, dim=1)
    a64, b64 = a.double().view(adapters * r, din), b.double().view(adapters * r, dout)
    zero = lambda d: torch.zeros((adapters * r, d), dtype=torch.float64, device=dev())  # noqa: E731
    da64, sa, db64, sb = zero(din), zero(din), zero(dout), zero(dout)
    rows = [0, 1, 262_144, 523_775, 523_776, 523_777, 529_950, 529_951, n - 1]
    for i in range(0, n, step):
        d, v = dy[i:i + step].double(), dropped[i:i + step].double() / 2
        u, t = (d @ b64.t()) * 2 * own[i:i + step], kt[i:i + step].double().repeat(1, adapters) * own[i:i + step]
        assert float((d.abs() @ b64.abs().t()).max()) * 2 < 1 << 24
        da64 += u.t() @ v
        sa += u.abs().t() @ v.abs()
        db64 += t.t() @ d
        sb += t.abs().t() @ d.abs()
        for k in rows:
            if i <= k < i + step:
                assert torch.equal(dx[k], torch.where(v[k - i] != 0, u[k - i] @ a64, 0.0).to(BF16)), k
    assert float(sa.max()) < 1 << 24 and float(sb.max()) < 1 << 24
    assert torch.equal(da.double().view(da64.shape), da64) and torch.equal(db.double().view(db64.shape), db64)
