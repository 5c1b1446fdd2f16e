"""The operators on vectors where definitions are easily missed: sums whose large terms cancel, quotients of tiny scales, numbers that are
not finite, zeros, many ids, long launches.  Every expected value is exact or from 64 bits."""
import math

import pytest
import torch

from test_gpu_vec import BF16, E4M3, E5M2, E8M0, F16, F32, U, close, dev, framed, half_step, product64, qb, quantized, rnd, same_values, untouched  # noqa: F401

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- products --
@pytest.mark.parametrize("st", [E8M0, F32])
@pytest.mark.parametrize("ta,tb", [(E4M3, E4M3), (E4M3, E5M2), (E5M2, E4M3), (E5M2, E5M2)])
@pytest.mark.parametrize("m,n,k,aligned", [(5, 70, 512, True), (70, 90, 384, True), (70, 90, 512, True), (129, 257, 520, False), (300, 130, 640, True), (600, 1500, 1160, True),
                                           (3600, 3700, 640, True)])
def test_sums_whose_large_terms_cancel(qb, m, n, k, aligned, ta, tb, st):
    """Products of 2^16 that cancel beside products of one: every partial sum is a whole number below 2^24, so float32 sums of exact products
    are exact in any order, and so is the result in bfloat16 (the ones are eight)."""
    half = k // 2
    row = torch.where(torch.arange(half) % 4 == 1, 256.0, 1.0)  # two large ones in each eight
    a = torch.cat([row, row]).expand(m, k)
    b = torch.cat([row, -row]).expand(n, k).clone()
    b[:, torch.arange(8) * 8 + 2] = 2.0  # (one in a, one in b until now)
    a, b = a.to(ta).to(dev()), b.to(tb).to(dev())
    nb = -(-k // 128)
    sa, sb = torch.ones((m, nb), device=dev()).to(st), torch.ones((n, nb), device=dev()).to(st)
    want, size = product64(a, sa, b, sb)
    assert bool((want == 8).all()) and float(size.max()) < 2 ** 25  # (half of it has one sign)
    if not aligned:
        a, _ = framed(a, 3, 4)
    for to in (BF16, F32):
        got = qb.vec_matmul_blocks(a, sa, b, sb, dtype=to)
        assert bool((got == 8).all()), (to, float(got.min()), float(got.max()))


@pytest.mark.parametrize("rows", [5, 70, 600])
@pytest.mark.parametrize("k", [200, 640])
def test_products_of_the_smallest_power(qb, rows, k):
    """A scale byte of 0 is 2^-127 (what the quantizer gives to tiny blocks)."""
    n, nb = 1500, -(-k // 128)
    a, b = torch.full((rows, k), 256.0, device=dev()).to(E4M3), torch.full((n, k), 1.5, device=dev()).to(E4M3)
    sa, sb = torch.zeros((rows, nb), dtype=torch.uint8, device=dev()).view(E8M0), torch.full((n, nb), 2.0 ** 119, device=dev()).to(E8M0)
    want = k * 1.5
    for x, sx, y, sy in ((a, sa, b, sb), (b[:rows], sb[:rows], a[:1].expand(n, k).contiguous(), sa[:1].expand(n, nb).contiguous())):
        for to in (F32, BF16):
            assert bool((qb.vec_matmul_blocks(x, sx, y, sy, dtype=to) == torch.tensor(want).to(to).to(dev())).all())


@pytest.mark.parametrize("st", [E8M0, F32])
@pytest.mark.parametrize("rows", [5, 70, 600])
@pytest.mark.parametrize("k", [200, 640])
def test_products_of_infinities_and_nan(qb, rows, k, st):
    """Infinities of E5M2 meet positive, negative and zero factors; a NaN scale meets zeros."""
    n, nb = 1500, -(-k // 128)
    a, b = torch.ones((rows, k)), torch.ones((n, k))
    sa, sb = torch.ones((rows, nb), device=dev()).to(st), torch.ones((n, nb), device=dev()).to(st)
    a[2, 150], a[4, 7], a[4, k - 1] = math.inf, math.inf, -math.inf
    a[1, :] = 0.0
    b[11, 150], b[12, 150] = -1.0, 0.0
    a, b = a.to(E5M2).to(dev()), b.to(E4M3).to(dev())
    want = torch.full((rows, n), float(k), device=dev())
    want[1] = 0
    want[:, 11], want[:, 12] = want[:, 11] - 2 * (want[:, 11] != 0), want[:, 12] - 1.0 * (want[:, 12] != 0)
    want[2], want[4] = math.inf, math.nan
    want[2, 11], want[2, 12] = -math.inf, math.nan
    if st == E8M0:
        sb.view(torch.uint8)[20, 1] = 255
    else:
        sb[20, 1] = math.nan
    want[:, 20] = math.nan
    for to in (F32, F16, BF16):
        got = qb.vec_matmul_blocks(a, sa, b, sb, dtype=to)
        assert same_values(got, want.to(to)), to


# --------------------------------------------------------------- quantizer --
def test_quotients_of_tiny_scales(qb):
    """Quotients next to a tie of the 8-bit type, with scales so small that a remainder's last bits lie below the smallest float32."""
    hexes = {E4M3: [("0x1.bffff8p-93", "0x1.fffff8p-112"), ("0x1.bffffap-91", "0x1.fffffcp-110"), ("0x1.bffff4p-89", "0x1.fffff4p-108"),
                    ("0x1.bffffap-87", "0x1.fffffcp-106"), ("0x1.c00004p-87", "0x1.800002p-104")],
             E5M2: [("0x1.bfd04p-84", "0x1.ffc97p-117"), ("0x1.c0154p-85", "0x1.400f2ep-115"), ("0x1.bffffap-83", "0x1.fffffcp-116"),
                    ("0x1.bffff6p-80", "0x1.fffff4p-113"), ("0x1.c00008p-79", "0x1.c00006p-109"), ("0x1.bffffep-76", "0x1p-108"),
                    ("0x1.bffffap-73", "0x1.fffffcp-106"), ("0x1.c00004p-73", "0x1.800002p-104")]}
    for qt, pairs in hexes.items():
        x = torch.zeros((len(pairs), 128))
        for i, (top, f) in enumerate(pairs):
            x[i, 0], x[i, 1], x[i, 2] = float.fromhex(top), float.fromhex(f), -float.fromhex(f)
        want, ws = quantized(x, qt, F32)
        for transposed in (False, True):
            q, s = qb.vec_quantize_blocks((x.t().contiguous() if transposed else x).to(dev()), dtype=qt, scale_dtype=F32, transposed=transposed)
            assert torch.equal(s.cpu().double(), ws) and same_values(q, want), qt


@pytest.mark.parametrize("qt", [E4M3, E5M2])
def test_quotients_next_to_ties(qb, qt):
    """Scales of every power from 2^-126 to 2^-60, values within three steps of a tie."""
    g = torch.Generator().manual_seed(7)
    n, least = 67 * 40, 2.0 ** (-10 if qt == E4M3 else -17)
    power = torch.arange(-126, -59).repeat_interleave(40).double()
    scale = ((1 + torch.randint(0, 1 << 23, (n,), generator=g).double() * 2 ** -23) * torch.exp2(power)).float()
    scale[::4] = (torch.exp2(power[::4]) * (2 - torch.randint(1, 8, (len(power[::4]),), generator=g).double() * 2 ** -23)).float()
    ties = (2 * torch.randint(0, 6, (n, 127), generator=g) + 1).double() * least
    f = (ties * scale[:, None].double()).float()
    f = (f.view(torch.int32) + torch.randint(-3, 4, (n, 127), generator=g, dtype=torch.int32)).clamp(min=0).view(torch.float32)
    x = torch.cat([(scale * (448.0 if qt == E4M3 else 57344.0))[:, None], f], 1)
    want, ws = quantized(x, qt, F32)
    q, s = qb.vec_quantize_blocks(x.to(dev()), dtype=qt, scale_dtype=F32)
    assert torch.equal(s.cpu().double(), ws) and same_values(q, want)


def test_more_blocks_of_rows_than_a_launch_has_in_a_row(qb):
    """2^28 + 100 rows of one value: more blocks of threads than one dimension of a launch takes."""
    n = (1 << 28) + 100
    x = torch.zeros((n, 1), dtype=BF16, device=dev())
    at = torch.tensor([0, 1, (1 << 27) + 5, (1 << 28) - 1, 1 << 28, n - 1], device=dev())
    vals = torch.tensor([1.0, -3.0, 5.0, 0.25, -7.0, 448.0], device=dev()).to(BF16)[:, None]
    x[at] = vals
    q, s = torch.full((n, 1), 9, dtype=torch.uint8, device=dev()), torch.full((n, 1), 9, dtype=torch.uint8, device=dev())
    qb.vec_quantize_blocks(x, out=(q.view(E4M3), s.view(E8M0)))
    want, ws = quantized(vals.cpu(), E4M3, E8M0)
    assert same_values(q[at].view(E4M3), want) and torch.equal(s[at].view(E8M0).cpu().double(), ws)
    assert int((q != 0).sum()) == len(at) and int((s != 127).sum()) == int((ws != 1).sum())


def test_more_blocks_of_columns_than_a_launch_has_in_a_row(qb):
    """2^31 + 200 rows of one value, in blocks along the column."""
    n = (1 << 31) + 200
    x = torch.zeros((n, 1), dtype=BF16, device=dev())
    at = torch.tensor([0, 300, (1 << 30) + 5, (1 << 31) - 1, 1 << 31, n - 1], device=dev())
    vals = torch.tensor([1.0, -3.0, 5.0, 0.25, -7.0, 448.0], device=dev()).to(BF16)[:, None]
    x[at] = vals
    q, s = torch.full((1, n), 9, dtype=torch.uint8, device=dev()), torch.full((1, -(-n // 128)), 9, dtype=torch.uint8, device=dev())
    qb.vec_quantize_blocks(x, transposed=True, out=(q.view(E4M3), s.view(E8M0)))
    want, ws = quantized(vals.cpu(), E4M3, E8M0)
    assert same_values(q[0, at, None].view(E4M3), want) and torch.equal(s[0, at // 128, None].view(E8M0).cpu().double(), ws)
    assert int((q != 0).sum()) == len(at) and int((s != 127).sum()) == int((ws != 1).sum())


def test_look_up_of_more_rows_than_a_launch_has_blocks(qb):
    """2^24 + 3 rows of 4097 values, a block of threads each."""
    n, d = (1 << 24) + 3, 4097
    table = rnd((5, d), 1, BF16)
    ids = torch.zeros(n, dtype=torch.int32, device=dev())
    at = torch.tensor([1, (1 << 23) + 1, (1 << 24) - 1, 1 << 24, n - 1], device=dev())
    ids[at] = torch.tensor([1, 2, 3, 4, -1], dtype=torch.int32, device=dev())
    out = torch.empty((n, d), dtype=BF16, device=dev())
    qb.vec_lookup(table, ids, out=out)
    assert torch.equal(out[at[:4]], table[1:]) and bool((out[n - 1] == 0).all())
    for i in (0, 2, 1 << 23, (1 << 24) - 2, (1 << 24) + 1):
        assert torch.equal(out[i], table[0])
    del out
    torch.cuda.empty_cache()


@pytest.mark.parametrize("st", [E8M0, F32])
def test_one_row_against_very_many(qb, st):
    """2^30 + 40 rows of sixteen bytes: more blocks of threads than one dimension of a launch takes."""
    n, k = (1 << 30) + 40, 16
    b = torch.zeros((n, k), dtype=torch.uint8, device=dev())
    sb = torch.full((n, 1), 127, dtype=torch.uint8, device=dev()).view(E8M0) if st == E8M0 else torch.ones((n, 1), device=dev())
    at = torch.tensor([0, 17, (1 << 29) + 1, (1 << 30) - 1, 1 << 30, n - 1], device=dev())
    vals = torch.randint(-8, 9, (6, k), generator=torch.Generator().manual_seed(1)).float().to(E4M3).to(dev())
    b[at] = vals.view(torch.uint8)
    a, sa = torch.ones((1, k), device=dev()).to(E4M3), torch.ones((1, 1), device=dev()).to(st)
    got = qb.vec_matmul_blocks(a, sa, b.view(E4M3), sb)
    assert torch.equal(got[0, at].float(), vals.float().sum(1)) and int((got != 0).sum()) == int((vals.float().sum(1) != 0).sum())


# ----------------------------------------------------------------- look-up --
@pytest.mark.parametrize("scale", [-2.0, math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("to", [F32, BF16, F16])
def test_rows_of_unknown_ids_are_zeros(qb, scale, to):
    """... whatever the scale, and zeros without a sign."""
    table = rnd((6, 37), 1, to)
    ids = torch.tensor([0, -1, 6, 5, -(2 ** 40), 2 ** 40], device=dev())
    got = qb.vec_lookup(table, ids, scale=scale)
    bits = got[[1, 2, 4, 5]].contiguous().view(torch.uint8)
    assert bool((bits == 0).all())
    assert same_values(got[[0, 3]], (table[[0, 5]].float() * scale).to(to))


def test_rows_of_2_to_the_32_columns_are_refused(qb):
    """Counts of columns are 32 bits behind the binding: 2^32 + 8 are not 8."""
    wide = torch.empty((1, (1 << 32) + 8), dtype=BF16, device=dev())
    ids = torch.zeros(1, dtype=torch.int64, device=dev())
    for call in (lambda: qb.vec_lookup(wide, ids, out=wide), lambda: qb.vec_lookup_grad(wide, ids, 1, out=wide),
                 lambda: qb.vec_norm(wide, wide[0], out=(wide, None, None, None)), lambda: qb.vec_norm_grad(wide, wide, wide[0])):
        with pytest.raises(qb.QadcError) as e:
            call()
        assert e.value.code == qb.PQ_EINVAL and str((1 << 32) + 8) in str(e.value)


# ---------------------------------------------------------- gradient by id --
def grad64(g, ids, rows, scale):
    """Sums by id, of magnitudes by id, and counts, in 64 bits, on the host."""
    g, ids = g.cpu(), ids.cpu()
    ok = ((ids >= 0) & (ids < rows)).nonzero()[:, 0]
    at, v = ids[ok].long(), g[ok].double() * float(torch.tensor(scale, dtype=F32))
    sums = [torch.zeros((rows, x.shape[1]), dtype=torch.float64).index_add_(0, at, x) for x in (v, v.abs(), torch.ones((len(ok), 1), dtype=torch.float64))]
    return [x.to(dev()) for x in sums]


def check_grad(qb, g, ids, rows, to, scale=0.77):
    want, size, count = grad64(g, ids, rows, scale)
    got = qb.vec_lookup_grad(g, ids, rows, scale=scale, dtype=to)
    close(got, want, U * (count + 1) * size * 1.001 + half_step(want, to))
    assert bool((got[count[:, 0] == 0] == 0).all())
    assert torch.equal(got, qb.vec_lookup_grad(g, ids, rows, scale=scale, dtype=to))
    base, store = framed(rnd((rows, g.shape[1]), 6, to))
    was, old = store.clone(), base.clone()
    qb.vec_lookup_grad(g, ids, rows, scale=scale, out=base, accumulate=True)
    ref = old.double() + want
    close(base, ref, U * ((count + 2) * size + old.double().abs()) * 1.001 + half_step(ref, to))
    assert torch.equal(base[count[:, 0] == 0], old[count[:, 0] == 0]) and untouched(base, store, was)


@pytest.mark.parametrize("t,to", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("rows,d,n,kind", [(100_003, 24, 262_144, "skew"), (5000, 130, 200_001, "skew"), (700, 9, 131_073, "one"), (40, 300, 140_000, "even"),
                                           (3, 16, 500_003, "even"), (1_100_000, 5, 300_000, "outside"), (70_000, 8, 1_200_007, "skew"), (900, 4, 2_100_001, "one"),
                                           (600_000, 3, 1_048_577, "even"), (3, 2, 700_003, "even")])
def test_gradient_of_many_ids(qb, rows, d, n, kind, t, to):
    """Whole pieces of 64 positions, ids whose runs cross thousands of them, up to hundreds of tiles of the sort."""
    u = torch.rand((n,), generator=torch.Generator().manual_seed(rows), dtype=torch.float64)
    ids = {"even": (u * rows).long(), "skew": (rows ** u - 1).long().clamp(0, rows - 1), "one": torch.where(u < 0.9, rows // 2, (u * rows).long()),
           "outside": torch.where(u < 0.3, -1, ((u * 2 - 0.7) * 1.1 * rows).long())}[kind].to(dev())
    check_grad(qb, rnd((n, d), 5, t), ids if n % 2 else ids.int(), rows, to)


@pytest.mark.parametrize("n", [50, 3000, 9000, 140_000])
def test_gradient_of_rows_that_are_not_finite(qb, n):
    """Infinities and NaN stay with their ids; those of positions without a row of the table go nowhere."""
    rows, d = 200, 40
    ids = torch.randint(10, rows, (n,), generator=torch.Generator().manual_seed(n)).to(dev())
    g = rnd((n, d), 1)
    at = torch.tensor([1, 2, 5, 7, 11, 13, 17, 19], device=dev())
    ids[at] = torch.tensor([0, 1, 2, 2, -1, rows, 2 ** 33, 3], device=dev())
    g[at[0]] = math.inf
    g[at[1], 3] = math.nan
    g[at[2]], g[at[3]] = math.inf, -math.inf
    g[at[4]], g[at[5]], g[at[6]] = math.nan, math.inf, -math.inf
    g[at[7]] = -math.inf
    got = qb.vec_lookup_grad(g, ids, rows, scale=2.0)
    assert bool((got[0] == math.inf).all()) and bool(got[2].isnan().all()) and bool((got[3] == -math.inf).all())
    assert bool(got[1, 3].isnan()) and bool(got[1, :3].isfinite().all()) and bool(got[1, 4:].isfinite().all())
    assert bool((got[4:10] == 0).all()) and bool(got[10:].isfinite().all())


def test_time_of_the_gradient_grows_with_the_ids(qb):
    """32 times as many ids, into the same table: not more than 64 times the time (sums over all pairs of tiles would take 1024 times)."""
    def us(n):
        ids = torch.randint(0, 1 << 20, (n,), device=dev(), dtype=torch.int32, generator=torch.Generator(device=dev()).manual_seed(1))
        g = torch.ones((n, 1), dtype=BF16, device=dev())
        out = torch.empty((1 << 20, 1), dtype=F32, device=dev())
        w = torch.empty(qb.vec_lookup_grad_workspace_bytes(n, 1 << 20, 1), dtype=torch.uint8, device=dev())
        best = math.inf
        for _ in range(3):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            qb.vec_lookup_grad(g, ids, 1 << 20, out=out, workspace=w)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b) * 1000)
        assert torch.equal(out[:, 0], torch.bincount(ids, minlength=1 << 20).float())
        return best
    few, many = us(1 << 20), us(1 << 25)
    print(f"2^20 ids {few:.0f} us, 2^25 {many:.0f} us")
    assert many <= 64 * few, (few, many)
