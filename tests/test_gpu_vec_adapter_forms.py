"""The adapters at the sizes between which the calls change their form: single rows in one launch or two, rows as they come or sorted by one kernel or by the radix
sort, few rows an adapter, slabs of columns, short pieces of the sums over rows, matrices of few columns."""
import math

import pytest
import torch

from test_gpu_vec import BF16, F16, F32, U, close, dev, half_step, rnd
from test_gpu_vec_adapter import LAYER, STEP, TYPES, check, check_grad, forward64, make_ids, state, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qb():
    from paper_1812_09162_amd import binding
    binding.load()
    return binding


@pytest.mark.parametrize("t,to", TYPES)
@pytest.mark.parametrize("n,din,dout,r,adapters,kind", [
    (1, 4096, 4096, 16, 64, "one"), (1, 63, 8, 1, 2, "even"), (1, 4095, 511, 33, 2, "even"), (2, 65, 513, 64, 3, "some"), (8, 512, 1025, 16, 1, "some"), (8, 513, 7, 17, 1, "one"),
    (9, 512, 1025, 16, 1, "some"), (64, 257, 1, 5, 9, "outside"), (64, 2, 1000, 32, 64, "alternate"), (31, 1000, 3, 64, 70, "even"), (5, 3, 3, 3, 2, "even"), (64, 1, 9, 2, 3, "none"),
    (1, 20_000, 600, 8, 2, "one"), (33, 700, 72, 65, 5, "even")])
def test_single_rows(qb, n, din, dout, r, adapters, kind, t, to):
    check(qb, n, din, dout, r, adapters, kind, t, to)


def test_single_rows_that_are_not_finite(qb):
    """An infinity or NaN stays in its row, and what is not named is not read."""
    x, (a, b, s) = rnd((6, 300), 1, BF16), weights(4, 16, 300, 200, BF16)
    ids = torch.tensor([0, -1, 2, 1, 0, 9], device=dev())
    base = rnd((6, 200), 2, BF16)
    y, t = qb.vec_adapter(x, a, b, ids, scales=s, base=base, want_t=True)
    x[1], x[5], a[3], b[3], s[3] = math.nan, math.inf, math.nan, math.nan, math.nan
    x[2, 7] = math.inf
    y2, t2 = qb.vec_adapter(x, a, b, ids, scales=s, base=base, want_t=True)
    others = torch.tensor([0, 1, 3, 4, 5], device=dev())
    assert torch.equal(y[others], y2[others]) and torch.equal(t[others], t2[others]) and torch.equal(y[1], base[1])
    assert not bool(y2[2].isfinite().any())


@pytest.mark.parametrize("t,to", [(BF16, F32), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("n,din,dout,r,adapters,kind,p", [
    (65, 2048, 300, 16, 30, "even", 0.0),       # just sorted; slabs; few rows an adapter
    (129, 4096, 520, 8, 60, "skew", 0.1), (200, 1500, 9, 31, 90, "some", 0.0), (150, 40, 4097, 16, 70, "outside", 0.5), (100, 3000, 2, 20, 33, "even", 0.0),
    (2048, 520, 136, 15, 128, "even", 0.0),     # 16 rows an adapter, 15 and 16 ranks: on the vector units and on the matrix cores
    (2048, 520, 136, 16, 128, "even", 0.1), (1000, 100, 264, 128, 499, "even", 0.0), (600, 5, 6, 4, 40, "skew", 0.5),
    (66_000, 24, 40, 4, 100, "skew", 0.0),      # more rows, and more adapters, than one kernel groups
    (9000, 16, 24, 4, 4096, "even", 0.0), (9000, 16, 24, 4, 4095, "even", 0.0), (70_000, 8, 8, 2, 65_535, "runs", 0.0), (65_536, 16, 32, 3, 2, "alternate", 0.1),
    (16_500, 1030, 2050, 20, 1, "some", 0.1), (17_000, 264, 2056, 24, 5, "runs", 0.0)])
def test_sorted_rows(qb, n, din, dout, r, adapters, kind, p, t, to):
    check(qb, n, din, dout, r, adapters, kind, t, to, p)


@pytest.mark.parametrize("t,to", [(BF16, F32), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("n,din,dout,r,adapters,kind,p", [
    (65, 512, 300, 16, 5, "some", 0.0), (256, 130, 72, 64, 1, "some", 0.0), (257, 130, 72, 64, 1, "some", 0.0),         # one launch and two, of one adapter
    (2048, 40, 24, 7, 9, "outside", 0.0), (2049, 40, 24, 7, 9, "outside", 0.0), (1500, 3, 2, 60, 2, "alternate", 0.0),  # of several
    (1152, 1024, 512, 32, 20, "skew", 0.0), (1153, 1024, 512, 32, 20, "skew", 0.0), (13, 264, 1600, 20, 9, "some", 0.1), (21, 100, 3100, 16, 5, "outside", 0.0),  # 72 MB of A, more; rows by eight
    (640, 1024, 512, 32, 20, "skew", 0.0), (641, 1024, 1026, 32, 20, "skew", 0.0),                                      # 40 and 80 MB
    (256, 300, 200, 20, 8, "even", 0.1), (257, 300, 200, 20, 8, "even", 0.1), (256, 1200, 9, 100, 8, "skew", 0.0), (256, 24, 2050, 200, 3, "some", 0.5),  # unsorted, sorted
    (4100, 2050, 2049, 8, 3, "skew", 0.0), (2100, 4100, 40, 33, 20, "even", 0.1)])                                     # few large tiles
def test_between_forms(qb, n, din, dout, r, adapters, kind, p, t, to):
    check(qb, n, din, dout, r, adapters, kind, t, to, p)


@pytest.mark.parametrize("t,to", [(BF16, F32), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("n,din,dout,r,adapters,kind,p", [
    (4100, 2050, 2049, 8, 3, "skew", 0.1), (700, 40, 2049, 16, 100, "even", 0.0), (700, 40, 2048, 16, 100, "even", 0.0),
    (79, 84, 3201, 4, 38, "even", 0.1), (40, 2000, 1500, 16, 200, "even", 0.0), (64, 3, 700, 9, 5, "skew", 0.5), (100, 600, 2, 33, 50, "some", 0.0), (33, 2, 3, 70, 8, "even", 0.5),
    (2100, 264, 136, 16, 130, "even", 0.1), (66_000, 24, 40, 4, 100, "skew", 0.1), (9000, 16, 24, 4, 4096, "even", 0.0), (70_000, 8, 8, 2, 65_535, "runs", 0.0),
    (4096, 1030, 514, 17, 2, "alternate", 0.1), (1025, 72, 40, 64, 600, "skew", 0.25)])
def test_gradients_of_sorted_rows(qb, n, din, dout, r, adapters, kind, p, t, to):
    check_grad(qb, n, din, dout, r, adapters, kind, t, to, p)


def test_one_run_over_many_pieces(qb):
    """Sums that begin and end inside pieces, at their borders, and fill them."""
    din, dout, r, adapters = 40, 24, 5, 6
    for lengths in ([32, 32, 64, 1, 31, 96], [1, 127, 128, 1, 0, 255], [1000, 24, 1024, 0, 1, 2047], [33, 31, 65, 63, 0, 7]):
        ids = torch.cat([torch.full((k,), e) for e, k in enumerate(lengths)] + [torch.full((5,), -1)]).to(dev())
        n = ids.numel()
        x, dy, t = rnd((n, din), 1), rnd((n, dout), 2), rnd((n, r), 3)
        a, b, s = weights(adapters, r, din, dout, F32)
        _, da, db = qb.vec_adapter_grad(dy, x, t, a, b, ids, scales=s)
        for e in range(adapters):
            at = (ids == e).nonzero()[:, 0]
            u = dy[at].double() @ b[e].double().t() * float(s[e])
            for got, f, v, more in ((da[e], u, x[at], dout), (db[e], t[at].double(), dy[at], 0)):
                ref = f.t() @ v.double()
                size = (dy[at].double().abs() @ b[e].double().abs().t() * float(s[e])).t() if more else f.abs().t()
                close(got, ref, (size @ v.double().abs()) * U * (len(at) + more + 16) + half_step(ref, F32))


def test_a_large_call_in_a_graph(qb):
    """Tiles of 64 rows, whose kernels take more LDS than a launch has by itself."""
    n, din, dout, r, adapters = 20_000, 1024, 520, 16, 3
    x, (a, b, s), ids = rnd((n, din), 1, BF16), weights(adapters, r, din, dout, BF16), make_ids(n, adapters, "runs")
    base = rnd((n, dout), 2, BF16)
    y = torch.empty_like(base)
    ws = torch.empty(qb.vec_adapter_workspace_bytes(n, din, dout, r, adapters, BF16), dtype=torch.uint8, device=dev())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qb.vec_adapter(x, a, b, ids, scales=s, base=base, out=(y, None), workspace=ws)
    for i in range(3):
        x.mul_(-0.5)
        y.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, qb.vec_adapter(x, a, b, ids, scales=s, base=base)[0])


def test_two_calls_on_two_streams(qb):
    """Each with a workspace of its own, beside each other."""
    n, din, dout, r, adapters = 5000, 512, 264, 16, 40
    x, (a, b, s), ids = rnd((n, din), 1, F16), weights(adapters, r, din, dout, F16), make_ids(n, adapters, "skew")
    dy, base = rnd((n, dout), 2, F16), rnd((n, dout), 3, F16)
    y, t = qb.vec_adapter(x, a, b, ids, scales=s, base=base, want_t=True)
    grads = qb.vec_adapter_grad(dy, x, t, a, b, ids, scales=s)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(4):
        got.append((qb.vec_adapter(x, a, b, ids, scales=s, base=base, want_t=True, stream=streams[0]), qb.vec_adapter_grad(dy, x, t, a, b, ids, scales=s, stream=streams[1])))
    torch.cuda.synchronize()
    for (y2, t2), g2 in got:
        assert torch.equal(y, y2) and torch.equal(t, t2) and all(torch.equal(u, v) for u, v in zip(grads, g2))


def test_masks_are_those_of_the_rows_own_numbers(qb):
    """Sorted or not, in the forward pass and in both gradients: rows keep the mask of their place in x (p = 1/2, whose factor is exact; one adapter for all, given in two halves)."""
    n, din, dout, r = 900, 200, 136, 8
    x, dy, t = rnd((n, din), 1), rnd((n, dout), 2), rnd((n, r), 3)
    a, b, _ = weights(1, r, din, dout, F32)
    a, b = a.expand(2, r, din), b.expand(2, r, dout)
    ids = torch.arange(n, device=dev()) % 2
    call = dict(p=0.5, state=state(), layer=LAYER)
    dropped = qb.vec_dropout(x, 0.5, state(), LAYER)
    y64, ty, _, _ = forward64(dropped, a, b, ids, None, None, 0.0)
    y, _ = qb.vec_adapter(x, a, b, ids, **call)
    close(y, y64, ty + half_step(y64, F32))
    dx, da, _ = qb.vec_adapter_grad(dy, x, t, a, b, ids, **call)
    dx2, da2, _ = qb.vec_adapter_grad(dy, dropped, t, a, b, ids)
    assert torch.equal(dx, qb.vec_dropout(dx2, 0.5, state(), LAYER)) and torch.equal(da, da2)
