"""vec_dropout against its definition: the mask bit for bit, the values within their roundings."""
import math

import pytest
import torch

from philox import factor, kept
from test_gpu_vec import BF16, F16, F32, U, WIDE, close, dev, framed, half_step, rnd, untouched

pytestmark = pytest.mark.gpu
SEED, STEP = 0x1234_5678_9ABC_DEF, 77


@pytest.fixture(scope="module")
def qb():
    from paper_1812_09162_amd import binding
    binding.load()
    return binding


def state(seed=SEED, step=STEP):
    return torch.tensor([seed, step], device=dev())


def expected(x, r, p, layer, rows=None, seed=SEED, step=STEP):
    n, d = x.shape
    m = kept(range(n) if rows is None else rows, d, p, seed, step, layer).to(x.device)
    y = torch.where(m, x.double() * factor(p), 0.0)
    return m, y if r is None else y + r.double()


@pytest.mark.parametrize("p,layer", [(0.1, 0), (0.5, 3), (0.9, 0xFFFFFFFF)])
@pytest.mark.parametrize("t", WIDE)
@pytest.mark.parametrize("n,d", [(1, 1), (3, 7), (5, 8), (130, 9), (1, 257), (700, 96), (33, 1001), (1025, 256), (7, 8192), (3, 8200), (5, 20_001)])
def test_dropout(qb, n, d, t, p, layer):
    x, _ = framed(rnd((n, d), 1, t))
    r, _ = framed(rnd((n, d), 2, t))
    for res in (None, r):
        m, want = expected(x, res, p, layer)
        got = qb.vec_dropout(x, p, state(), layer, residual=res)
        close(got, want, half_step(want, t) + U * (want.abs() + 2 * x.double().abs() * factor(p)))
        if res is None:
            assert bool((got[~m] == 0).all()) and bool((got[m & (x != 0)] != 0).all())
        out, store = framed(torch.zeros((n, d), dtype=t, device=dev()))
        was = store.clone()
        qb.vec_dropout(x, p, state(), layer, residual=res, out=out)
        assert torch.equal(out, got) and untouched(out, store, was)


def test_rates(qb):
    x = torch.ones((64, 1000), device=dev())
    assert torch.equal(qb.vec_dropout(x, 0.0), x)
    assert torch.equal(qb.vec_dropout(x, 2.0 ** -18, state()), x)  # rounds to 0
    last = qb.vec_dropout(x, 65535 / 65536, state())
    m, want = expected(x, None, 65535 / 65536, 0)
    assert torch.equal(last.double(), want)


def test_in_place_and_its_gradient(qb):
    for t in WIDE:
        x, r = rnd((77, 515), 3, t), rnd((77, 515), 4, t)
        want = qb.vec_dropout(x, 0.3, state(), 9, residual=r)
        for at in (x.clone(), r.clone()):
            first = torch.equal(at, x)
            got = qb.vec_dropout(at if first else x, 0.3, state(), 9, residual=r if first else at, out=at)
            assert got is at and torch.equal(got, want)
        # sum of dy * y's derivative along v = sum of the call on dy times v
        dy, v = rnd((77, 515), 5, F32), rnd((77, 515), 6, F32)
        dx = qb.vec_dropout(dy, 0.3, state(), 9)
        y0, y1 = (qb.vec_dropout(u, 0.3, state(), 9) for u in (torch.zeros_like(v), v))
        a, b = (dy.double() * (y1 - y0).double()).sum(), (dx.double() * v.double()).sum()
        assert abs(float(a - b)) <= 4 * U * float((dy.double() * y1.double()).abs().sum())


def test_dropped_elements_are_zero_whatever_they_are(qb):
    for t in WIDE:
        x = rnd((40, 100), 7, t)
        m, _ = expected(x, None, 0.5, 1)
        x[~m] = torch.tensor([math.nan, math.inf, -math.inf], dtype=t, device=dev()).repeat(int((~m).sum()) // 3 + 1)[:int((~m).sum())]
        r = rnd((40, 100), 8, t)
        assert torch.equal(qb.vec_dropout(x, 0.5, state(), 1, residual=r)[~m], r[~m])
        x[m] = math.inf
        assert bool((qb.vec_dropout(x, 0.5, state(), 1)[m] == math.inf).all())


def test_masks_differ_by_seed_step_and_layer(qb):
    x = torch.ones((512, 512), device=dev())
    masks = [qb.vec_dropout(x, 0.5, s, layer) != 0 for s, layer in ((state(), 0), (state(), 1), (state(SEED + 1), 0), (state(SEED + (1 << 32)), 0), (state(step=STEP + 1), 0))]
    for i, a in enumerate(masks):
        for b in masks[:i]:
            assert abs(float((a == b).double().mean()) - 0.5) < 5 * 0.5 / 512
    assert torch.equal(masks[0], qb.vec_dropout(x, 0.5, state(step=STEP + (1 << 32)), 0) != 0)  # the step's low 32 bits
    assert torch.equal(masks[0], qb.vec_dropout(x, 0.5, state(), 0) != 0)


def test_beyond_32_bits(qb):
    n, d = 270_000, 16_384
    x = torch.ones((n, d), dtype=BF16, device=dev())
    y = qb.vec_dropout(x, 0.25, state(), 2, out=x)
    rows = [0, 1, 131_071, 131_072, 262_143, 262_144, 269_999]
    m = kept(rows, d, 0.25, SEED, STEP, 2).to(dev())
    want = torch.where(m, torch.tensor(factor(0.25), device=dev()).to(BF16), torch.zeros((), dtype=BF16, device=dev()))
    assert torch.equal(y[rows], want)


def test_replayed_with_another_step(qb):
    x, r = rnd((300, 640), 9, BF16), rnd((300, 640), 10, BF16)
    st, out = state(), torch.empty_like(x)
    qb.vec_dropout(x, 0.2, st, 4, residual=r, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qb.vec_dropout(x, 0.2, st, 4, residual=r, out=out)
        st[1] += 1
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, qb.vec_dropout(x, 0.2, state(step=STEP + i), 4, residual=r))


def test_another_stream(qb):
    x = rnd((500, 500), 11)
    want = qb.vec_dropout(x, 0.2, state())
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = qb.vec_dropout(x, 0.2, state(), stream=s)
    s.synchronize()
    assert torch.equal(got, want)


def test_refusals(qb):
    x = rnd((4, 8), 1)
    for kw in (dict(p=0.5), dict(p=0.5, state=state().int()), dict(p=0.5, state=state()[:1]), dict(p=0.5, state=state(), layer=-1), dict(p=0.5, state=state().cpu()),
               dict(p=0.5, state=state(), layer=1 << 32), dict(p=1.0, state=state()), dict(p=-0.1, state=state()), dict(p=math.nan, state=state()),
               dict(p=0.5, state=state(), residual=x[:3]), dict(p=0.5, state=state(), residual=x.half()), dict(p=0.5, state=state(), out=x.half())):
        with pytest.raises(qb.QadcError):
            qb.vec_dropout(x, **kw)
    assert qb.vec_dropout(x[:0], 0.5, state()).shape == (0, 8)
