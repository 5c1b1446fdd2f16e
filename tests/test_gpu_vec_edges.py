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
