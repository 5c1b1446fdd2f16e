"""CPU-side checks of the operators on vectors: every declared function is exported, and bad arguments come back as an error
code with a message before anything is launched (the pointers here are never followed)."""
import os
import re

import pytest
import torch

from paper_1812_09162_amd import binding as qb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, F16, E4M3, E5M2, E8M0 = range(6)
P = 0x1000  # an aligned address


def test_library_exports_every_declared_symbol():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "qadc_vec.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(vec_[a-z_]+)\s*\(", text))
    assert names == set(qb.VEC_EXPORTS)
    for n in names:
        assert hasattr(qb.load(), n), n


def refused(rc, text, code=qb.PQ_EINVAL):
    msg = qb.load().pq_last_error().decode()
    assert rc == code and text in msg, (rc, msg)


def lookup(table=P, rows=10, d=8, ld=8, t=F32, ids=P, idb=4, n=5, scale=1.0, out=P, ldo=8, to=F32):
    return qb.load().vec_lookup(table, rows, d, ld, t, ids, idb, n, scale, out, ldo, to, None)


@pytest.mark.parametrize("kw,text", [
    (dict(n=-1), "n=-1"), (dict(rows=-1), "rows=-1"), (dict(d=0), "d=0"), (dict(t=E4M3), "types"), (dict(to=E8M0), "types"), (dict(t=9), "types"),
    (dict(idb=2), "ids of 2 bytes"), (dict(ld=7), "hold no"), (dict(ldo=7), "hold no"), (dict(table=None), "null"), (dict(ids=None), "null"),
    (dict(out=None), "null"), (dict(out=P + 2), "misaligned"), (dict(t=BF16, table=P + 1), "misaligned"), (dict(ids=P + 4, idb=8), "misaligned"),
    (dict(n=1 << 60), "too large")])
def test_lookup_refuses(kw, text):
    refused(lookup(**kw), text)


def test_lookup_of_nothing():
    assert lookup(n=0, table=None, ids=None, out=None) == qb.PQ_OK


def grad(g=P, n=5000, d=8, ld=8, t=F32, ids=P, idb=4, scale=1.0, acc=0, out=P, rows=10, ldo=8, to=F32, ws=P, wb=1 << 40):
    return qb.load().vec_lookup_grad(g, n, d, ld, t, ids, idb, scale, acc, out, rows, ldo, to, ws, wb, None)


@pytest.mark.parametrize("kw,text", [
    (dict(n=-1), "n=-1"), (dict(rows=1 << 31), "rows="), (dict(n=1 << 31), "n="), (dict(d=0), "d=0"), (dict(t=E5M2), "types"), (dict(to=E4M3), "types"),
    (dict(idb=1), "ids of"), (dict(ld=7), "hold no"), (dict(ldo=7), "hold no"), (dict(g=None), "null"), (dict(ids=None), "null"), (dict(out=None), "null"),
    (dict(out=P + 1), "misaligned"), (dict(ws=None), "workspace"), (dict(ws=P + 16), "workspace")])
def test_lookup_grad_refuses(kw, text):
    refused(grad(**kw), text)


def test_lookup_grad_workspace():
    lib = qb.load()
    need = lib.vec_lookup_grad_workspace_bytes(5000, 10, 8)
    assert need > 0
    refused(grad(wb=need - 1), str(need), qb.PQ_ENOMEM)
    assert grad(rows=0, out=None) == qb.PQ_OK and grad(n=0, acc=1, out=None) == qb.PQ_OK
    assert lib.vec_lookup_grad_workspace_bytes(0, 10, 8) == 0 == lib.vec_lookup_grad_workspace_bytes(-1, 10, 8)


def norm(x=P, ldx=256, r=P, ldr=256, t=BF16, w=P, tw=BF16, n=4, d=256, eps=1e-6, h=P, ldh=256, y=P, ldy=256, q=P, ldq=256, tq=E4M3, s=P, lds=2, ts=E8M0):
    return qb.load().vec_norm(x, ldx, r, ldr, t, w, tw, n, d, eps, h, ldh, y, ldy, q, ldq, tq, s, lds, ts, None)


@pytest.mark.parametrize("kw,text", [
    (dict(n=-1), "n=-1"), (dict(d=0), "d=0"), (dict(d=16385, ldx=20000), "d=16385"), (dict(eps=-1.0), "eps"), (dict(t=E4M3), "types"), (dict(tw=F16), "types"),
    (dict(r=None), "together"), (dict(h=None), "together"), (dict(q=None), "together"), (dict(s=None), "together"), (dict(y=None, q=None, s=None), "neither"),
    (dict(tq=BF16), "of type"), (dict(ts=BF16), "of type"), (dict(ldx=255), "distance"), (dict(ldh=255), "distance"), (dict(ldr=255), "distance"),
    (dict(ldy=255), "distance"), (dict(ldq=255), "distance"), (dict(lds=1), "distance"), (dict(x=None), "null"), (dict(w=None), "null"),
    (dict(y=P + 1), "misaligned"), (dict(s=P + 2, ts=F32), "misaligned")])
def test_norm_refuses(kw, text):
    refused(norm(**kw), text)


def norm_grad(dy=P, ldy=64, h=P, ldh=64, dh=P, lde=64, t=F16, w=P, tw=F32, n=4, d=64, eps=1e-6, dx=P, ldx=64, dw=P, ws=P, wb=1 << 40):
    return qb.load().vec_norm_grad(dy, ldy, h, ldh, dh, lde, t, w, tw, n, d, eps, dx, ldx, dw, ws, wb, None)


@pytest.mark.parametrize("kw,text", [
    (dict(n=-1), "n=-1"), (dict(d=0), "d=0"), (dict(d=16385), "d=16385"), (dict(eps=-1.0), "eps"), (dict(t=E5M2), "types"), (dict(tw=BF16), "types"),
    (dict(ldy=63), "distance"), (dict(ldh=63), "distance"), (dict(lde=63), "distance"), (dict(ldx=63), "distance"), (dict(dy=None), "null"),
    (dict(h=None), "null"), (dict(w=None), "null"), (dict(dx=None), "null"), (dict(dw=None), "null"), (dict(dw=P + 2), "misaligned"),
    (dict(ws=None), "workspace"), (dict(ws=P + 8), "workspace")])
def test_norm_grad_refuses(kw, text):
    refused(norm_grad(**kw), text)


def test_norm_grad_workspace():
    need = qb.load().vec_norm_grad_workspace_bytes(4, 64)
    assert need > 0
    refused(norm_grad(wb=need - 1), str(need), qb.PQ_ENOMEM)


def quantize(x=P, ldx=300, t=BF16, n=200, d=300, tr=0, q=P, ldq=300, tq=E4M3, s=P, lds=3, ts=E8M0):
    return qb.load().vec_quantize_blocks(x, ldx, t, n, d, tr, q, ldq, tq, s, lds, ts, None)


@pytest.mark.parametrize("kw,text", [
    (dict(n=-1), "n=-1"), (dict(d=-1), "d=-1"), (dict(tr=2), "transposed=2"), (dict(t=E4M3), "type"), (dict(tq=F16), "type"), (dict(ts=F16), "type"),
    (dict(ldx=299), "distance"), (dict(ldq=299), "distance"), (dict(lds=2), "distance"), (dict(tr=1, ldq=199), "distance"), (dict(tr=1, lds=1), "distance"),
    (dict(x=None), "null"), (dict(q=None), "null"), (dict(s=None), "null"), (dict(x=P + 1), "misaligned"), (dict(s=P + 1, ts=F32), "misaligned"),
    (dict(n=1 << 45), "too large"), (dict(n=1 << 36), "too large")])
def test_quantize_refuses(kw, text):
    refused(quantize(**kw), text)


def test_quantize_of_nothing():
    assert quantize(n=0, x=None, q=None) == qb.PQ_OK and quantize(d=0, x=None, q=None) == qb.PQ_OK


def matmul(a=P, lda=300, ta=E4M3, sa=P, ldas=3, b=P, ldb=300, tb=E5M2, sb=P, ldbs=3, ts=E8M0, m=100, n=200, k=300, c=P, ldc=200, tc=BF16, ws=P, wb=1 << 40):
    return qb.load().vec_matmul_blocks(a, lda, ta, sa, ldas, b, ldb, tb, sb, ldbs, ts, m, n, k, c, ldc, tc, ws, wb, None)


@pytest.mark.parametrize("kw,text", [
    (dict(m=-1), "m=-1"), (dict(n=-1), "n=-1"), (dict(k=-1), "k=-1"), (dict(m=1 << 31), "m="), (dict(ta=BF16), "types"), (dict(tb=F32), "types"),
    (dict(ts=BF16), "types"), (dict(tc=E4M3), "types"), (dict(lda=299), "distance"), (dict(ldb=299), "distance"), (dict(ldas=2), "distance"),
    (dict(ldbs=2), "distance"), (dict(ldc=199), "distance"), (dict(a=None), "null"), (dict(b=None), "null"), (dict(sa=None), "null"), (dict(sb=None), "null"),
    (dict(c=None), "null"), (dict(c=P + 1), "misaligned"), (dict(ts=F32, sa=P + 2), "misaligned")])
def test_matmul_refuses(kw, text):
    refused(matmul(**kw), text)


def test_matmul_workspace():
    lib = qb.load()
    m, n, k = 128, 128, 1 << 16
    need = lib.vec_matmul_blocks_workspace_bytes(m, n, k)
    assert need >= 2 * 4 * m * n
    call = dict(m=m, n=n, k=k, lda=k, ldb=k, ldas=k // 128, ldbs=k // 128, ldc=n)
    refused(matmul(wb=need - 1, **call), str(need), qb.PQ_ENOMEM)
    refused(matmul(ws=None, **call), "workspace")
    assert matmul(m=0, a=None, c=None) == qb.PQ_OK and matmul(n=0, b=None, c=None) == qb.PQ_OK
    assert lib.vec_matmul_blocks_workspace_bytes(0, 5, 5) == 0 == lib.vec_matmul_blocks_workspace_bytes(5, -5, 5)


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 128)
    for call in (lambda: qb.vec_lookup(x, torch.zeros(3, dtype=torch.int64)), lambda: qb.vec_lookup_grad(x, torch.zeros(4, dtype=torch.int64), 5),
                 lambda: qb.vec_norm(x, x[0]), lambda: qb.vec_norm_grad(x, x, x[0]), lambda: qb.vec_quantize_blocks(x),
                 lambda: qb.vec_matmul_blocks(x, x, x, x)):
        with pytest.raises(qb.QadcError) as e:
            call()
        assert e.value.code == qb.PQ_EINVAL and "GPU" in str(e.value)


def test_rows_of_too_many_columns_are_refused():
    """Counts of columns near 2^31 would overflow."""
    lib = qb.load()
    for d in ((1 << 24) + 1, (1 << 31) - 1):
        refused(lib.vec_lookup(P, 5, d, d, BF16, P, 8, 3, 1.0, P, d, BF16, None), f"d={d}")
        refused(lib.vec_lookup_grad(P, 3, d, d, BF16, P, 8, 1.0, 0, P, 5, d, BF16, P, 1 << 40, None), f"d={d}")


def test_products_of_more_tiles_than_a_launch_has_threads_are_refused():
    """2^24 tiles of 256 threads, 2^23 of 512: 2^32 threads."""
    n = (1 << 31) - 1
    refused(matmul(m=33, n=n, k=16, lda=16, ldb=16, ldas=1, ldbs=1, ldc=n), "too large")
    refused(matmul(m=33, n=n, k=16, lda=17, ldb=17, ldas=1, ldbs=1, ldc=n), "too large")
