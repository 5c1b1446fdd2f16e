"""CPU-side checks of dropout and the adapters: bad arguments come back as an error code with a message before anything is launched (the
pointers here are never followed)."""
import pytest
import torch

from paper_1812_09162_amd import binding as qb
from test_vec_host import BF16, E4M3, F16, F32, P, refused


def dropout(x=P, ldx=64, r=P, ldr=64, t=BF16, n=5, d=64, p=0.1, state=P, layer=0, y=P, ldy=64):
    return qb.load().vec_dropout(x, ldx, r, ldr, t, n, d, p, state, layer, y, ldy, None)


@pytest.mark.parametrize("kw,text", [
    (dict(n=-1), "n=-1"), (dict(n=1 << 32), "n="), (dict(d=0), "d=0"), (dict(d=(1 << 24) + 1, ldx=1 << 25, ldr=1 << 25, ldy=1 << 25), "d="), (dict(p=-0.1), "p="),
    (dict(p=1.0), "p="), (dict(p=0.999995), "p="), (dict(p=float("nan")), "p="), (dict(t=E4M3), "type"), (dict(ldx=63), "distance"), (dict(ldr=63), "distance"),
    (dict(ldy=63), "distance"), (dict(state=None), "state"), (dict(state=P + 4), "state"), (dict(x=None), "null"), (dict(y=None), "null"), (dict(x=P + 1), "misaligned"),
    (dict(r=P + 1), "misaligned"), (dict(y=P + 1), "misaligned"), (dict(n=(1 << 32) - 1, d=1 << 23, ldx=1 << 24, ldr=1 << 24, ldy=1 << 24), "too large")])
def test_dropout_refuses(kw, text):
    refused(dropout(**kw), text)


def test_dropout_of_nothing():
    assert dropout(n=0, x=None, y=None) == qb.PQ_OK and dropout(n=0, p=0.0, state=None, x=None, y=None) == qb.PQ_OK


def adapter(x=P, ldx=64, a=P, lda=64, sta=512, b=P, ldb=32, stb=256, t=BF16, count=3, rank=8, s=P, ids=P, idb=8, n=5, din=64, dout=32, base=P, ldbase=32, y=2 * P,
            ldy=32, ty=BF16, p=0.1, state=P, layer=0, kt=P, ws=P, wb=1 << 40):
    return qb.load().vec_adapter(x, ldx, a, lda, sta, b, ldb, stb, t, count, rank, s, ids, idb, n, din, dout, base, ldbase, y, ldy, ty, p, state, layer, kt, ws, wb, None)


def grad(dy=P, lddy=32, x=P, ldx=64, kt=P, a=P, lda=64, sta=512, b=P, ldb=32, stb=256, t=BF16, count=3, rank=8, s=P, ids=P, idb=8, n=5, din=64, dout=32, dx0=P, lddx0=64,
         dx=2 * P, lddx=64, p=0.1, state=P, layer=0, acc=0, da=P, ldda=64, stda=512, db=P, lddb=32, stdb=256, tg=F32, ws=P, wb=1 << 40):
    return qb.load().vec_adapter_grad(dy, lddy, x, ldx, kt, a, lda, sta, b, ldb, stb, t, count, rank, s, ids, idb, n, din, dout, dx0, lddx0, dx, lddx, p, state, layer, acc, da,
                                      ldda, stda, db, lddb, stdb, tg, ws, wb, None)


COMMON = [
    (dict(n=-1), "n=-1"), (dict(n=1 << 31), "n="), (dict(din=0), "din=0"), (dict(dout=0), "dout=0"), (dict(din=(1 << 20) + 1, ldx=1 << 21, lda=1 << 21), "din="),
    (dict(rank=0), "rank=0"), (dict(rank=257), "rank=257"), (dict(count=-1), "adapters=-1"), (dict(count=65536), "adapters=65536"), (dict(p=1.0), "p="), (dict(t=E4M3), "types"),
    (dict(idb=2), "ids of 2"), (dict(state=None), "state"), (dict(lda=63), "distance"), (dict(ldb=31), "distance"), (dict(sta=-1), "below 0"), (dict(stb=-512), "below 0"),
    (dict(ldx=63), "distance"), (dict(x=None), "null"), (dict(a=None), "null"), (dict(b=None), "null"), (dict(ids=None), "null"), (dict(x=P + 1), "misaligned"),
    (dict(a=P + 1), "misaligned"), (dict(b=P + 1), "misaligned"), (dict(s=P + 2), "misaligned"), (dict(ids=P + 4), "misaligned"), (dict(ws=None), "workspace"),
    (dict(ws=P + 16), "workspace")]


@pytest.mark.parametrize("kw,text", COMMON + [
    (dict(ty=F16), "types"), (dict(ldbase=31), "distance"), (dict(ldy=31), "distance"), (dict(base=P, y=P, ldy=40), "in place"), (dict(y=None), "null"), (dict(y=2 * P + 1), "misaligned"),
    (dict(base=P + 1), "misaligned"), (dict(kt=P + 2), "misaligned")])
def test_adapter_refuses(kw, text):
    refused(adapter(**kw), text)


@pytest.mark.parametrize("kw,text", COMMON + [
    (dict(tg=F16), "types"), (dict(dx=None), "dx_base without dx"), (dict(lddy=31), "distance"), (dict(lddx=63), "distance"), (dict(lddx0=63), "distance"), (dict(ldda=63), "distance"),
    (dict(lddb=31), "distance"), (dict(stda=511), "overlap"), (dict(stdb=255), "overlap"), (dict(dx0=P, dx=P, lddx=72), "in place"), (dict(dy=None), "null"), (dict(kt=None), "null"),
    (dict(da=None), "null"), (dict(db=None), "null"), (dict(dy=P + 1), "misaligned"), (dict(kt=P + 2), "misaligned"), (dict(dx=2 * P + 1), "misaligned"), (dict(dx0=P + 1), "misaligned"),
    (dict(da=P + 2), "misaligned"), (dict(db=P + 2), "misaligned")])
def test_adapter_grad_refuses(kw, text):
    refused(grad(**kw), text)


def test_workspaces():
    lib = qb.load()
    for size, call in ((lib.vec_adapter_workspace_bytes, adapter), (lib.vec_adapter_grad_workspace_bytes, grad)):
        need = size(5, 64, 32, 8, 3, BF16)
        assert need > 0
        refused(call(wb=need - 1), str(need), qb.PQ_ENOMEM)
        assert size(0, 64, 32, 8, 3, BF16) == 0 == size(5, 64, 32, 8, 0, BF16) == size(-1, 64, 32, 8, 3, BF16) == size(5, 64, 32, 999, 3, BF16)
    assert adapter(n=0, x=None, y=None, ids=None, ws=None) == qb.PQ_OK
    assert grad(n=0, count=0, dy=None, x=None, ids=None, da=None, db=None, ws=None) == qb.PQ_OK


def test_binding_refuses_host_tensors():
    x, w, ids = torch.zeros(4, 128), torch.zeros(2, 3, 128), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: qb.vec_dropout(x, 0.0), lambda: qb.vec_adapter(x, w, w, ids), lambda: qb.vec_adapter_grad(x, x, x[:, :3], w, w, ids)):
        with pytest.raises(qb.QadcError) as e:
            call()
        assert e.value.code == qb.PQ_EINVAL and "GPU" in str(e.value)


@pytest.mark.parametrize("kw", [dict(x=P, y=P, r=2 * P, ldy=72), dict(x=P, y=P, r=2 * P, ldx=72), dict(x=2 * P, y=P, r=P, ldy=72), dict(x=2 * P, y=P, r=P, ldr=72),
                                dict(x=P, y=P, r=None, ldy=72), dict(x=P, y=P, r=P, ldr=72)])
def test_dropout_in_place_with_other_distances(kw):
    """A row of y would lie over rows of x or of the residual that are still to be read."""
    refused(dropout(**kw), "in place")


@pytest.mark.parametrize("kw", [dict(), dict(n=1), dict(base=None), dict(ldy=64), dict(dout=64, ldb=64, stb=512, ldbase=64, ldy=64)])
def test_adapter_in_place_of_its_input(kw):
    """Single rows in one launch read x in several blocks, each of which writes a part of y."""
    refused(adapter(**dict(dict(x=2 * P, y=2 * P), **kw)), "in place of x")


def test_pieces_of_the_long_sums_are_those_that_their_tests_mean():
    from test_gpu_vec_adapter_long import PIECES, pieces, sizes
    for case, lengths in PIECES:
        assert pieces(qb.vec_adapter_grad_workspace_bytes(*sizes(case), case[4]), *sizes(case)) == {lengths}, case
    assert {k for _, lengths in PIECES for k in lengths} >= {32, 256, 512, 1024}
