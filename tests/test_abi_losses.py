"""Refusals of eat_ce_loss and eat_balance_loss: all on the host, before any
HIP call (fake addresses that nothing reads)."""
import os

import pytest

from paper_2609_33614_amd import _lib as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libeat.so not built")

F = 1 << 20           # an aligned address


def refused(status, fn, *args, **kw):
    with pytest.raises(L.EatError) as e:
        fn(*args, **kw)
    assert e.value.status == status, e.value


@pytest.mark.parametrize("T,d,V,grads,status", [
    (-1, 64, 10, 0, L.EAT_ERR_INVALID_ARG), (2 ** 20 + 1, 64, 10, 0, L.EAT_ERR_INVALID_ARG),
    (1, 0, 10, 0, L.EAT_ERR_INVALID_ARG), (1, 65, 10, 0, L.EAT_ERR_INVALID_ARG), (1, 32, 10, 0, L.EAT_ERR_INVALID_ARG),
    (1, 64, 0, 0, L.EAT_ERR_INVALID_ARG), (1, 64, 2 ** 24 + 1, 0, L.EAT_ERR_INVALID_ARG),
    (1, 64, 10, 4, L.EAT_ERR_INVALID_ARG), (1, 64, 10, -1, L.EAT_ERR_INVALID_ARG),
    (1, 65600, 10, 0, L.EAT_ERR_UNSUPPORTED)])
def test_ce_shapes(T, d, V, grads, status):
    refused(status, L.eat_ce_workspace_size, T, d, V, grads)


def test_ce_workspace_is_bounded():
    """At most 4 GiB of G at a time (4096 columns in the smallest), a pair of
    floats per position and 128 to 256 head rows, the counted rows' copies and
    fp32 slices of dh; never T V floats."""
    loss, least = L.eat_ce_workspace_size(8192, 4096, 128256, 0)
    assert loss == least < 2 ** 28
    both, least = L.eat_ce_workspace_size(8192, 4096, 128256, L.EAT_CE_DH | L.EAT_CE_DW)
    assert least < 2 ** 26 + 2 ** 29 and 8192 * 128256 * 2 < both < 8192 * 128256 * 2 + 2 ** 29
    T, d, V = 2 ** 20, 64, 2 ** 17
    most, least = L.eat_ce_workspace_size(T, d, V, L.EAT_CE_DW)
    rest = T * V // 32 + T * (2 * d + 64)
    assert most < max(2 ** 32, 8192 * T) + rest and least <= 8192 * T + rest
    assert min(L.eat_ce_workspace_size(0, 64, 10, 3)) > 0


@pytest.mark.parametrize("T,d,V", [(1, 64, 2 ** 24), (64, 64, 2 ** 24), (256, 65536, 2 ** 24), (2 ** 20, 65536, 2 ** 24),
                                   (300, 64, 2 ** 23), (1, 64, 1)])
def test_ce_workspace_at_the_limits(T, d, V):
    for grads in range(4):
        most, least = L.eat_ce_workspace_size(T, d, V, grads)
        assert 0 < least <= most < 2 ** 47


def test_ce_validation_happens_on_the_host():
    T, d, V = 100, 128, 1000
    n = L.eat_ce_workspace_size(T, d, V, 3)[1]

    W = 64 * F           # (every array at an address of its own)

    def go(h=F, T=T, d=d, w=4 * F, V=V, y=5 * F, ignore=-100, mean=1, scale=1.0, loss=6 * F, nll=7 * F, count=8 * F, dh=2 * F,
           dw=3 * F, ws=W, wsn=n):
        L.eat_ce_loss(h, T, d, w, V, y, ignore, mean, scale, loss, nll, count, dh, dw, ws, wsn, stream=0)

    bad = L.EAT_ERR_INVALID_ARG
    for kw in (dict(h=None), dict(w=None), dict(y=None), dict(loss=None), dict(mean=2), dict(mean=-1),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(T=-1), dict(d=96), dict(V=0),
               dict(h=F + 8), dict(w=F + 2), dict(y=F + 2), dict(loss=F + 1), dict(nll=F + 2), dict(count=F + 1),
               dict(dh=F + 8), dict(dw=F + 4), dict(ws=W + 128), dict(T=0, w=None),
               # overlaps (h: 25600 bytes at F, dh at 2 F, dw: 256000 at 3 F, w at 4 F)
               dict(dh=F + 16), dict(dh=F - 16), dict(dh=4 * F + 16), dict(dw=4 * F), dict(dw=4 * F - 16), dict(dw=F),
               dict(dh=3 * F + 255984), dict(loss=F), dict(loss=5 * F + 396), dict(nll=5 * F), dict(nll=4 * F), dict(count=6 * F),
               dict(nll=8 * F - 396), dict(loss=3 * F), dict(dh=5 * F), dict(dh=W + n - n % 16 - 16), dict(ws=F), dict(ws=3 * F),
               dict(ws=7 * F - 256), dict(h=W + 1024), dict(y=W)):
        refused(bad, go, **kw)
    refused(L.EAT_ERR_WORKSPACE, go, ws=None)
    refused(L.EAT_ERR_WORKSPACE, go, wsn=n - 1)
    refused(L.EAT_ERR_UNSUPPORTED, go, d=65600)


@pytest.fixture
def handle():
    h = L.eat_create(L.eat_params_default(mode="topk", E=60, d_model=128, d_ffn=64, top_k=4), 256)
    yield h
    L.eat_destroy(h)


def test_balance_validation_happens_on_the_host(handle):
    T = 100
    n = L.eat_balance_workspace_size(handle, T)
    bad = L.EAT_ERR_INVALID_ARG

    W = 64 * F

    def go(h=handle, x=F, T=T, w=2 * F, prob=3 * F, mask=7 * F, valid=8 * F, coef=0.01, ent=0.0, loss=9 * F, count=10 * F,
           mean=11 * F, dz=4 * F, dx=5 * F, dw=6 * F, ws=W, wsn=n):
        L.eat_balance_loss(h, x, T, w, prob, mask, valid, coef, ent, loss, count, mean, dz, dx, dw, ws, wsn, stream=0)

    for kw in (dict(h=None), dict(T=-1), dict(T=257), dict(prob=None), dict(mask=None), dict(loss=None),
               dict(coef=float("nan")), dict(ent=float("inf")), dict(x=None), dict(w=None), dict(x=F + 8),
               dict(w=F + 4), dict(prob=F + 2), dict(mask=F + 4), dict(loss=F + 2), dict(count=F + 4), dict(mean=F + 1),
               dict(dz=F + 2), dict(dx=F + 8), dict(dw=F + 8), dict(ws=W + 64),
               # overlaps (x and dx: 25600 bytes, w and dw: 30720, prob and dz: 24000)
               dict(dx=F), dict(dx=F + 16, dw=None), dict(dz=3 * F + 16), dict(dx=2 * F + 30704), dict(dw=2 * F), dict(dw=F),
               dict(dw=5 * F + 16), dict(dz=F), dict(dz=5 * F + 25596), dict(dz=2 * F), dict(dz=6 * F), dict(dz=7 * F + 796),
               dict(dz=8 * F + 96), dict(dx=3 * F), dict(dx=7 * F), dict(dx=8 * F), dict(dw=3 * F + 16), dict(loss=3 * F),
               dict(loss=10 * F), dict(count=11 * F + 232), dict(mean=8 * F), dict(ws=F), dict(ws=4 * F), dict(ws=11 * F),
               dict(prob=W), dict(valid=W + 5)):
        refused(bad, go, **kw)
    refused(L.EAT_ERR_WORKSPACE, go, ws=None)
    refused(L.EAT_ERR_WORKSPACE, go, wsn=n - 1)
    refused(bad, L.eat_balance_workspace_size, handle, 257)
    refused(bad, L.eat_balance_workspace_size, handle, -1)
    refused(bad, L.eat_balance_workspace_size, None, 1)
