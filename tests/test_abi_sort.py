"""Refusals of the sort and combine entry points: all on the host, before any
HIP call (fake addresses that nothing reads)."""
import os

import pytest

from paper_2609_33614_amd import _lib as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libeat.so not built")

F = 1 << 24           # an aligned address; the arrays below are smaller than the steps between them
T, CAP, E, D = 100, 400, 60, 128
BAD = L.EAT_ERR_INVALID_ARG
ROWS, X, PAIRS, MASK = CAP * D * 2, T * D * 2, T * E * 4, T * 8


def refused(status, fn, *args, **kw):
    with pytest.raises(L.EatError) as e:
        fn(*args, **kw)
    assert e.value.status == status, (kw, e.value)


@pytest.fixture
def handle():
    h = L.eat_create(L.eat_params_default(mode="topk", E=E, d_model=D, d_ffn=64, top_k=4), 40000)
    yield h
    L.eat_destroy(h)


def test_workspace_sizes(handle):
    assert L.eat_sort_workspace_size(handle, 0) == 0 and L.eat_sort_workspace_size(handle, 256) == 0
    n = L.eat_sort_workspace_size(handle, 40000)
    assert n >= (157 + 1) * E * 4 and n < 2 ** 20
    for t in (-1, 40001):
        refused(BAD, L.eat_sort_workspace_size, handle, t)
    refused(BAD, L.eat_sort_workspace_size, None, 1)


def test_sort(handle):
    def go(h=handle, x=F, T=T, mask=2 * F, cap=CAP, rows=3 * F, off=4 * F, tok=5 * F, place=6 * F, ws=None, wsn=0):
        L.eat_sort_tokens(h, x, T, mask, cap, rows, off, tok, place, ws, wsn, stream=0)

    for kw in (dict(h=None), dict(T=-1), dict(T=40001), dict(cap=-1), dict(mask=None), dict(place=None), dict(off=None),
               dict(tok=None), dict(x=None), dict(rows=None), dict(x=F + 8), dict(rows=3 * F + 8), dict(mask=2 * F + 4),
               dict(off=4 * F + 2), dict(tok=5 * F + 1), dict(place=6 * F + 2),
               dict(rows=F), dict(rows=F + X - 16), dict(rows=2 * F), dict(off=F), dict(off=2 * F + MASK - 4), dict(tok=4 * F),
               dict(tok=4 * F + E * 4), dict(place=3 * F + ROWS - 4), dict(place=5 * F), dict(place=2 * F), dict(tok=F)):
        refused(BAD, go, **kw)
    n = L.eat_sort_workspace_size(handle, 40000)
    big = dict(T=40000, x=None, rows=None, place=16 * F, mask=32 * F, tok=33 * F)
    refused(L.EAT_ERR_WORKSPACE, go, **big)
    refused(L.EAT_ERR_WORKSPACE, go, ws=40 * F, wsn=n - 1, **big)
    refused(BAD, go, ws=40 * F + 128, wsn=n, **big)
    refused(BAD, go, ws=16 * F, wsn=n, **big)
    refused(BAD, go, ws=32 * F, wsn=n, **big)


def test_sort_backward_and_combine(handle):
    def back(h=handle, src=F, cap=CAP, T=T, mask=2 * F, place=3 * F, out=5 * F):
        L.eat_sort_backward(h, src, cap, T, mask, place, out, stream=0)

    def comb(h=handle, src=F, cap=CAP, T=T, mask=2 * F, gate=4 * F, place=3 * F, out=5 * F):
        L.eat_combine(h, src, cap, T, mask, gate, place, out, stream=0)

    for go in (back, comb):
        for kw in (dict(h=None), dict(T=-1), dict(T=40001), dict(cap=-1), dict(src=None), dict(mask=None), dict(place=None),
                   dict(out=None), dict(src=F + 8), dict(mask=2 * F + 4), dict(place=3 * F + 1), dict(out=5 * F + 8),
                   dict(out=F), dict(out=F + ROWS - 16), dict(out=2 * F), dict(out=3 * F + PAIRS - 16)):
            refused(BAD, go, **kw)
    for kw in (dict(gate=None), dict(gate=4 * F + 2), dict(out=4 * F)):
        refused(BAD, comb, **kw)


def test_combine_backward(handle):
    def go(h=handle, dy=F, rows=2 * F, cap=CAP, T=T, mask=3 * F, gate=4 * F, place=5 * F, prob=6 * F, drows=7 * F, dg=8 * F, dz=9 * F):
        L.eat_combine_backward(h, dy, rows, cap, T, mask, gate, place, prob, drows, dg, dz, stream=0)

    for kw in (dict(h=None), dict(T=-1), dict(T=40001), dict(cap=-1), dict(dy=None), dict(rows=None), dict(mask=None),
               dict(gate=None), dict(place=None), dict(prob=None), dict(rows=None, dz=None), dict(dy=F + 8), dict(rows=2 * F + 8),
               dict(drows=7 * F + 8), dict(dg=8 * F + 2), dict(dz=9 * F + 2), dict(prob=6 * F + 2), dict(gate=4 * F + 1),
               dict(drows=2 * F + 16), dict(drows=F), dict(drows=4 * F), dict(dg=4 * F + 4), dict(dg=6 * F), dict(dg=9 * F),
               dict(dz=4 * F), dict(dz=6 * F + 4), dict(dz=3 * F), dict(dz=5 * F), dict(dg=7 * F + ROWS - 4), dict(dz=2 * F)):
        refused(BAD, go, **kw)


def test_calls_without_work_touch_nothing(handle):
    """No tokens (fake addresses again): nothing to enqueue but sort's offsets."""
    L.eat_sort_backward(handle, None, 0, 0, None, None, None, stream=0)
    L.eat_combine(handle, None, 0, 0, None, None, None, None, stream=0)
    L.eat_combine_backward(handle, None, None, 0, 0, None, None, None, None, None, None, None, stream=0)
    L.eat_combine_backward(handle, F, 2 * F, CAP, T, 3 * F, 4 * F, 5 * F, None, None, None, None, stream=0)
