"""Calls of sort, combine and the 8-bit products on a stream that the caller
names, while the current one has work pending: what a call allocates must be
memory that its own stream may use at once."""
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import Fp8Experts, Fp8Matrix, _Workspace
from tests import test_gpu_fp8 as Q
from tests import test_gpu_sort as S

pytestmark = pytest.mark.gpu


def cases():
    T, E, d, k = 700, 60, 128, 4
    b = S.make(T, E, d, True, k)
    lay = S.make_layer(E, d, True, T)

    def rows(stream=None):
        lay._bws.buf = None
        r, off, token, place = lay.sort(b["x"], b["mask"], cap=b["n"], stream=stream)
        # (what follows reads them: on the call's stream)
        y = lay.combine(r, b["mask"], b["gate"], place, stream=stream)
        return [r, off, token, place, y, lay.sort_backward(r, b["mask"], place, stream=stream)]

    w, x, off, token = Q.make_experts(T, d, 192, 8, 2)
    off, token = off.int().cuda(), token.int().cuda()
    m, ex = Fp8Matrix(w["w1"], gradients=True), Fp8Experts(w, gradients=True)
    saved = torch.empty(2 * T, 2 * 192, dtype=torch.bfloat16, device="cuda")

    def product(stream=None):
        m._ws = _Workspace(m.device)
        p = m.product(x, off, token, stream=stream)
        return [p, m.product_backward(p, off, stream=stream)]

    def experts(stream=None):
        ex._ws = _Workspace(ex.device)
        y = ex.forward(x, off, token, saved=saved, stream=stream)
        return [y, ex.backward(y, saved, off, stream=stream)]

    need = {"rows": L.eat_sort_workspace_size(lay.handle, T), "product": L.eat_fp8_product_workspace_size(T, 2 * T, 8, 192, d),
            "experts": L.eat_fp8_experts_workspace_size(ex.handle, T, 2 * T, 0)}
    return {"rows": rows, "product": product, "experts": experts}, need


@pytest.mark.parametrize("which", ["rows", "product", "experts"])
@pytest.mark.parametrize("how", ["stream", "address"])
def test_the_current_streams_pending_work_and_the_call_do_not_meet(which, how):
    runs, need = cases()
    run = runs[which]
    want = [t.clone() for t in run()]
    sizes = sorted({t.numel() * t.element_size() for t in want} | {need[which]})
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    # blocks of the sizes that the call allocates, given back while the current
    # stream has still to read and then to overwrite them
    blocks = [torch.full((n,), 5, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(8)]
    copies = [torch.empty_like(t) for t in blocks]
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    for t, c in zip(blocks, copies):
        c.copy_(t)
        t.fill_(0xFF)
    del blocks, t
    got = run(side if how == "stream" else side.cuda_stream)
    side.synchronize()
    first = [t.clone() for t in got]
    torch.cuda.synchronize()
    for a, b, r in zip(first, got, want):
        assert torch.equal(a, r) and torch.equal(b, r)
    assert all((c == 5).all() for c in copies)


@pytest.mark.parametrize("which", ["rows", "product", "experts"])
def test_what_a_call_returns_may_be_dropped_while_the_current_stream_reads_it(which):
    run = cases()[0][which]
    want = [t.clone() for t in run()]
    sizes = sorted({t.numel() * t.element_size() for t in want})
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = run(side)
    side.synchronize()
    torch.cuda._sleep(200_000_000)
    copy = [t.clone() for t in got]               # (pending)
    with torch.cuda.stream(side):
        del got
        fill = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(16)]
    torch.cuda.synchronize()
    assert all(torch.equal(c, r) for c, r in zip(copy, want)) and all((f == 0xFF).all() for f in fill)


def test_workspaces_are_not_given_away_while_another_stream_uses_them():
    """Calls on two streams in turn, the object's workspace growing between them."""
    w, x, off, token = Q.make_experts(300, 256, 192, 8, 2)
    w2, x2, off2, token2 = Q.make_experts(1500, 256, 192, 8, 2, seed=9)
    ex = Fp8Experts(w)
    a = (x, off.int().cuda(), token.int().cuda())
    b = (x2, off2.int().cuda(), token2.int().cuda())
    wa, wb = Fp8Experts(w).forward(*a), Fp8Experts(w).forward(*b)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
        got = ex.forward(*a)                          # (pending on the side stream)
    big = ex.forward(*b)                              # (a larger workspace: the first one is dropped)
    junk = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in (1 << 16, 1 << 18, 1 << 20, 1 << 21) for _ in range(16)]
    torch.cuda.synchronize()
    assert torch.equal(got, wa) and torch.equal(big, wb) and junk
