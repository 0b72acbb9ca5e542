"""What a pending call on a named stream uses may be dropped: its source
weights, the object with its 8-bit ones, the tensors given.  Blocks of their
sizes are taken and overwritten at once on the current stream."""
import pytest
import torch

from paper_2609_33614_amd.layer import Fp8Experts, Fp8Matrix
from tests import test_gpu_fp8 as Q
from tests import test_gpu_sort as S

pytestmark = pytest.mark.gpu

T, d, F, E, k = 700, 256, 192, 8, 2


def sizes(*tensors):
    return sorted({t.numel() * t.element_size() for t in tensors})


def overwrite(which):
    """(pending on nothing: the current stream has no work)"""
    return [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in which for _ in range(16)]


def busy():
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    return side


def test_the_source_weights_right_after_construction():
    w, x, off, token = Q.make_experts(T, d, F, E, k)
    off, token = off.int().cuda(), token.int().cuda()
    want = Fp8Experts(w).forward(x, off, token), Fp8Matrix(w["w1"], gradients=True).product(x, off, token)
    src, mat = {n: t.clone() for n, t in w.items()}, w["w1"].clone()
    side, n = busy(), sizes(*w.values())
    ex, m = Fp8Experts(src, stream=side), Fp8Matrix(mat, gradients=True, stream=side)
    del src, mat
    junk = overwrite(n)
    torch.cuda.synchronize()
    assert torch.equal(ex.forward(x, off, token), want[0]) and torch.equal(m.product(x, off, token), want[1]) and junk


@pytest.mark.parametrize("named", [True, False])
def test_the_object_right_after_a_call(named):
    w, x, off, token = Q.make_experts(T, d, F, E, k)
    off, token = off.int().cuda(), token.int().cuda()
    saved, dy = torch.empty(T * k, 2 * F, dtype=torch.bfloat16, device="cuda"), Q.normal(T * k, d)

    def run(stream=None):
        ex, m = Fp8Experts(w, gradients=True), Fp8Matrix(w["w1"], gradients=True)
        n = sizes(ex.buf, m.q, m.scale, m.qt, m.scale_t)
        side = busy()
        stream = side if named else None
        with torch.cuda.stream(torch.cuda.current_stream() if named else side):
            y = ex.forward(x, off, token, saved=saved, stream=stream)
            p = m.product(x, off, token, stream=stream)
            out = [y, ex.backward(dy, saved, off, stream=stream), p, m.product_backward(p, off, stream=stream)]
        del ex, m
        junk = overwrite(n)
        torch.cuda.synchronize()
        return out, junk

    ex, m = Fp8Experts(w, gradients=True), Fp8Matrix(w["w1"], gradients=True)
    y, p = ex.forward(x, off, token, saved=saved), m.product(x, off, token)
    want = [y, ex.backward(dy, saved, off), p, m.product_backward(p, off)]
    got, _ = run()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_tensors_given():
    b = S.make(T, E, d, True, k)
    lay = S.make_layer(E, d, True, T)
    w, _, _, _ = Q.make_experts(T, d, F, E, k)
    ex = Fp8Experts(w, gradients=True)

    def run(given, stream):
        """Every tensor given is dropped after the call that reads it."""
        g = {n: t.clone() for n, t in given.items()}
        side = busy()
        stream = side if stream else None
        n = sizes(*g.values())
        _, off, token, place = lay.sort(None, g["mask"], cap=b["n"], stream=stream)
        saved = torch.empty(b["n"], 2 * F, dtype=torch.bfloat16, device="cuda")
        rows = ex.forward(g.pop("x"), off, token, saved=saved, stream=stream)
        y = lay.combine(rows, g["mask"], g["gate"], place, stream=stream)
        drows, dz = torch.empty_like(rows), torch.empty_like(g["prob"])
        lay.combine_backward(g.pop("dy"), rows, g["mask"], g.pop("gate"), place, prob=g.pop("prob"), drows=drows, dlogits=dz, stream=stream)
        dr = ex.backward(drows, saved, off, stream=stream)
        del drows, saved
        dx = lay.sort_backward(dr, g.pop("mask"), place, stream=stream)
        junk = overwrite(n + [b["n"] * d * 2, b["n"] * F * 4])
        torch.cuda.synchronize()
        return [y, rows, dz, dx], junk

    given = {n: b[n] for n in ("x", "mask", "gate", "prob", "dy")}
    want, got = run(given, False)[0], run(given, True)[0]
    assert all(torch.equal(a, c) for a, c in zip(want, got))
