"""Few positions that count among many that do not: their gradients are as
exact as in a call of their own (up to 64 counted positions G has two bf16
parts, whatever the call's length; see tests/test_gpu_ce.py for the bounds)."""
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import CrossEntropy, capture
from tests.test_gpu_ce import IGN, call, check, make, reference

pytestmark = pytest.mark.gpu


def few(T, d, V, n, seed=0, lift=8.0):
    """n positions count, spread over the T."""
    h, w, y = make(T, d, V, seed=seed, lift=lift)
    g = torch.Generator().manual_seed(seed + n)
    off = torch.ones(T, dtype=torch.bool)
    off[torch.randperm(T, generator=g)[:n]] = False
    y[off.cuda()] = IGN
    return h, w, y


def tight(h, w, y, mean=True, scale=1.0):
    """The reference with the bounds of a call of the counted rows alone."""
    rows = (y != IGN).nonzero()[:, 0]
    ref, own = reference(h, w, y, mean, scale), reference(h[rows], w, y[rows], mean, scale)
    ref["bounds"]["dw"] = own["bounds"]["dw"]
    ref["bounds"]["dh"][rows] = own["bounds"]["dh"]
    return ref


# T, d, V: first passes on 128- and 256-row tiles, one piece and (least workspace) several
CALLS = [(65, 64, 129), (128, 128, 4999), (200, 256, 1500), (300, 192, 4096 * 2 + 300), (2100, 512, 16387)]


@pytest.mark.parametrize("T,d,V", CALLS)
@pytest.mark.parametrize("n", [0, 1, 2, 5, 33, 63, 64])
@pytest.mark.parametrize("most", [None, 0])
def test_bounds_of_the_counted_rows_alone(T, d, V, n, most):
    h, w, y = few(T, d, V, n)
    ref = tight(h, w, y)
    got = call(h, w, y, most=most)
    check(f"ce few {T} {V} {n}", got, ref)
    assert (got["dh"][y == IGN] == 0).all()
    for kw in (dict(dh=False), dict(dw=False)):
        check(f"ce few {T} {V} {n} {kw}", call(h, w, y, most=most, **kw), ref)
    again = call(h, w, y, most=most, poison=False)
    for k in got:
        assert torch.equal(got[k], again[k]), k


@pytest.mark.parametrize("T,V,most", [(200, 1500, None), (4096, 1500, None), (2100, 16387, None), (300, 8500, 0)])
@pytest.mark.parametrize("n", [1, 2, 5])
def test_the_outputs_precision(T, V, most, n):
    """As test_few_rows_keep_the_outputs_precision, the rows inside longer calls."""
    for seed in range(3):
        h, w, y = few(T, 256, V, n, seed=seed, lift=3.0)
        wrong = torch.randint(0, V, (T,), device="cuda")
        h = (h.float() + 12.0 * w[wrong].float()).to(torch.bfloat16)
        got, ref = call(h, w, y, most=most), reference(h, w, y, True, 1.0)
        for k in ("dh", "dw"):
            err = (got[k].double() - ref[k]).norm() / ref[k].norm()
            assert err <= 2.0 ** -8 + 2.0 ** -14, (seed, k, float(err))


@pytest.mark.parametrize("n", [65, 66, 127, 128])
def test_just_over_64_counted(n):
    for most in (None, 0):
        h, w, y = few(300, 192, 8500, n)
        check(f"ce few over {n}", call(h, w, y, most=most), reference(h, w, y, True, 1.0))


def test_a_captured_call_over_counts_around_64():
    T, d, V = 300, 192, 5000
    h, w, y = make(T, d, V)
    ce = CrossEntropy(w, max_workspace=0)
    out = {"dh": torch.empty_like(h), "dw": torch.empty_like(w)}
    box = {}
    g = capture(lambda: box.update(loss=ce.loss(h, y, **out)))
    for n in (64, 300, 0, 65, 1, 64, 200):
        hn, _, yn = few(T, d, V, n, seed=n)
        h.copy_(hn)
        y.copy_(yn)
        g.replay()
        torch.cuda.synchronize()
        ref = call(hn, w, yn, most=0)
        assert torch.equal(box["loss"], ref["loss"])
        for k in out:
            assert torch.equal(out[k], ref[k]), (n, k)


@pytest.mark.parametrize("T", [200, 2100])
def test_nan_rows_and_in_place(T):
    h, w, y = few(T, 256, 16387, 40)
    got = call(h, w, y)
    rows = (y != IGN).nonzero()[:, 0]
    x = h.clone()
    CrossEntropy(w).loss(x, y, dh=x)
    assert torch.equal(x, got["dh"])
    bad = h.clone()
    bad[rows[3], 5] = float("nan")
    res = call(bad, w, y)
    keep = torch.arange(T, device="cuda") != rows[3]
    assert torch.isnan(res["dh"][rows[3]]).all() and torch.isnan(res["dw"]).all()
    assert torch.equal(res["dh"][keep], got["dh"][keep])
