"""The cross entropy on its 256 x 256 tiles: first pass, recomputed pieces, dh
in slices, written directly and added over pieces, dW (which tile each takes:
tests/test_launch_lists_losses_large.py), against the formulas in 64 bits."""
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import CrossEntropy
from tests.ce_large import CALLS
from tests.test_gpu_ce import IGN, call, check, make, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ignored", [None, 0.25, 0.97])
@pytest.mark.parametrize("name", list(CALLS))
def test_large_tiles(name, ignored):
    T, d, V, least, several = CALLS[name]
    h, w, y = make(T, d, V, ignored=ignored)
    y[:3] = torch.tensor([0, V - 1, IGN], dtype=torch.int32)
    ref = reference(h, w, y, True, 1.0)
    most = 0 if least else None
    got = call(h, w, y, most=most)
    check(f"ce large {name} {ignored}", got, ref)
    assert (got["dh"][y == IGN] == 0).all()
    again = call(h, w, y, most=most, poison=False)
    for k in got:
        assert torch.equal(got[k], again[k]), k
    for kw in (dict(dh=False), dict(dw=False)):
        part = call(h, w, y, most=most, **kw)
        assert torch.equal(part["loss"], got["loss"]) and torch.equal(part["nll"], got["nll"])
        check(f"ce large {name} {ignored} {kw}", part, ref)


@pytest.mark.parametrize("name", [n for n, c in CALLS.items() if c[4] is not None])
def test_dh_has_the_slices_it_is_said_to_have(name):
    """(The count is the fourth word of the workspace.)"""
    T, d, V, _, several = CALLS[name]
    h, w, y = make(T, d, V)
    ce = CrossEntropy(w)
    ce.loss(h, y, dh=torch.empty_like(h))
    slices = int(ce.workspace(T, L.EAT_CE_DH)[:16].view(torch.int32)[3])
    assert (slices > 1) == several, slices


def test_rows_and_targets_that_are_not_numbers():
    T, d, V = 2049, 512, 16387
    h, w, y = make(T, d, V, ignored=0.1)
    y[7], y[1030] = 3, 4
    clean = call(h, w, y)
    bad, yb = h.clone(), y.clone()
    bad[7, 3], yb[1030] = float("nan"), V
    got = call(bad, w, yb)
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[[7, 1030]] = False
    assert torch.isnan(got["nll"][~keep]).all() and torch.equal(got["nll"][keep], clean["nll"][keep])
    assert torch.isnan(got["dh"][~keep]).all() and torch.equal(got["dh"][keep], clean["dh"][keep])
    assert torch.isnan(got["dw"]).all()
