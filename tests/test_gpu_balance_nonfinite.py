"""Tokens that do not count have gradients of zero whatever the others and the
router weights hold, in calls of every size (the sums' own workgroup, the
fp32 products and the products of bf16 parts each have their way of leaving
them out)."""
import pytest
import torch

from tests.test_gpu_balance import call, make_valid, routed

pytestmark = pytest.mark.gpu

# (T, E, d, bf16): gradients of the scores by the sums' workgroup, by a launch of their own, on bf16 parts
SIZES = [(20, 8, 64, False), (700, 12, 64, True), (700, 60, 128, True), (900, 200, 128, False), (2300, 60, 1024, True),
         (2100, 250, 4160, False)]


@pytest.mark.parametrize("T,E,d,bf16", SIZES)
def test_a_nan_token_reaches_no_token_that_does_not_count(T, E, d, bf16):
    layer, x, prob, mask = routed(E, d, bf16, T)
    valid = make_valid(T, "some")
    prob[int(valid.nonzero()[0]), E // 2] = float("nan")
    got = call(layer, x, prob, mask, valid)
    assert torch.isnan(got["loss"]).all() and torch.isnan(got["dlogits"][valid]).all() and torch.isnan(got["dw_router"]).all()
    assert (got["dlogits"][~valid] == 0).all() and (got["dx"][~valid] == 0).all()


@pytest.mark.parametrize("T,E,d,bf16", SIZES)
def test_an_infinite_router_weight_reaches_no_token_that_does_not_count(T, E, d, bf16):
    """(0 times infinity is no 0.)"""
    layer, x, prob, mask = routed(E, d, bf16, T)
    valid = make_valid(T, "some")
    clean = call(layer, x, prob, mask, valid)
    layer.w["w_router"][E // 3, 5], layer.w["w_router"][0, d - 1] = float("inf"), float("nan")
    got = call(layer, x, prob, mask, valid)
    assert (got["dx"][~valid] == 0).all()
    keep = [c for c in range(d) if c not in (5, d - 1)]
    assert torch.equal(got["dx"][:, keep], clean["dx"][:, keep]) and not torch.isfinite(got["dx"][valid][:, [5, d - 1]]).any()
    for k in ("loss", "dlogits", "dw_router"):
        assert torch.equal(got[k], clean[k]), k
