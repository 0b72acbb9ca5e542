"""The cross entropy of logits near the ends of fp32's range."""
import pytest
import torch

from tests.test_gpu_ce import call, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [40, 300])
@pytest.mark.parametrize("most", [None, 0])
def test_logits_up_to_the_largest_floats(T, most):
    """One column of h and W is not zero, so every logit is one product and
    exact: +-2^64 times 1.25 to 1.75 times 2^63.  exp of their differences is 0 or 1."""
    d, V = 128, 8192 + 300                       # (three pieces of the smallest workspace)
    h = torch.zeros(T, d)
    h[:, 3] = 2.0 ** 64
    h[1::2, 3] = -2.0 ** 64
    w = torch.zeros(V, d)
    step = torch.arange(V) % 40                  # 128 + 2 step: eighths of a bf16's last place
    w[:, 3] = (160 + step) / 128 * 2.0 ** 63     # 1.25 to 1.5546875
    top, low = 8200, 4100                        # the largest and the smallest, once each
    w[top, 3], w[low, 3] = 1.75 * 2.0 ** 63, 2.0 ** 63
    y = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(T))
    y[4], y[5] = top, low
    h, w, y = h.bfloat16().cuda(), w.bfloat16().cuda(), y.to(torch.int32).cuda()
    got = call(h, w, y, mean=False, most=most)
    z = h.double() @ w.double().T
    t = y.long()[:, None]
    nll = (z.max(1, keepdim=True).values - z.gather(1, t))[:, 0]
    assert ((got["nll"].double() - nll).abs() <= 2.0 ** -23 * nll).all()
    G = torch.zeros_like(z).scatter_(1, z.argmax(1, keepdim=True), 1.0)
    G.scatter_add_(1, t, torch.full_like(z[:, :1], -1.0))
    dh, dw = G @ w.double(), G.T @ h.double()
    assert ((got["dh"].double() - dh).abs() <= 2.0 ** -8 * dh.abs()).all()
    # (dW of an entry: a sum of whole multiples of 2^64, fewer than 2^24 of them, then bf16)
    assert ((got["dw"].double() - dw).abs() <= 2.0 ** -8 * dw.abs()).all()


@pytest.mark.parametrize("T,V", [(100, 1000), (2100, 4219)])
def test_the_logits_gradient_is_rounded_once(T, V):
    """Hidden rows of one column each, a power of two, and no factor: dW is the
    logits' gradient as the products read it, off by one rounding to bf16 (2^-8)
    and what the first pass keeps of its exponentials (2^-10; its and the
    softmax's own error is under 2^-14)."""
    d = (T + 63) // 64 * 64
    h = torch.zeros(T, d)
    h[torch.arange(T), torch.arange(T)] = 4.0
    g = torch.Generator().manual_seed(T)
    w = (torch.randn(V, d, generator=g) * 0.7).bfloat16().cuda()
    y = torch.randint(0, V, (T,), generator=g).to(torch.int32).cuda()
    got = call(h.bfloat16().cuda(), w, y, mean=False)
    z = 4.0 * w[:, :T].double().T
    G = torch.softmax(z, 1)
    G[torch.arange(T), y.long()] -= 1.0
    mine = got["dw"][:, :T].double().T / 4.0
    assert ((mine - G).abs() <= (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -14) * G.abs()).all()
    assert (got["dw"][:, T:] == 0).all()


@pytest.mark.parametrize("T", [40, 300])
def test_an_infinite_logit(T):
    """One row's logit of one entry, not its target's, is past fp32's range."""
    d, V, t, v = 128, 1500, 7, 700
    h, w, y = make(T, d, V)
    h[:, 0] = 0.0
    y[y == v] = v + 1
    clean = call(h, w, y)
    bad, wb = h.clone(), w.clone()
    bad[t, 0] = wb[v, 0] = 2.0 ** 127             # (their product passes fp32's range; 0 times infinity would not be 0)
    got = call(bad, wb, y)
    assert torch.isinf(got["nll"][t]) and torch.isinf(got["loss"]).all()
    assert torch.isnan(got["dh"][t]).all() and torch.isnan(got["dw"][v]).any()
    keep = torch.arange(T, device="cuda") != t
    assert torch.equal(got["nll"][keep], clean["nll"][keep])
    assert torch.isfinite(got["dh"][keep]).all()
