"""The losses' gradients against central differences of the 64-bit losses, in
directions in which a wrong gradient shows.

The 64-bit gradient (the formula) is held to the differences along random
directions, at the differences' own error: the step's third-order term, under
1e-6 of the absolute terms.  The kernels' gradient is then held to them along
the 64-bit gradient, where the slope is its square: what its elementwise bound
allows there has to be under a quarter of the slope, so a gradient that is
zero, has another sign or is off by a quarter fails."""
import pytest
import torch

from tests import test_gpu_balance as B
from tests import test_gpu_ce as X

pytestmark = pytest.mark.gpu


def against_differences(name, f, at, mine, want, bound, extra=0.0):
    """f: the loss of the fp64 tensor `at`; want: its gradient by the formula,
    mine: the kernels' gradient, within `bound` of it; extra: relative."""
    g = torch.Generator(device="cuda").manual_seed(11)

    def slope(u, e):
        return (f(at + e * u) - f(at - e * u)) / (2 * e)

    for _ in range(3):
        u = torch.randn(at.shape, generator=g, device="cuda", dtype=torch.float64)
        terms = (want * u).abs().sum()
        assert ((want * u).sum() - slope(u, 1e-5)).abs() <= (1e-6 + extra) * terms, name
    u = want / want.abs().max()
    s = slope(u, 1e-5)
    allowed = (bound * u.abs()).sum() + (1e-6 + extra) * s.abs()
    assert 4 * allowed < s, (name, float(allowed), float(s))
    assert ((mine.double() * u).sum() - s).abs() <= allowed, (name, float(s))


@pytest.mark.parametrize("T", [33, 290, 1500])
@pytest.mark.parametrize("mean", [True, False])
def test_cross_entropy(T, mean):
    d, V = 128, 400
    h, w, y = X.make(T, d, V, ignored=0.1)
    got, ref = X.call(h, w, y, mean=mean, scale=0.5), X.reference(h, w, y, mean, 0.5)
    rows = (y != X.IGN).nonzero()[:, 0]
    t = y[rows].long()

    def loss64(a, b):
        z = a[rows] @ b.T
        nll = torch.logsumexp(z, 1) - z.gather(1, t[:, None])[:, 0]
        return 0.5 * (nll.mean() if mean else nll.sum())

    hd, wd = h.double(), w.double()
    against_differences("dh", lambda a: loss64(a, wd), hd, got["dh"], ref["dh"], ref["bounds"]["dh"])
    against_differences("dw", lambda b: loss64(hd, b), wd, got["dw"], ref["dw"], ref["bounds"]["dw"])


@pytest.mark.parametrize("T,E,d,bf16", [(150, 24, 64, False), (2300, 60, 1024, True)])
def test_balance(T, E, d, bf16):
    layer, x, prob, mask = B.routed(E, d, bf16, T)
    valid = B.make_valid(T, "some")
    got, ref = B.call(layer, x, prob, mask, valid, 0.5, 0.1), B.reference(layer, x, prob, mask, valid, 0.5, 0.1)
    f = ref["count"].double() / int(ref["count"].sum())

    def loss64(a, w):
        P = torch.softmax(a[valid] @ w.T, 1).mean(0)
        return 0.5 * E * (f * P).sum() + 0.1 * (P * P.log()).sum()

    xd, wd = x.double(), layer.w["w_router"].double()
    # (prob is the fp32 softmax of fp32 scores: 2e-5 relative, as the routing tests have it)
    against_differences("dx", lambda a: loss64(a, wd), xd, got["dx"], ref["dx"], ref["bounds"]["dx"], 1e-4)
    against_differences("dw_router", lambda b: loss64(xd, b), wd, got["dw_router"], ref["dw_router"],
                        ref["bounds"]["dw_router"], 1e-4)


def test_both_as_one_function():
    """As test_gradients_of_the_sum_against_differences, with directions that tell."""
    from tests.test_gpu_losses_together import COEF, ENT, Step
    s = Step("topk", 80, 16, 128, 300)
    s.feed(5)
    s.run()
    torch.cuda.synchronize()
    rows = s.valid.nonzero()[:, 0]
    f = s.out["count"].double() / int(s.out["count"].sum())
    t = s.y[rows].long()

    def total(x, router, h, head):
        P = torch.softmax(x[rows] @ router.T, 1).mean(0)
        bal = COEF * 16 * (f * P).sum() + ENT * (P * P.log()).sum()
        return torch.nn.functional.cross_entropy(h[rows] @ head.T, t) + bal

    at = [s.x.double(), s.layer.w["w_router"].double(), s.out["h"].double(), s.head.double()]
    rc, rb = X.reference(s.out["h"], s.head, s.y, True, 1.0), B.reference(s.layer, s.x, s.out["prob"], s.out["mask"], s.valid, COEF, ENT)
    for k, (mine, ref, key) in enumerate(((s.bal["dx"], rb, "dx"), (s.bal["dw_router"], rb, "dw_router"), (s.ces["dh"], rc, "dh"),
                                          (s.ces["dw"], rc, "dw"))):
        against_differences(key, lambda a: total(*[a if i == k else b for i, b in enumerate(at)]), at[k], mine, ref[key],
                            ref["bounds"][key], 1e-4 if k < 2 else 0.0)
