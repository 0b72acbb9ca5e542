"""A training step's tail out of the layer and the two losses: the layer routes
and runs its experts, CrossEntropy takes the loss of the layer's output, its
gradients and the head's, EatLayer.balance_loss the router's from the same
routing, the padded positions left out of both; then a step of descent on the
head and the router's weights.  Eagerly and as one captured graph that is
replayed over new inputs, each pass against the formulas in 64 bits."""
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import CrossEntropy, EatLayer, capture
from tests import test_gpu_balance as B
from tests import test_gpu_ce as X

pytestmark = pytest.mark.gpu

IGN, COEF, ENT, LR = -100, 0.01, 0.002, 0.05


class Step:
    """Inputs, weights and outputs of one step, at fixed addresses."""

    def __init__(self, mode, T, E, d, V, F=128):
        g = torch.Generator().manual_seed(T + E + d + V)
        rnd = lambda *s: torch.randn(*s, generator=g) * s[-1] ** -0.5
        w = {"w_router": 2 * rnd(E, d), "w1": rnd(E, F, d), "w3": rnd(E, F, d), "w2": rnd(E, d, F)}
        w = {k: (v if k == "w_router" else v.to(torch.bfloat16)).cuda() for k, v in w.items()}
        p = L.eat_params_default(mode=mode, E=E, d_model=d, d_ffn=F, top_k=2)
        self.layer, self.head = EatLayer(p, T, w), rnd(V, d).to(torch.bfloat16).cuda()
        self.ce = CrossEntropy(self.head, ignore=IGN)
        self.T, self.d, self.V = T, d, V
        self.x, self.y = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
        self.valid = torch.zeros(T, dtype=torch.bool, device="cuda")
        e = lambda *s, t=torch.bfloat16: torch.empty(*s, dtype=t, device="cuda")
        self.ces = {"nll": e(T, t=torch.float32), "count": e(1, t=torch.int32), "dh": e(T, d), "dw": e(V, d)}
        self.bal = {"dlogits": e(T, E, t=torch.float32), "dx": e(T, d), "dw_router": e(E, d, t=torch.float32)}
        self.out = {}

    def feed(self, seed):
        g = torch.Generator().manual_seed(seed)
        self.x.copy_(torch.randn(self.T, self.d, generator=g))
        y = torch.randint(0, self.V, (self.T,), generator=g).int()
        y[torch.rand(self.T, generator=g) < 0.25] = IGN
        y[(3 * self.T + 3) // 4:] = IGN
        self.y.copy_(y)
        self.valid.copy_(y != IGN)

    def run(self):
        mask, _, _, prob = self.layer.route(self.x)
        h = self.layer.forward(self.x)
        loss = self.ce.loss(h, self.y, **self.ces)
        bloss, count, mean = self.layer.balance_loss(self.x, prob, mask, self.valid, COEF, ENT, **self.bal)
        self.out = {"mask": mask, "prob": prob, "h": h, "loss": loss, "bloss": bloss, "count": count, "mean": mean}

    def descend(self):
        self.head.add_(self.ces["dw"], alpha=-LR)
        self.layer.w["w_router"].add_(self.bal["dw_router"], alpha=-LR)

    def check(self, name, head, router):
        """Against the weights as they were before the step."""
        o, now = self.out, self.layer.w["w_router"]
        X.check(f"{name} ce", {"loss": o["loss"], **self.ces}, X.reference(o["h"], head, self.y, True, 1.0))
        try:
            self.layer.w["w_router"] = router
            ref = B.reference(self.layer, self.x, o["prob"], o["mask"], self.valid, COEF, ENT)
        finally:
            self.layer.w["w_router"] = now
        B.check(f"{name} bal", {"loss": o["bloss"], "count": o["count"], "mean": o["mean"], **self.bal}, ref)
        assert int(self.ces["count"]) == int(self.valid.sum())
        off = ~self.valid
        assert (self.ces["dh"][off] == 0).all() and (self.bal["dx"][off] == 0).all()


@pytest.mark.parametrize("mode,T,E,d,V", [("topk", 1, 8, 128, 100), ("eat", 48, 8, 256, 1000), ("topp", 300, 60, 256, 777),
                                          ("topk", 600, 128, 512, 1500), ("topk", 4100, 128, 1024, 600)])
def test_a_step_eager_and_replayed(mode, T, E, d, V):
    s = Step(mode, T, E, d, V)
    for seed in range(2):
        s.feed(seed)
        head, router = s.head.clone(), s.layer.w["w_router"].clone()
        s.run()
        s.descend()
        torch.cuda.synchronize()
        s.check(f"step {mode} {T} eager", head, router)

    def step():
        s.run()
        s.descend()

    g = capture(step)
    for seed in range(10, 14):
        s.feed(seed)
        head, router = s.head.clone(), s.layer.w["w_router"].clone()
        g.replay()
        torch.cuda.synchronize()
        s.check(f"step {mode} {T} replay", head, router)
        assert not torch.equal(head, s.head) or int(s.valid.sum()) == 0


def test_gradients_of_the_sum_against_differences():
    """Both losses as one function of the router's input and weights and of the
    head, the selections and the layer's output held: central differences in 64
    bits along random directions."""
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
    mine = [s.bal["dx"], s.bal["dw_router"], s.ces["dh"], s.ces["dw"]]
    rc, rb = X.reference(s.out["h"], s.head, s.y, True, 1.0), B.reference(s.layer, s.x, s.out["prob"], s.out["mask"], s.valid, COEF, ENT)
    bounds = [rb["bounds"]["dx"], rb["bounds"]["dw_router"], rc["bounds"]["dh"], rc["bounds"]["dw"]]
    g = torch.Generator(device="cuda").manual_seed(3)
    e = 1e-4
    for k in range(4):
        u = torch.randn(at[k].shape, generator=g, device="cuda", dtype=torch.float64)
        hi, lo = ([a + sign * e * u if i == k else a for i, a in enumerate(at)] for sign in (1, -1))
        slope = (total(*hi) - total(*lo)) / (2 * e)
        # the step's third derivative and the routing's fp32 probabilities: 1e-4
        bound = (bounds[k] * u.abs()).sum() + 1e-4 * slope.abs() + 1e-7
        assert ((mine[k].double() * u).sum() - slope).abs() <= bound, (k, float(slope))
