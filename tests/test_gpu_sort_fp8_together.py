"""A step that trains a router over experts held in 8 bits: the layer routes and
sorts, Fp8Experts runs the rows, combine joins them, CrossEntropy takes the loss
and its gradient, which goes back through combine (to the rows and the router's
scores), the experts and the sort; balance_loss adds its own.  Eagerly and as
one captured graph that is replayed over new inputs, each operator against its
formula in 64 bits on what the step handed to it."""
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import CrossEntropy, EatLayer, Fp8Experts, capture
from tests import test_gpu_balance as B
from tests import test_gpu_ce as X
from tests import test_gpu_fp8 as Q
from tests import test_gpu_sort as S

pytestmark = pytest.mark.gpu

IGN, COEF, ENT, LR = -100, 0.01, 0.002, 0.05


class Step:
    def __init__(self, mode, T, E, d, F, V):
        g = torch.Generator().manual_seed(T + E + d + V)
        rnd = lambda *s: torch.randn(*s, generator=g) * s[-1] ** -0.5
        w = {"w_router": 2 * rnd(E, d), "w1": rnd(E, F, d), "w3": rnd(E, F, d), "w2": rnd(E, d, F)}
        self.w = {k: (v if k == "w_router" else v.to(torch.bfloat16)).cuda() for k, v in w.items()}
        self.layer = EatLayer(L.eat_params_default(mode=mode, E=E, d_model=d, d_ffn=F, top_k=2), T, self.w)
        self.experts = Fp8Experts(self.w, gradients=True)
        self.head = rnd(V, d).to(torch.bfloat16).cuda()
        self.ce = CrossEntropy(self.head, ignore=IGN)
        self.T, self.E, self.d, self.F, self.V = T, E, d, F, V
        self.x = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
        self.y = torch.zeros(T, dtype=torch.int32, device="cuda")
        self.valid = torch.zeros(T, dtype=torch.bool, device="cuda")

    def feed(self, seed):
        g = torch.Generator().manual_seed(seed)
        self.x.copy_(torch.randn(self.T, self.d, generator=g))
        y = torch.randint(0, self.V, (self.T,), generator=g).int()
        y[torch.rand(self.T, generator=g) < 0.25] = IGN
        y[0] = 0
        self.y.copy_(y)
        self.valid.copy_(y != IGN)

    def run(self):
        lay = self.layer
        mask, _, gate, prob = lay.route(self.x)
        _, off, token, place = lay.sort(None, mask)
        rows = token.shape[0]
        e = lambda *s, t=torch.bfloat16: torch.empty(*s, dtype=t, device="cuda")
        saved, drows = e(rows, 2 * self.F), e(rows, self.d)
        # (behind the last selected pair token is not written: the experts do not look there)
        out = self.experts.forward(self.x, off, token, saved=saved)
        h = lay.combine(out, mask, gate, place)
        ces = {"nll": e(self.T, t=torch.float32), "count": e(1, t=torch.int32), "dh": e(self.T, self.d), "dw": e(self.V, self.d)}
        loss = self.ce.loss(h, self.y, **ces)
        dz, bz = e(self.T, self.E, t=torch.float32), e(self.T, self.E, t=torch.float32)
        lay.combine_backward(ces["dh"], out, mask, gate, place, prob=prob, drows=drows, dlogits=dz)
        dsort = self.experts.backward(drows, saved, off)
        dx = lay.sort_backward(dsort, mask, place)
        bal = {"dlogits": bz, "dx": e(self.T, self.d), "dw_router": e(self.E, self.d, t=torch.float32)}
        bloss, count, mean = lay.balance_loss(self.x, prob, mask, self.valid, COEF, ENT, **bal)
        self.out = dict(mask=mask, gate=gate, prob=prob, off=off, token=token, place=place, saved=saved, drows=drows, rows=out, h=h,
                        ces=ces, loss=loss, dz=dz, dsort=dsort, dx=dx, bal=bal, bloss=bloss, count=count, mean=mean)

    def descend(self):
        # the scores are the router's rows times x
        self.layer.w["w_router"].add_((self.out["dz"].T @ self.x.float()) * self.layer.params.inv_temperature, alpha=-LR)
        self.layer.w["w_router"].add_(self.out["bal"]["dw_router"], alpha=-LR)

    def check(self, name, router):
        o, lay, T = self.out, self.layer, self.T
        sel = torch.stack([((o["mask"].view(T, -1)[:, e // 64] >> (e % 64)) & 1) > 0 for e in range(self.E)], 1)
        off, token, place = S.index(sel)
        n = token.shape[0]
        assert torch.equal(o["off"].long(), off) and torch.equal(o["token"][:n].long(), token) and torch.equal(o["place"].long(), place)
        w = {k: self.w[k] for k in ("w1", "w3", "w2")}
        offc = off.cpu()
        (ry, by, _), (rs, bs) = Q.experts_reference(self.x, w, offc, token)
        Q.within(f"{name} rows", o["rows"][:n], ry, by)
        half = 2.0 ** -8
        Q.within(f"{name} saved", o["saved"][:n], rs, (1 + half) * bs + half * rs.abs() + Q.TINY)
        rows, drows = o["rows"][:n], o["drows"][:n]
        wt = o["gate"].double()[place >= 0][torch.argsort(place[place >= 0])]
        S.within(f"{name} h", o["h"], *S.sums(token, rows, wt, T, half))
        ces = o["ces"]
        X.check(f"{name} ce", {"loss": o["loss"], **ces}, X.reference(o["h"], self.head, self.y, True, 1.0))
        b = {"sel": sel, "gate": o["gate"], "prob": o["prob"], "dy": ces["dh"], "rows": rows, "half": half}
        ref = S.grads(b, place, lay.params.eps)
        S.within(f"{name} drows", drows, *ref["drows"])
        S.within(f"{name} dlogits", o["dz"], *ref["dlogits"])
        rdx, bdx, _ = Q.backward_reference(drows, o["saved"][:n], w, offc)
        Q.within(f"{name} dsort", o["dsort"][:n], rdx, bdx)
        one = torch.ones(n, dtype=torch.float64, device="cuda")
        S.within(f"{name} dx", o["dx"], *S.sums(token, o["dsort"][:n], one, T, half))
        now = lay.w["w_router"]
        try:
            lay.w["w_router"] = router
            ref = B.reference(lay, self.x, o["prob"], o["mask"], self.valid, COEF, ENT)
        finally:
            lay.w["w_router"] = now
        B.check(f"{name} bal", {"loss": o["bloss"], "count": o["count"], "mean": o["mean"], **o["bal"]}, ref)


@pytest.mark.parametrize("mode,T,E,d,F,V", [("topk", 1, 8, 128, 192, 100), ("eat", 48, 8, 256, 128, 300), ("topp", 300, 60, 256, 128, 250),
                                            ("topk", 600, 128, 256, 192, 500), ("topk", 2100, 16, 512, 320, 300)])
def test_a_step_eager_and_replayed(mode, T, E, d, F, V):
    s = Step(mode, T, E, d, F, V)

    def step():
        s.run()
        s.descend()

    for seed in range(2):
        s.feed(seed)
        router = s.layer.w["w_router"].clone()
        step()
        torch.cuda.synchronize()
        s.check(f"8-bit step {mode} {T} eager", router)
    graph = capture(step)
    held = s.out                                     # (what the replays write)
    for seed in range(10, 13):
        s.feed(seed)
        router = s.layer.w["w_router"].clone()
        graph.replay()
        torch.cuda.synchronize()
        s.out = held
        s.check(f"8-bit step {mode} {T} replay", router)
        after = s.layer.w["w_router"].clone()
        got = {k: v.clone() for k, v in held.items() if torch.is_tensor(v)}
        s.layer.w["w_router"].copy_(router)
        step()                                       # (eagerly, on the same inputs)
        torch.cuda.synchronize()
        n = int(got["off"][-1])
        for k in ("off", "place", "h", "dz", "dx", "loss"):
            assert torch.equal(got[k], s.out[k]), k
        assert torch.equal(got["rows"][:n], s.out["rows"][:n]) and torch.equal(after, s.layer.w["w_router"])


@pytest.mark.parametrize("T,E,d,F", [(1, 8, 512, 1024), (40, 60, 512, 256), (900, 16, 256, 512)])
def test_the_layers_own_output_is_near(T, E, d, F):
    """EatLayer.forward keeps the experts in bf16.  An 8-bit rounding is off by at most 2^-4, 2^-4 / sqrt(3) =
    0.036 at the root of its mean square, a product of two of them 0.051.  g and u are about
    normal with variance 1 here: silu's slope is at most 1.1 and silu(g) has the mean square
    0.36, so h is off by sqrt((1.1 / 0.6 0.051)^2 + 0.051^2) = 0.107 of its own, and y by
    sqrt(0.107^2 + 0.051^2) = 0.119."""
    s = Step("topk", T, E, d, F, 64)
    s.feed(3)
    s.run()
    want = s.layer.forward(s.x).double()
    off = (s.out["h"].double() - want).square().sum().sqrt() / want.square().sum().sqrt()
    assert float(off) <= 0.125, float(off)
    assert float(off) >= 2.0 ** -9                   # (the numbers are the 8-bit ones)
