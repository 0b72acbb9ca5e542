"""A captured step of sort, 8-bit experts, combine and their gradients replayed
with eager calls of the same objects between the replays, on other tokens (a
larger and a smaller batch: their workspaces are the graph's, or replace them).
Every replay and every eager call gives the bits of objects that nothing else uses."""
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import EatLayer, Fp8Experts, Fp8Matrix, capture
from tests import test_gpu_fp8 as Q

pytestmark = pytest.mark.gpu


class Step:
    def __init__(self, w, mode, max_tokens):
        E, F, d = w["w1"].shape
        self.F = F
        self.lay = EatLayer(L.eat_params_default(mode=mode, E=E, d_model=d, d_ffn=F, top_k=3), max_tokens, {"w_router": w["w_router"]})
        self.ex, self.m = Fp8Experts(w, gradients=True), Fp8Matrix(w["w2"], gradients=True)

    def run(self, x, dy, n):
        mask, _, gate, prob = self.lay.route(x)
        rows, off, token, place = self.lay.sort(x, mask, cap=n)
        saved = torch.empty(n, 2 * self.F, dtype=torch.bfloat16, device="cuda")
        y = self.ex.forward(x, off, token, y=torch.zeros_like(rows), saved=saved)
        out = self.lay.combine(y, mask, gate, place)
        drows, dz = torch.zeros_like(y), torch.empty_like(prob)
        self.lay.combine_backward(dy, y, mask, gate, place, prob=prob, drows=drows, dlogits=dz)
        dx = self.lay.sort_backward(self.ex.backward(drows, saved, off, dx=drows), mask, place)
        wide = torch.zeros(n, self.F, dtype=torch.bfloat16, device="cuda")
        self.m.product_backward(y, off, dx=wide)
        back = torch.zeros_like(y)
        return [mask, off, place, out, dz, dx, wide, self.m.product(wide, off, out=back)]


def batch(T, d, seed):
    return Q.normal(T, d, seed=seed), Q.normal(T, d, seed=seed + 1, std=0.1)


@pytest.mark.parametrize("mode", ["topk", "eat"])
def test_eager_calls_of_the_same_objects_between_the_replays(mode):
    T, d, F, E = 300, 256, 192, 60
    w, _, _, _ = Q.make_experts(T, d, F, E, 1)
    w["w_router"] = Q.normal(E, d, std=d ** -0.5, dtype=torch.float32)
    rows = lambda T: T * (3 if mode == "topk" else E)
    used, alone = Step(w, mode, 1000), Step(w, mode, 1000)
    x, dy = batch(T, d, 0)
    got = []

    def step():
        got[:] = used.run(x, dy, rows(T))

    graph = capture(step)
    kept = list(got)
    for k, other in enumerate((700, 100, 1, 1000)):
        a = batch(T, d, 10 + k)
        x.copy_(a[0])
        dy.copy_(a[1])
        graph.replay()
        b = batch(other, d, 50 + k)
        eager = used.run(*b, rows(other))                 # (behind the replay, on the same stream)
        torch.cuda.synchronize()
        for have, want in ((kept, alone.run(*a, rows(T))), (eager, alone.run(*b, rows(other)))):
            assert all(torch.equal(p, q) for p, q in zip(have, want))
