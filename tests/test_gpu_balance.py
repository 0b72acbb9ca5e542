"""The router's balance loss, counts and gradients (eat_balance_loss) against
the formulas in 64 bits.

Bounds.  Counts are exact.  P and the loss are fp64 sums rounded once to fp32.
q is rounded once to fp32; dz = p (q - <q, p>) / n has the difference of q
(one rounding) and an fp64 sum, its rounding and one product's: with
Q = max |q|, |dz| is off by p Q (2^-24 + ...) -- 4 2^-24 p Q covers the three.
The products are fp32 sums of K terms: K 2^-24 of the sum of absolute terms
more (matrix instructions may also flush denormals: 2^-126 each), and the
outputs' own rounding (fp32 2^-24, bf16 2^-8).  A product whose operands are
split into bf16 parts keeps 2^-22 of each factor in fp32 outputs, 2^-15 in bf16 ones."""
import numpy as np
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import EatLayer, capture
from tests import parity as PT

pytestmark = pytest.mark.gpu


def make_layer(E, d, bf16, T, mode="topk", k=2, inv_temp=1.0, seed=0, **kw):
    dt = L.EAT_BF16 if bf16 else L.EAT_F32
    p = L.eat_params_default(mode=mode, E=E, d_model=d, d_ffn=64, top_k=min(k, E), act_dtype=dt, expert_dtype=dt,
                             inv_temperature=inv_temp, **kw)
    g = torch.Generator().manual_seed(seed + E + d)
    w = (torch.randn(E, d, generator=g) * 2 * d ** -0.5).cuda()
    return EatLayer(p, max(T, 1), {"w_router": w})


def make_x(T, d, bf16, seed=0):
    g = torch.Generator().manual_seed(seed + T + d)
    mu = torch.randn(4, d, generator=g)
    x = mu[torch.randint(0, 4, (T,), generator=g)] + torch.randn(T, d, generator=g)
    return x.to(torch.bfloat16 if bf16 else torch.float32).cuda()


def make_valid(T, kind, seed=0):
    g = torch.Generator().manual_seed(seed + T)
    if kind is None:
        return None
    v = {"some": torch.rand(T, generator=g) < 0.7, "none": torch.zeros(T, dtype=torch.bool),
         "one": torch.arange(T) == T // 2, "tail": torch.arange(T) < (3 * T) // 4}[kind]
    return v.cuda()


def call(layer, x, prob, mask, valid, coef=0.01, ent=0.002, dz=True, dx=True, dw=True, guard=256):
    def out(shape, dtype):
        n = int(np.prod(shape))
        buf = torch.full((n + 2 * guard,), 7.0, dtype=dtype, device="cuda")
        return buf, buf[guard:guard + n].view(*shape)

    bufs = {}
    if dz:
        bufs["dlogits"] = out(prob.shape, torch.float32)
    if dx:
        bufs["dx"] = out(x.shape, x.dtype)
    if dw:
        bufs["dw_router"] = out(layer.w["w_router"].shape, torch.float32)
    views = {k: v for k, (_, v) in bufs.items()}
    layer.balance_loss(x, prob, mask, valid, coef, ent)
    layer._bws.buf.fill_(0xFF)
    loss, count, mean = layer.balance_loss(x, prob, mask, valid, coef, ent, **views)
    torch.cuda.synchronize()
    for k, (buf, _) in bufs.items():
        assert (buf[:guard] == 7).all() and (buf[-guard:] == 7).all(), f"{k}: written outside"
    return {"loss": loss, "count": count, "mean": mean, **views}


def unpack(mask, E):
    m = mask.reshape(mask.shape[0], -1)
    return torch.stack([(m[:, e // 64] >> (e % 64)) & 1 for e in range(E)], dim=1) if m.shape[0] else m.new_zeros(0, E)


def reference(layer, x, prob, mask, valid, coef, ent):
    E, it = layer.params.E, float(layer.params.inv_temperature)
    T = prob.shape[0]
    live = valid.bool() if valid is not None else torch.ones(T, dtype=torch.bool, device=prob.device)
    rows = live.nonzero()[:, 0]
    n = max(rows.numel(), 1)
    c = unpack(mask, E)[rows].sum(0)
    f = c.double() / max(int(c.sum()), 1)
    p = prob[rows].double()
    P = p.sum(0) / n
    lg = torch.where(P > 0, torch.log(P), torch.zeros_like(P))
    loss = coef * E * (f * P).sum() + ent * (P * lg).sum()
    q = (coef * E * f + ent * (lg + 1)) / n
    u = 2.0 ** -24
    dz = torch.zeros(T, E, dtype=torch.float64, device=prob.device)
    dz[rows] = p * (q - (p @ q)[:, None])
    bz = torch.zeros_like(dz)
    bz[rows] = 4 * u * p * (q.abs().max() + (p @ q).abs()[:, None])
    bz += u * dz.abs() + 2.0 ** -126
    w, xd = layer.w["w_router"].double(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    xd[rows] = x[rows].double()
    half = 2.0 ** -8 if x.dtype == torch.bfloat16 else u
    split = 2.0 ** -15 if x.dtype == torch.bfloat16 else 2.0 ** -22
    dx, dw = it * (dz @ w), it * (dz.T @ xd)
    bx = it * ((bz + (split + E * u) * dz.abs()) @ w.abs()) * (1 + half) + half * dx.abs() + 2.0 ** -120
    bw = it * ((bz + (2.0 ** -22 + max(T, 1) * u) * dz.abs()).T @ xd.abs()) * (1 + u) + u * dw.abs() + 2.0 ** -120
    terms = coef * E * (f * P).sum() + abs(ent) * (P * lg).abs().sum()
    return {"loss": loss, "count": c, "mean": P, "dlogits": dz, "dx": dx, "dw_router": dw,
            "bounds": {"loss": 2 * u * abs(terms) + 2.0 ** -140, "mean": 2 * u * P + 2.0 ** -140, "dlogits": bz, "dx": bx, "dw_router": bw}}


def check(name, got, ref):
    assert torch.equal(got["count"], ref["count"]), name
    for k, b in ref["bounds"].items():
        if k not in got:
            continue
        err = (got[k].double().reshape(ref[k].shape) - ref[k]).abs()
        worst = float((err / b).max()) if err.numel() else 0.0
        PT.report(f"{name} {k}", err_over_bound=f"{worst:.2f}")
        assert (err <= b).all(), f"{name}: {k} off by {worst:.2f} of its bound"


def routed(E, d, bf16, T, mode="topk", k=2, seed=0, **kw):
    layer = make_layer(E, d, bf16, T, mode, k, seed=seed, **kw)
    x = make_x(T, d, bf16, seed)
    mask, _, _, prob = layer.route(x)
    return layer, x, prob, mask


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("T,E,d,k", [(1, 1, 64, 1), (1, 8, 128, 2), (3, 5, 64, 2), (32, 8, 128, 2), (63, 64, 192, 8),
                                     (65, 60, 128, 4), (100, 65, 64, 3), (200, 100, 320, 8), (257, 128, 256, 8),
                                     (1000, 200, 128, 8), (777, 256, 512, 8), (2049, 16, 64, 1), (5000, 33, 128, 2),
                                     (2111, 64, 1024, 8), (1030, 256, 576, 8), (4111, 130, 320, 4), (20000, 7, 1024, 2),
                                     (257, 256, 2112, 2), (64, 250, 8640, 8), (16400, 1, 64, 1), (1027, 70, 8192, 4),
                                     (530, 256, 4096, 8), (250, 64, 67200, 8), (2050, 250, 4224, 8)])
def test_loss_counts_gradients(T, E, d, k, bf16):
    layer, x, prob, mask = routed(E, d, bf16, T, k=k)
    check(f"bal {T} {E} {d}", call(layer, x, prob, mask, None), reference(layer, x, prob, mask, None, 0.01, 0.002))


@pytest.mark.parametrize("kind", ["some", "none", "one", "tail"])
@pytest.mark.parametrize("T,E,d,bf16", [(1, 8, 64, False), (70, 60, 128, True), (600, 130, 192, True), (600, 12, 64, False),
                                        (2300, 60, 1024, True), (2300, 60, 1024, False), (1100, 200, 640, True),
                                        (1100, 200, 640, False), (2060, 130, 1408, True), (8000, 60, 1152, True),
                                        (16500, 12, 64, True),
                                        (2100, 250, 4160, False)])
def test_tokens_that_do_not_count(T, E, d, bf16, kind):
    layer, x, prob, mask = routed(E, d, bf16, T)
    valid = make_valid(T, kind)
    got = call(layer, x, prob, mask, valid)
    check(f"bal {kind} {T}", got, reference(layer, x, prob, mask, valid, 0.01, 0.002))
    off = ~valid
    assert (got["dx"][off] == 0).all() and (got["dlogits"][off] == 0).all()
    xb, pb = x.clone(), prob.clone()
    xb[off], pb[off] = float("nan"), float("inf")
    again = call(layer, xb, pb, mask, valid.to(torch.uint8) * 255)
    for k in got:
        assert torch.equal(got[k], again[k]), k


@pytest.mark.parametrize("mode,E", [("eat", 8), ("eat", 128), ("topp", 64), ("topk", 64)])
def test_after_every_kind_of_routing(mode, E):
    """What route returned is taken as it is: variable numbers of experts, the
    temperature, the OPD scales; a NaN token that EAT routes to no expert."""
    T, d = 300, 256
    scale = (torch.rand(E) + 0.5).cuda()
    layer = make_layer(E, d, True, T, mode, 4, inv_temp=2.0, expert_scale=scale.data_ptr())
    if mode == "eat":
        n = torch.randint(1, 50, (E,))
        layer.load_accounts(n, n * 0.02, torch.rand(E) * 0.05)
    x = make_x(T, d, True)
    mask, _, _, prob = layer.route(x)
    check(f"bal {mode} {E}", call(layer, x, prob, mask, None), reference(layer, x, prob, mask, None, 0.01, 0.002))
    if mode == "eat":
        x[5] = float("nan")
        mask, kk, _, prob = layer.route(x)
        assert int(kk[5]) == 0
        valid = torch.arange(T, device="cuda") != 5
        check(f"bal {mode} nan", call(layer, x, prob, mask, valid), reference(layer, x, prob, mask, valid, 0.01, 0.002))
        assert torch.isnan(call(layer, x, prob, mask, None)["loss"]).all()


def test_no_selection_and_zero_probabilities():
    layer, x, prob, mask = routed(60, 128, True, 90)
    mask.zero_()
    prob[:, 7] = 0.0
    got = call(layer, x, prob, mask, None)
    check("bal empty", got, reference(layer, x, prob, mask, None, 0.01, 0.002))
    assert (got["count"] == 0).all() and (got["dlogits"][:, 7] == 0).all()


@pytest.mark.parametrize("coef,ent", [(0.0, 0.0), (1.0, 0.0), (0.0, -0.8), (-3.0, 0.5)])
def test_coefficients(coef, ent):
    layer, x, prob, mask = routed(64, 128, True, 200, k=8)
    check(f"bal {coef} {ent}", call(layer, x, prob, mask, None, coef, ent), reference(layer, x, prob, mask, None, coef, ent))


def test_uniform_load_gives_the_coefficients():
    """Every expert once per 8 tokens, probabilities 1/8: loss = coef + ent log(1/8),
    no gradient but rounding."""
    layer = make_layer(8, 64, False, 64)
    prob = torch.full((64, 8), 0.125, device="cuda")
    mask = (torch.ones(64, dtype=torch.int64) << (torch.arange(64) % 8)).cuda()
    got = call(layer, make_x(64, 64, False), prob, mask, None, 0.5, 0.25)
    assert abs(got["loss"].item() - (0.5 + 0.25 * np.log(0.125))) < 1e-7
    assert (got["count"] == 8).all() and got["dlogits"].abs().max() <= 2.0 ** -24


def test_gradients_against_differences():
    """Central differences of the 64-bit loss through the softmax, over x and
    the router weights, the counts held."""
    T, E, d = 150, 24, 64
    layer, x, prob, mask = routed(E, d, False, T)
    valid = make_valid(T, "some")
    got, ref = call(layer, x, prob, mask, valid), reference(layer, x, prob, mask, valid, 0.01, 0.002)
    f = ref["count"].double() / int(ref["count"].sum())

    def loss64(a, w):
        P = torch.softmax(a[valid] @ w.T, 1).mean(0)
        return 0.01 * E * (f * P).sum() + 0.002 * (P * P.log()).sum()

    g = torch.Generator(device="cuda").manual_seed(2)
    w = layer.w["w_router"]
    for name, t in (("dx", x), ("dw_router", w)):
        u = torch.randn(t.shape, generator=g, device="cuda", dtype=torch.float64)
        e = 1e-4
        at = lambda s: (x.double() + s * u, w.double()) if name == "dx" else (x.double(), w.double() + s * u)
        slope = (loss64(*at(e)) - loss64(*at(-e))) / (2 * e)
        mine = (got[name].double() * u).sum()
        # prob is the fp32 softmax of fp32 scores: 1e-5 relative on p (the routing tests' 2e-5 on p)
        bound = (ref["bounds"][name] * u.abs()).sum() + 1e-4 * slope.abs() + 1e-7
        assert (mine - slope).abs() <= bound, (name, float(mine), float(slope))


@pytest.mark.parametrize("T,E,d,bf16", [(40, 8, 192, True), (500, 128, 192, True), (2200, 128, 512, True), (2200, 128, 512, False),
                                         (4300, 128, 1024, True), (4100, 128, 4160, False)])
def test_every_choice_of_outputs_and_aliases(T, E, d, bf16):
    layer, x, prob, mask = routed(E, d, bf16, T)
    valid = make_valid(T, "some")
    full = call(layer, x, prob, mask, valid)
    for bits in range(8):
        part = call(layer, x, prob, mask, valid, dz=bits & 1, dx=bits & 2, dw=bits & 4)
        for k in part:
            assert torch.equal(part[k], full[k]), (bits, k)
    pc, xc = prob.clone(), x.clone()
    layer.balance_loss(xc, pc, mask, valid, 0.01, 0.002, dlogits=pc, dx=xc)
    assert torch.equal(pc, full["dlogits"]) and torch.equal(xc, full["dx"])
    L.eat_balance_loss(layer.handle, None, T, layer.w["w_router"], prob, mask, valid, 0.01, 0.002, full["loss"], None,
                       None, None, xc, None, layer._bws.buf, layer._bws.buf.numel())
    assert torch.equal(xc, full["dx"])


def test_empty_call():
    layer = make_layer(64, 128, True, 8)
    e = lambda *s, **k: torch.empty(*s, device="cuda", **k)
    dw = torch.full((64, 128), 3.0, device="cuda")
    loss, count, mean = layer.balance_loss(e(0, 128, dtype=torch.bfloat16), e(0, 64), e(0, dtype=torch.int64), dw_router=dw)
    assert loss.item() == 0 and (count == 0).all() and (mean == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("T,E,d", [(700, 60, 128), (2200, 128, 512), (4300, 128, 1024)])
def test_other_stream_and_graph_replays(T, E, d):
    layer, x, prob, mask = routed(E, d, True, T)
    valid = make_valid(T, "some")
    ref = call(layer, x, prob, mask, valid)
    out = {k: torch.empty_like(ref[k]) for k in ("dlogits", "dx", "dw_router")}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    loss, _, _ = layer.balance_loss(x, prob, mask, valid, 0.01, 0.002, stream=side, **out)
    side.synchronize()
    assert torch.equal(loss, ref["loss"]) and all(torch.equal(out[k], ref[k]) for k in out)
    box = {}

    def step():
        m, _, _, p = layer.route(x)
        box["mask"], box["prob"] = m, p
        box["res"] = layer.balance_loss(x, p, m, valid, 0.01, 0.002, **out)

    g = capture(step)
    for seed, kind in ((1, "some"), (2, "none"), (3, "tail"), (1, "some")):
        x.copy_(make_x(T, d, True, seed))
        valid.copy_(make_valid(T, kind, seed))
        g.replay()
        torch.cuda.synchronize()
        mask, _, _, prob = layer.route(x)
        ref = call(layer, x, prob, mask, valid)
        assert torch.equal(box["res"][0], ref["loss"]) and torch.equal(box["res"][1], ref["count"])
        for k in out:
            assert torch.equal(out[k], ref[k]), (seed, k)


def test_workspace_is_not_given_away_while_another_stream_uses_it():
    layer, x, prob, mask = routed(60, 128, True, 700)
    ref = call(layer, x, prob, mask, None)
    side = torch.cuda.Stream()
    at, size = layer._bws.buf.data_ptr(), layer._bws.buf.numel()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
        loss, count, mean = layer.balance_loss(x, prob, mask, None, 0.01, 0.002)
    layer.close()
    del layer
    fill = [torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(3)]
    assert all(f.data_ptr() != at for f in fill)
    torch.cuda.synchronize()
    assert torch.equal(loss, ref["loss"]) and torch.equal(count, ref["count"]) and torch.equal(mean, ref["mean"])


def test_owner_refuses_what_it_would_misread():
    layer, x, prob, mask = routed(60, 128, True, 20)
    for kw in (dict(x=x.float()), dict(prob=prob.double()), dict(mask=mask.to(torch.int32)), dict(mask=mask[:19]),
               dict(valid=torch.ones(20, device="cuda")), dict(dlogits=torch.empty(20, 61, device="cuda")),
               dict(dw_router=torch.empty(60, 128, dtype=torch.bfloat16, device="cuda")),
               dict(x=x[:, :64]), dict(x=x.cpu()), dict(mask=mask.cpu()), dict(valid=torch.ones(20, dtype=torch.bool)),
               dict(dx=torch.empty(20, 128, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            layer.balance_loss(**(dict(x=x, prob=prob, mask=mask) | kw))
