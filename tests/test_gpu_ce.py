"""The LM head's cross entropy and its gradients (eat_ce_loss) against the
formulas in 64 bits.

Bounds.  A logit is an fp32 sum of d products of bf16 values: off by at most
eps_z = d 2^-24 max_v sum |h w|, and its exponent's argument by a few 2^-24
|z| more.  The NLL is log(1 + R) of the other logits' distance to the target's
(taken in fp64): off by (1 - p_y) times the rest's error, V-term sums in fp32
trees adding 2^-24 per level (under 100 levels), and one rounding to fp32.  G
is off by those of two logits (its own and the denominator), relative, and two
roundings (the exponential as it is kept, then times its row's factor): to bf16,
2^-8 each, or in calls of up to 64 positions to two bf16 parts, 2^-16 each; a product of K terms in fp32 by K 2^-24 of the sum of
absolute terms; the output by one rounding to bf16."""
import numpy as np
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import CrossEntropy, capture
from tests import parity as PT

pytestmark = pytest.mark.gpu

IGN = -100


def make(T, d, V, seed=0, ignored=None, lift=8.0):
    """Hidden rows, head and targets; `ignored`: share, or a list of positions."""
    g = torch.Generator().manual_seed(1000 * seed + T + 7 * d + 13 * V)
    h = torch.randn(T, d, generator=g)
    w = (torch.randn(V, d, generator=g) * d ** -0.5).to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=g)
    h = (h + lift * torch.rand(T, 1, generator=g) * w[y].float()).to(torch.bfloat16)
    y = y.to(torch.int32)
    if isinstance(ignored, float):
        y[torch.rand(T, generator=g) < ignored] = IGN
    elif ignored is not None:
        y[ignored] = IGN
    return h.cuda(), w.cuda(), y.cuda()


def call(h, w, y, mean=True, scale=1.0, dh=True, dw=True, ignore=IGN, guard=512, poison=True, most=None):
    """One call with its outputs inside larger buffers that must keep their
    surroundings, and a workspace full of NaN patterns."""
    ce = CrossEntropy(w, ignore=ignore, max_workspace=most)
    T = h.shape[0]

    def out(shape, dtype):
        n = int(np.prod(shape))
        buf = torch.full((n + 2 * guard,), 7.0 if dtype.is_floating_point else 7, dtype=dtype, device="cuda")
        return buf, buf[guard:guard + n].view(*shape)

    bufs = {"nll": out((T,), torch.float32), "count": out((1,), torch.int32)}
    if dh:
        bufs["dh"] = out(h.shape, torch.bfloat16)
    if dw:
        bufs["dw"] = out(w.shape, torch.bfloat16)
    for buf, view in bufs.values():
        view.fill_(-3)
    ws = ce.workspace(T, (L.EAT_CE_DH if dh else 0) | (L.EAT_CE_DW if dw else 0))
    if poison:
        ws.fill_(0xFF)
    views = {k: v for k, (_, v) in bufs.items()}
    loss = ce.loss(h, y, mean=mean, scale=scale, **views)
    torch.cuda.synchronize()
    for k, (buf, _) in bufs.items():
        assert (buf[:guard] == 7).all() and (buf[-guard:] == 7).all(), f"{k}: written outside"
    return {"loss": loss, **views}


def reference(h, w, y, mean, scale, ignore=IGN):
    rows = (y != ignore).nonzero()[:, 0]
    a, wd, t = h[rows].double(), w.double(), y[rows].long()[:, None]
    z = a @ wd.T
    zy = z.gather(1, t)
    rest = torch.logsumexp(z.scatter(1, t, -np.inf), 1, keepdim=True) - zy
    nll = torch.logaddexp(rest, torch.zeros_like(rest))
    n = rows.numel()
    c = scale / (max(n, 1) if mean else 1)
    G = torch.exp(z - zy - nll).scatter(1, t, torch.expm1(-nll))
    T = h.shape[0]
    full = torch.zeros(T, dtype=torch.float64, device=h.device)
    full[rows] = nll[:, 0]
    dh = torch.zeros(h.shape, dtype=torch.float64, device=h.device)
    dh[rows] = c * (G @ wd)
    ref = {"loss": c * nll.sum(), "nll": full, "dh": dh, "dw": c * (G.T @ a), "n": n}
    # bounds (module docstring)
    d, V = h.shape[1], w.shape[0]
    u = 2.0 ** -24
    if n:
        eps = d * u * (a.abs() @ wd.abs().T).max(1, keepdim=True).values + u * (120 + 8 * z.abs().max(1, keepdim=True).values)
    else:
        eps = torch.zeros(0, 1, dtype=torch.float64, device=h.device)
    bn = torch.zeros(T, dtype=torch.float64, device=h.device)
    bn[rows] = (-torch.expm1(-nll) * eps * (1 + eps) + u * nll + 2.0 ** -140)[:, 0]
    step = 2.0 ** -16 if T <= 64 else 2.0 ** -8
    eg = 2 * step + step * step + 2.02 * eps
    bh = torch.zeros_like(dh)
    ga = G.abs()
    bh[rows] = abs(c) * ((ga * (eg + 2 * V * u)) @ wd.abs())
    bw = abs(c) * ((ga * (eg + 2 * n * u)).T @ a.abs())
    half = 2.0 ** -8
    tiny = 2.0 ** -126                         # a flushed denormal
    ref["bounds"] = {"loss": abs(c) * bn.sum() + 2 * u * abs(ref["loss"]), "nll": bn,
                     "dh": bh * (1 + half) + half * dh.abs() + tiny, "dw": bw * (1 + half) + half * ref["dw"].abs() + tiny}
    return ref


def check(name, got, ref):
    assert int(got["count"]) == ref["n"]
    for k, b in ref["bounds"].items():
        if k not in got:
            continue
        err = (got[k].double().reshape(ref[k].shape) - ref[k]).abs()
        worst = float((err / b.clamp(min=1e-300)).max()) if err.numel() else 0.0
        PT.report(f"{name} {k}", err_over_bound=f"{worst:.2f}")
        assert (err <= b).all(), f"{name}: {k} off by {worst:.2f} of its bound"


SHAPES = [  # T, d, V
    (1, 64, 1), (1, 64, 2), (2, 64, 63), (1, 512, 4099), (3, 128, 64), (31, 192, 65), (63, 64, 127), (64, 320, 1000),
    (65, 64, 129), (100, 128, 255), (255, 64, 256), (256, 192, 257), (257, 320, 513), (300, 64, 1), (513, 512, 1000),
    (700, 1088, 771), (1025, 256, 2050), (2000, 128, 300), (40, 2048, 5003),
]


@pytest.mark.parametrize("T,d,V", SHAPES)
def test_loss_and_gradients(T, d, V):
    h, w, y = make(T, d, V)
    check(f"ce {T} {d} {V}", call(h, w, y), reference(h, w, y, True, 1.0))


@pytest.mark.parametrize("T,d,V", [(1, 64, 100), (64, 128, 300), (65, 128, 300), (600, 320, 777)])
@pytest.mark.parametrize("ignored", ["none", "some", "most", "first", "last", "all"])
def test_positions_that_do_not_count(T, d, V, ignored):
    which = {"none": None, "some": 0.3, "most": 0.97, "first": [0], "last": [T - 1], "all": list(range(T))}[ignored]
    h, w, y = make(T, d, V, seed=3, ignored=which)
    got, ref = call(h, w, y, mean=False, scale=0.25), reference(h, w, y, False, 0.25)
    check(f"ce {ignored} {T}", got, ref)
    off = y == IGN
    assert (got["nll"][off] == 0).all() and (got["dh"][off] == 0).all()
    if ref["n"] == 0:
        assert got["loss"].item() == 0 and (got["dw"] == 0).all()
    # whatever the rows that do not count hold, nothing changes
    bad = h.clone()
    bad[off] = float("nan")
    bad[off, ::3] = float("inf")
    again = call(bad, w, y, mean=False, scale=0.25)
    for k in got:
        assert torch.equal(got[k], again[k]), k


@pytest.mark.parametrize("T", [40, 300])
def test_every_choice_of_outputs_is_the_same_call(T):
    h, w, y = make(T, 256, 1100, ignored=0.2)
    full = call(h, w, y)
    for dh in (True, False):
        for dw in (True, False):
            part = call(h, w, y, dh=dh, dw=dw)
            for k in part:
                assert torch.equal(part[k], full[k]), (dh, dw, k)
    bare = CrossEntropy(w).loss(h, y)
    assert torch.equal(bare, full["loss"])


@pytest.mark.parametrize("T,scale,mean", [(50, -2.0, True), (300, 0.0, True), (300, 1e-3, False), (300, 1024.0, False)])
def test_scale_and_mean(T, scale, mean):
    h, w, y = make(T, 128, 500, ignored=0.2)
    check(f"ce scale {scale}", call(h, w, y, mean=mean, scale=scale), reference(h, w, y, mean, scale))


def test_ignored_target_inside_the_vocabulary():
    h, w, y = make(200, 128, 300)
    y[::3] = 5
    check("ce ignore 5", call(h, w, y, ignore=5), reference(h, w, y, True, 1.0, ignore=5))


@pytest.mark.parametrize("T,d,V", [(20, 128, 900), (330, 192, 1300)])
def test_confident_and_repeated_targets(T, d, V):
    """Targets up to 45 above the rest (G at the target is -(1 - p), down to
    1e-19), and one target shared by many rows."""
    g = torch.Generator().manual_seed(T)
    h = torch.randn(T, d, generator=g).to(torch.bfloat16)
    w = (torch.randn(V, d, generator=g) * d ** -0.5).to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=g)
    y[T // 2:] = V - 1
    lift = torch.linspace(0.0, 45.0, T)[:, None]
    hf = h.float()
    w[y] = (w[y].float() + lift * hf / hf.square().sum(1, keepdim=True)).to(torch.bfloat16)
    h, w, y = h.cuda(), w.cuda(), y.to(torch.int32).cuda()
    check(f"ce confident {T}", call(h, w, y), reference(h, w, y, True, 1.0))


@pytest.mark.parametrize("T,V", [(40, 4096 * 2 + 33), (300, 4096 * 4 + 1), (300, 4097), (300, 4096 * 3)])
def test_several_pieces_of_the_vocabulary(T, V):
    """The smallest workspace (pieces of 4096 entries), one between, and the
    largest: the loss is the same bits, the gradients within the same bound."""
    d = 192
    h, w, y = make(T, d, V, ignored=0.1)
    y[:5] = torch.tensor([0, V - 1, 4095, 4096, IGN], dtype=torch.int32)
    ref = reference(h, w, y, True, 1.0)
    full = call(h, w, y)
    most, least = L.eat_ce_workspace_size(T, d, V, 3)
    assert least < most
    for size in (0, (least + most) // 2, most):
        got = call(h, w, y, most=size)
        check(f"ce pieces {T} {V} {size}", got, ref)
        assert torch.equal(got["loss"], full["loss"]) and torch.equal(got["nll"], full["nll"])
        again = call(h, w, y, most=size)
        assert torch.equal(got["dh"], again["dh"]) and torch.equal(got["dw"], again["dw"])
        for kw in (dict(dh=False), dict(dw=False)):
            check(f"ce pieces {T} {V} {size} {kw}", call(h, w, y, most=size, **kw), ref)


@pytest.mark.parametrize("T", [1, 2, 5])
@pytest.mark.parametrize("lift", [0.0, 3.0, 9.0])
def test_few_rows_keep_the_outputs_precision(T, lift):
    """One entry of G can be a whole gradient row: with few rows nothing averages
    its rounding.  The gradients' error over their norm stays that of the
    outputs' own rounding (2^-8 at most, plus the parts' 2^-15)."""
    for seed in range(6):
        h, w, y = make(T, 256, 1500, seed=seed, lift=lift)
        wrong = torch.randint(0, 1500, (T,), device="cuda")
        h = (h.float() + 12.0 * w[wrong].float()).to(torch.bfloat16)       # confident of something else
        got, ref = call(h, w, y), reference(h, w, y, True, 1.0)
        for k in ("dh", "dw"):
            err = (got[k].double() - ref[k]).norm() / ref[k].norm()
            assert err <= 2.0 ** -8 + 2.0 ** -14, (seed, k, float(err))


@pytest.mark.parametrize("T", [48, 320])
def test_unknown_targets_and_nonfinite_rows(T):
    d, V = 128, 700
    h, w, y = make(T, d, V)
    clean = call(h, w, y)
    for target in (-1, V, V + 5000, 2 ** 31 - 1, -2 ** 31):
        yb = y.clone()
        yb[7] = target
        got = call(h, w, yb)
        keep = torch.arange(T, device="cuda") != 7
        assert torch.isnan(got["nll"][7]) and torch.isnan(got["loss"]).all()
        assert torch.equal(got["nll"][keep], clean["nll"][keep]) and torch.equal(got["dh"][keep], clean["dh"][keep])
        assert torch.isnan(got["dh"][7]).all() and torch.isnan(got["dw"]).all()
    hb = h.clone()
    hb[9, 3] = float("nan")
    got = call(hb, w, y)
    keep = torch.arange(T, device="cuda") != 9
    assert torch.isnan(got["nll"][9]) and torch.equal(got["nll"][keep], clean["nll"][keep])
    assert torch.equal(got["dh"][keep], clean["dh"][keep]) and torch.isnan(got["dw"]).all()


def test_head_rows_of_minus_infinity_take_no_probability():
    """A vocabulary's unused entries switched off by -inf logits (h[:, 0] = 1
    picks the head's first column)."""
    T, d, V = 70, 128, 600
    h, w, y = make(T, d, V)
    h[:, 0] = 1.0
    off = torch.tensor([3, 255, 256, 511, V - 1], device="cuda")
    for s in range(T):
        while int(y[s]) in off.tolist():
            y[s] = (int(y[s]) + 1) % V
    w[off, 0] = -float("inf")
    got = call(h, w, y, dh=False)
    keep = torch.ones(V, dtype=torch.bool, device="cuda")
    keep[off] = False
    renum = torch.cumsum(keep, 0) - 1
    ref = reference(h, w[keep], renum[y.long()].to(torch.int32), True, 1.0)
    check("ce -inf", {"loss": got["loss"], "nll": got["nll"], "count": got["count"], "dw": got["dw"][keep]}, ref)
    assert (got["dw"][off] == 0).all()


@pytest.mark.parametrize("T", [33, 290])
def test_gradients_against_differences(T):
    """<dh, u> and <dW, u> against central differences of the 64-bit loss along
    u: the step's third-order term is under 1e-6 of the slope, the rest is the
    gradients' own bound."""
    d, V = 128, 400
    h, w, y = make(T, d, V, ignored=0.1)
    got, ref = call(h, w, y), reference(h, w, y, True, 1.0)
    g = torch.Generator(device="cuda").manual_seed(5)

    def loss64(a, b):
        rows = (y != IGN).nonzero()[:, 0]
        z = a[rows] @ b.T
        return (torch.logsumexp(z, 1) - z.gather(1, y[rows].long()[:, None])[:, 0]).mean()

    for name, x in (("dh", h), ("dw", w)):
        u = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64)
        e = 1e-4
        args = lambda s: (h.double() + s * u, w.double()) if name == "dh" else (h.double(), w.double() + s * u)
        slope = (loss64(*args(e)) - loss64(*args(-e))) / (2 * e)
        mine = (got[name].double() * u).sum()
        bound = (ref["bounds"][name] * u.abs()).sum() + 1e-6 * slope.abs() + 1e-9
        assert (mine - slope).abs() <= bound, (name, float(mine), float(slope))


@pytest.mark.parametrize("T", [5, 64, 300])
def test_runs_are_bit_equal_and_dh_may_be_h(T):
    h, w, y = make(T, 256, 900, ignored=0.2)
    a, b = call(h, w, y), call(h, w, y, poison=False)
    for k in a:
        assert torch.equal(a[k], b[k]), k
    x = h.clone()
    CrossEntropy(w).loss(x, y, dh=x)
    assert torch.equal(x, a["dh"])


def test_empty_call():
    h, w, y = make(4, 128, 300)
    got = call(h[:0], w, y[:0])
    assert got["loss"].item() == 0 and int(got["count"]) == 0 and (got["dw"] == 0).all()


def test_one_object_over_growing_and_shrinking_calls():
    """One workspace, calls of many sizes in turn (what one call leaves in it
    is the next one's)."""
    h, w, y = make(700, 192, 1500, ignored=0.2)
    ce = CrossEntropy(w)
    for T in (700, 3, 65, 512, 1, 300):
        dh, dw = torch.empty_like(h[:T]), torch.empty_like(w)
        loss = ce.loss(h[:T], y[:T], dh=dh, dw=dw)
        ref = call(h[:T], w, y[:T])
        assert torch.equal(loss, ref["loss"]) and torch.equal(dh, ref["dh"]) and torch.equal(dw, ref["dw"]), T


def test_other_stream():
    h, w, y = make(300, 192, 1500, ignored=0.2)
    ref = call(h, w, y)
    ce = CrossEntropy(w)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    ce.loss(h, y, dh=dh, dw=dw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dh.zero_()
    side.wait_stream(torch.cuda.current_stream())
    loss = ce.loss(h, y, dh=dh, dw=dw, stream=side)
    side.synchronize()
    assert torch.equal(loss, ref["loss"]) and torch.equal(dh, ref["dh"]) and torch.equal(dw, ref["dw"])


@pytest.mark.parametrize("T", [40, 300])
def test_graph_replays(T):
    """A captured call replayed over new inputs (another number of counted
    positions among them), eager work between the replays."""
    d, V = 192, 1200
    h, w, y = make(T, d, V)
    ce = CrossEntropy(w)
    out = {"nll": torch.empty(T, device="cuda"), "count": torch.empty(1, dtype=torch.int32, device="cuda"),
           "dh": torch.empty_like(h), "dw": torch.empty_like(w)}
    box = {}

    def step():
        box["loss"] = ce.loss(h, y, **out)

    g = capture(step)
    for seed, ignored in ((1, None), (2, 0.5), (3, list(range(T))), (4, 0.1), (2, 0.5)):
        hn, _, yn = make(T, d, V, seed=seed, ignored=ignored)
        h.copy_(hn)
        y.copy_(yn)
        g.replay()
        torch.cuda.synchronize()
        ref = call(hn, w, yn)
        assert torch.equal(box["loss"], ref["loss"])
        for k in out:
            assert torch.equal(out[k], ref[k]), (seed, k)


def test_graph_outlives_its_workspace():
    """A graph captured with a small workspace is replayed after a larger call
    gave the object another one (and other tensors took the memory it freed)."""
    h, w, y = make(900, 192, 1200, ignored=0.2)
    ce = CrossEntropy(w)
    hs, ys = h[:100].clone(), y[:100].clone()
    dh, dw = torch.empty_like(hs), torch.empty_like(w)
    box = {}
    g = capture(lambda: box.update(loss=ce.loss(hs, ys, dh=dh, dw=dw)))
    small = ce._ws.buf.numel()
    ce.loss(h, y, dh=torch.empty_like(h), dw=torch.empty_like(w))
    assert ce._ws.buf.numel() > small
    fill = [torch.full((small,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(4)]
    ref = call(hs, w, ys)
    for _ in range(3):
        dh.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(box["loss"], ref["loss"]) and torch.equal(dh, ref["dh"]) and torch.equal(dw, ref["dw"])
    assert all((f == 0xFF).all() for f in fill)


def test_workspace_is_not_given_away_while_another_stream_uses_it():
    """Made on one stream, used on another (the current one, or one given) that
    is still busy when its owner goes: new tensors do not get its memory."""
    h, w, y = make(500, 128, 3000)
    ref = call(h, w, y, dw=False)
    side = torch.cuda.Stream()
    for given in (False, True, "address"):
        ce, dh = CrossEntropy(w), torch.empty_like(h)
        ce.loss(h, y, dh=dh)
        at, size = ce._ws.buf.data_ptr(), ce._ws.buf.numel()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
            if not given:
                loss = ce.loss(h, y, dh=dh)
        if given:
            loss = ce.loss(h, y, dh=dh, stream=side if given is True else side.cuda_stream)
        del ce
        fill = [torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(3)]
        assert all(f.data_ptr() != at for f in fill)
        torch.cuda.synchronize()
        assert torch.equal(loss, ref["loss"]) and torch.equal(dh, ref["dh"])


def test_the_nll_is_the_perplexity_signals():
    """eat_ppl_trend's NLL of the same rows: both are within the NLL's bound."""
    from paper_2609_33614_amd.layer import PplSignal
    h, w, y = make(64, 512, 2048)
    sig = PplSignal(64, w)
    sig.step(h, y)
    got, ref = call(h, w, y, dh=False, dw=False), reference(h, w, y, True, 1.0)
    b = ref["bounds"]["nll"]
    assert ((sig.nll.double() - ref["nll"]).abs() <= b).all() and ((got["nll"] - sig.nll).double().abs() <= 2 * b).all()


def test_owner_refuses_what_it_would_misread():
    h, w, y = make(8, 128, 300)
    ce = CrossEntropy(w)
    for kw in (dict(h=h.float()), dict(target=y.long()), dict(h=h[:, :64]), dict(target=y[:7]),
               dict(dh=torch.empty_like(h).float()), dict(dw=torch.empty(300, 64, dtype=torch.bfloat16, device="cuda")),
               dict(h=h.t().contiguous().t()), dict(nll=torch.empty(7, device="cuda")), dict(target=y.cpu()), dict(h=h.cpu()),
               dict(dw=torch.empty_like(w, device="cpu"))):
        args = dict(h=h, target=y) | kw
        with pytest.raises(ValueError):
            ce.loss(**args)
