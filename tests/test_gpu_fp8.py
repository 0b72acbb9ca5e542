"""Products and experts in 8 bits (Fp8Matrix, Fp8Experts) against 64 bits."""
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import Fp8Experts, Fp8Matrix, capture
from tests import fp8_reference as R
from tests import parity as PT

pytestmark = pytest.mark.gpu

U, TINY = R.U, R.TINY
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


def normal(*s, seed=0, std=1.0, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed + sum(s))
    return (std * torch.randn(*s, generator=g)).to(dtype).cuda()


def rows_of(n, K, seed=0):
    """Rows whose blocks differ by orders of magnitude, some columns large, some rows and blocks zero."""
    g = torch.Generator().manual_seed(seed + 7 * n + K)
    x = torch.randn(n, K, generator=g)
    x *= torch.exp2(torch.randint(-12, 12, (n, -(-K // 128)), generator=g).float()).repeat_interleave(128, 1)[:, :K]
    x[:, torch.randint(0, K, (max(1, K // 100),), generator=g)] *= 16.0
    x[::5, : K // 2] = 0.0
    return x.to(torch.bfloat16).cuda()


def within(name, got, ref, bound):
    err = (got.double() - ref).abs()
    worst = float((err / bound).nan_to_num(0.0).max()) if err.numel() else 0.0
    PT.report(name, err_over_bound=f"{worst:.2f}")
    assert (err <= bound).all(), f"{name}: off by {worst:.2f} of its bound"


def unpadded(m, q, scale, rows, cols):
    """The values that q and scale hold."""
    s = torch.exp2(scale.double() - 127)[:, :, : -(-cols // 128)]
    full = q.double().view(q.shape[0], rows, -1, 128) * s.repeat_interleave(128, 1)[:, :rows, :, None]
    return full.view(q.shape[0], rows, -1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("G,M,K", [(1, 8, 8), (1, 128, 128), (3, 136, 264), (2, 640, 1000), (5, 64, 512), (256, 8, 136), (1, 1032, 2056)])
def test_weights_are_rounded_as_defined(G, M, K, dtype):
    w = normal(G, M, K, dtype=torch.float32) * torch.exp2(torch.randint(-40, 40, (G, M, K // 8), generator=torch.Generator().manual_seed(G)).float()).cuda().repeat_interleave(8, 2)
    w[0, :128, :128] = 0.0
    w = w.to(dtype)
    m = Fp8Matrix(w, gradients=True)
    want, k = R.quantize(w, 128)
    got = unpadded(m, m.q, m.scale, M, K)
    assert torch.equal(got[:, :, :K], want) and (got[:, :, K:] == 0).all()
    assert torch.equal(m.scale[:, :, : k.shape[-1]].int() - 127, k.int()) and (m.scale[:, :, k.shape[-1]:] == 127).all()
    back = unpadded(m, m.qt, m.scale_t, K, M)
    assert torch.equal(back[:, :, :M], want.transpose(1, 2)) and (back[:, :, M:] == 0).all()
    assert torch.equal(m.scale_t[:, :, : k.shape[1]].int() - 127, k.transpose(1, 2).int())


def test_ends_of_the_numbers():
    """Ties, the largest magnitude at and past 448 2^k, subnormal numbers and scales, NaN and infinities."""
    v = torch.zeros(128, 1024)
    v[0, :8] = torch.tensor([448.0, 1.0625, 1.1875, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 0.0293, -448.0])
    v[0, 128:134] = torch.tensor([449.0, 2.125, 2.375, 1e-3, -1.0, 0.5])
    v[1, 256:259] = torch.tensor([3.3e38, 1e30, -2.0 ** 127])
    v[2, 384:388] = torch.tensor([2.0 ** -133, 2.0 ** -149, -2.0 ** -130, 2.0 ** -126])
    v[3, 512:516] = torch.tensor([float("nan"), float("inf"), -float("inf"), 7.0])
    v[4, 640:642] = torch.tensor([447.99997, -448.00003])
    m = Fp8Matrix(v.cuda())
    want, k = R.quantize(v, 128)
    got = unpadded(m, m.q, m.scale, 128, 1024)[0].cpu()
    assert torch.equal(torch.nan_to_num(got, 5.0), torch.nan_to_num(want, 5.0)) and torch.equal(got.isnan(), want.isnan())
    assert torch.equal(m.scale[0, :, :8].int().cpu() - 127, k.int())


PRODUCTS = [(1, 8, 8, 1, "even"), (1, 64, 64, 1, "even"), (3, 128, 256, 1, "even"), (32, 136, 264, 1, "even"), (33, 512, 128, 1, "even"),
            (100, 1000, 520, 1, "even"), (161, 72, 1032, 1, "even"), (300, 640, 256, 1, "even"), (500, 4096, 512, 1, "even"),
            (1, 8192, 256, 1, "even"), (37, 4096, 520, 1, "even"), (2, 64, 64, 4, "one"), (74, 512, 384, 8, "skewed"),
            (500, 256, 264, 60, "skewed"), (2000, 1408, 192, 60, "skewed"), (5003, 192, 320, 7, "skewed"), (700, 128, 128, 256, "skewed"),
            (300, 2048, 136, 3, "inside"), (900, 384, 512, 30, "inside"), (4000, 1024, 264, 5, "inside"), (90, 640, 128, 128, "one"),
            (3000, 392, 1544, 8, "even"), (257, 128, 2048, 1, "even"), (1030, 256, 4104, 2, "skewed")]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,K,M,G,kind", PRODUCTS)
def test_product_and_its_gradient(n, K, M, G, kind, dtype):
    w, x, dy = normal(G, M, K, std=K ** -0.5), rows_of(n, K), rows_of(n, M, 3)
    off = R.sizes(n, G, kind)
    m = Fp8Matrix(w, gradients=True)
    o32 = None if G == 1 and kind == "even" else off.int().cuda()
    out, dx = (torch.full((n, c), 7.0, dtype=dtype, device="cuda") for c in (M, K))
    assert m.product(x, o32, out=out) is out and m.product_backward(dy, o32, dx=dx) is dx
    wq, _ = R.quantize(w, 128)
    inside = torch.zeros(n, dtype=torch.bool)
    inside[int(off[0]): int(off[-1])] = True
    for name, got, src, mat in (("y", out, x, wq), ("dx", dx, dy, wq.transpose(1, 2))):
        ref, bound, var = R.grouped(R.quantize(src)[0], mat, off, exact=dtype == torch.float32)
        h = HALF[dtype]
        within(f"fp8 {name} {n} {K} {M} {G}", got[inside], ref[inside], ((1 + h) * bound + h * ref.abs() + TINY)[inside])
        if dtype == torch.bfloat16 and n * M >= 1000:      # the whole's error, the cuts and roundings adding up as squares
            assert (got[inside].double() - ref[inside]).square().sum() <= (var + (h * ref).square())[inside].sum()
        assert (got[~inside] == 7.0).all()
    again = m.product(x, o32, out=torch.full_like(out, 7.0))
    assert torch.equal(again, out)


@pytest.mark.parametrize("n,src,K,M,G", [(5, 1, 128, 128, 2), (300, 40, 512, 264, 8), (700, 900, 72, 128, 3), (3000, 500, 256, 512, 4)])
def test_product_of_gathered_rows(n, src, K, M, G):
    w, x = normal(G, M, K, std=K ** -0.5), rows_of(src, K)
    token = torch.randint(0, src, (n,), generator=torch.Generator().manual_seed(n))
    off = R.sizes(n, G, "skewed").int().cuda()
    m = Fp8Matrix(w)
    got = m.product(x, off, token=token.int().cuda())
    assert torch.equal(got, m.product(x[token.cuda()].contiguous(), off))
    # entries that are no rows are kept inside
    wild = token.int()
    wild[0], wild[n - 1] = -1, 2 ** 31 - 1
    held = token.clone()
    held[0] = held[n - 1] = src - 1
    assert torch.equal(m.product(x, off, token=wild.cuda()), m.product(x, off, token=held.int().cuda()))


def test_offsets_outside_the_rows_are_kept_inside():
    n, G = 200, 4
    w, x = normal(G, 128, 128), rows_of(n, 128)
    m = Fp8Matrix(w)
    for bad, good in (([-5, 50, 120, 10 ** 9, 2 ** 31 - 1], [0, 50, 120, 200, 200]), ([0, 300, 300, 300, 300], [0, 200, 200, 200, 200])):
        a, b = (m.product(x, torch.tensor(o, dtype=torch.int32).cuda()) for o in (bad, good))
        assert torch.equal(a, b)
    # a group that ends before it begins has no rows
    out = torch.full((n, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    m.product(x, torch.tensor([0, 100, 60, 60, 60], dtype=torch.int32).cuda(), out=out)
    assert (out[100:] == 7.0).all()


@pytest.mark.parametrize("n", [40, 300, 2000])
def test_what_is_not_finite_stays_where_it_is(n):
    K, M, G = 640, 264, 4
    w, x = normal(G, M, K), rows_of(n, K)
    off = R.sizes(n, G, "even").int().cuda()
    want = Fp8Matrix(w).product(x, off)
    x2, w2 = x.clone(), w.clone()
    x2[3, 500], x2[7, 1], x2[n - 1, 639] = float("nan"), float("inf"), -float("inf")
    w2[1, 17, 3] = float("nan")
    got = Fp8Matrix(w2).product(x2, off)
    bad = torch.zeros(n, M, dtype=torch.bool, device="cuda")
    bad[3] = bad[7] = bad[n - 1] = True
    bad[int(off[1]):int(off[2]), 17] = True
    assert got[bad].isnan().all() and torch.equal(got[~bad], want[~bad])


def test_no_rows():
    m = Fp8Matrix(normal(3, 64, 128), gradients=True)
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert m.product(rows_of(0, 128) if False else torch.empty(0, 128, dtype=torch.bfloat16, device="cuda"), off).shape == (0, 64)
    out = torch.full((5, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    m.product(normal(5, 128), off, out=out)
    assert (out == 7.0).all()


# ---- experts -----------------------------------------------------------------

def experts_reference(x, w, off, token):
    """y with its bound and the square of what its errors come to where they are independent, and g, u with their bound."""
    F = w["w1"].shape[1]
    w1, w3, w2 = (R.quantize(w[k], 128)[0] for k in ("w1", "w3", "w2"))
    xq = R.quantize(x)[0][token]
    (g, eg, _), (u, eu, _) = R.grouped(xq, w1, off, exact=True), R.grouped(xq, w3, off, exact=True)
    g, u = g.nan_to_num(0.0), u.nan_to_num(0.0)
    sg = g * torch.sigmoid(g)
    h = sg * u
    # silu's slope is at most 1.1; its own arithmetic is within (|g| + 8) 2^-23 of itself
    own = (g.abs() + 8) * 2 * U * h.abs() + 2.0 ** -100
    hq, he = R.quantize_between(h, 1.1 * eg * (u.abs() + eu) + sg.abs() * eu + own)
    y, ey, vy = R.grouped(hq, w2, off, he)
    vy = vy + R.grouped(he.square(), w2.square(), off)[0] + (2.0 ** -8 * y).square()
    return (y, (1 + 2.0 ** -8) * ey + 2.0 ** -8 * y.abs() + TINY, vy), (torch.cat([g, u], 1), torch.cat([eg, eu], 1))


def backward_reference(dy, saved, w, off):
    F = w["w1"].shape[1]
    w1, w3, w2 = (R.quantize(w[k], 128)[0] for k in ("w1", "w3", "w2"))
    dh, eh, _ = R.grouped(R.quantize(dy)[0], w2.transpose(1, 2), off, exact=True)
    dh = dh.nan_to_num(0.0)
    g, u = saved.double().split(F, 1)
    s = torch.sigmoid(g)
    slope = 1 + g * (1 - s)
    dg, du = dh * u * s * slope, dh * g * s
    rel = (g.abs() + 10) * 2 * U                          # of s, 1 - s and the products
    og, ou = (dh * u * s).abs() * (1 + g.abs()) * 2 * rel + 2.0 ** -100, du.abs() * 2 * rel + 2.0 ** -100
    ag, au = (u * s * slope).abs(), (g * s).abs()
    (gq, ge), (uq, ue) = R.quantize_between(dg, eh * ag + og), R.quantize_between(du, eh * au + ou)
    a, b = R.grouped(gq, w1.transpose(1, 2), off, ge), R.grouped(uq, w3.transpose(1, 2), off, ue)
    dx = a[0] + b[0]
    var = a[2] + b[2] + R.grouped(ge.square(), w1.transpose(1, 2).square(), off)[0] + R.grouped(ue.square(), w3.transpose(1, 2).square(), off)[0]
    # (one sum over both products)
    return dx, (1 + 2.0 ** -8) * 2 * (a[1] + b[1]) + 2.0 ** -8 * dx.abs() + TINY, var + (2.0 ** -8 * dx).square()


def make_experts(T, d, F, E, k, kind="skewed", seed=0):
    w = {"w1": normal(E, F, d, std=d ** -0.5, seed=seed), "w3": normal(E, F, d, std=d ** -0.5, seed=seed + 1), "w2": normal(E, d, F, std=F ** -0.5, seed=seed + 2)}
    n = T * k
    off = R.sizes(n, E, kind)
    token = torch.randint(0, T, (n,), generator=torch.Generator().manual_seed(n))
    return w, normal(T, d, seed=seed + 3), off, token


EXPERTS = [(1, 64, 64, 1, 1, "even"), (1, 128, 256, 8, 2, "skewed"), (1, 1024, 1024, 8, 2, "skewed"), (3, 192, 320, 4, 2, "one"),
           (37, 512, 704, 8, 2, "skewed"), (64, 256, 128, 128, 8, "skewed"), (100, 128, 832, 60, 4, "inside"), (200, 576, 192, 3, 2, "skewed"),
           (500, 256, 448, 7, 1, "even"), (1500, 384, 256, 16, 2, "skewed"), (900, 512, 512, 2, 2, "even"), (20, 2048, 128, 2, 1, "even"),
           (10, 128, 2048, 2, 1, "even")]


@pytest.mark.parametrize("T,d,F,E,k,kind", EXPERTS)
def test_experts_and_their_gradient(T, d, F, E, k, kind):
    w, x, off, token = make_experts(T, d, F, E, k, kind)
    n = T * k
    ex = Fp8Experts(w, gradients=True)
    o32, t32 = off.int().cuda(), token.int().cuda()
    y, saved, dx = (torch.full((n, c), 7.0, dtype=torch.bfloat16, device="cuda") for c in (d, 2 * F, d))
    ex.forward(x, o32, t32, y=y, saved=saved)
    (ry, by, vy), (rs, bs) = experts_reference(x, w, off, token.cuda())
    inside = torch.zeros(n, dtype=torch.bool)
    inside[int(off[0]): int(off[-1])] = True
    within(f"experts y {T} {d} {F} {E}", y[inside], ry[inside], by[inside])
    h = 2.0 ** -8
    within(f"experts saved {T} {d} {F} {E}", saved[inside], rs[inside], ((1 + h) * bs + h * rs.abs() + TINY)[inside])
    assert (y[~inside] == 7.0).all() and (saved[~inside] == 7.0).all()
    assert torch.equal(ex.forward(x, o32, t32)[inside], y[inside])
    dy = normal(n, d, seed=11, std=0.01)
    ex.backward(dy, saved, o32, dx=dx)
    rdx, bdx, vdx = backward_reference(dy, saved, w, off)
    within(f"experts dx {T} {d} {F} {E}", dx[inside], rdx[inside], bdx[inside])
    for name, got, ref, var in (("y", y, ry, vy), ("dx", dx, rdx, vdx)):
        if n * d >= 1000:
            share = ((got.double() - ref)[inside].square().sum() / var[inside].sum()).sqrt()
            PT.report(f"experts {name} {T} {d} {F} {E}", whole_error_over_expected=f"{float(share):.2f}")
            assert share <= 1
    assert (dx[~inside] == 7.0).all()
    in_place = dy.clone()
    ex.backward(in_place, saved, o32, dx=in_place)
    assert torch.equal(in_place[inside], dx[inside])
    assert torch.equal(Fp8Experts(w).forward(x, o32, t32)[inside], y[inside])


def test_experts_gradient_against_differences():
    """Central differences of the smooth function through the rounded weights: the gradient's own
    roundings (dy, dg and du to 4 bits: 2^-4 of each at most) bound the distance."""
    T, d, F, E = 24, 128, 256, 3
    w, x, off, token = make_experts(T, d, F, E, 1, "even")
    token = torch.arange(T)
    ex = Fp8Experts(w, gradients=True)
    saved = torch.empty(T, 2 * F, dtype=torch.bfloat16, device="cuda")
    ex.forward(x, off.int().cuda(), token.int().cuda(), saved=saved)
    dy = normal(T, d, seed=3)
    dx = ex.backward(dy, saved, off.int().cuda())
    w1, w3, w2 = (R.quantize(w[k], 128)[0] for k in ("w1", "w3", "w2"))
    xq = R.quantize(x)[0]

    def f(v):
        g, u = R.grouped(v, w1, off)[0], R.grouped(v, w3, off)[0]
        return (R.grouped(g * torch.sigmoid(g) * u, w2, off)[0] * dy.double()).sum()

    g, u = R.grouped(xq, w1, off)[0], R.grouped(xq, w3, off)[0]
    s = torch.sigmoid(g)
    q = 2.0 ** -4
    dh = R.grouped(dy.double().abs(), w2.transpose(1, 2).abs(), off)[0]
    # |dh| is at most (1 + q) of the sum of its terms' magnitudes; what rounding, g and u in bf16 (2^-8; |g| < 8, so that slopes move by less than 2^-4) do to dg and du
    room = 3 * q * R.grouped(dh * (u * s).abs() * (1 + g.abs()) + 2.0 ** -4 * dh, w1.transpose(1, 2).abs(), off)[0] \
        + 3 * q * R.grouped(dh * (g * s).abs() + 2.0 ** -4 * dh, w3.transpose(1, 2).abs(), off)[0]
    gen = torch.Generator(device="cuda").manual_seed(0)
    h = 1e-5
    for _ in range(4):
        v = torch.randn(T, d, dtype=torch.float64, device="cuda", generator=gen)
        slope = (f(xq + h * v) - f(xq - h * v)) / (2 * h)
        got = (dx.double() * v).sum()
        assert abs(float(got - slope)) <= float((room * v.abs()).sum()) + 1e-6
        # the roundings are independent: far inside that sum, at 2^-4 of what they add up to at random
        spread = float(((room * v) ** 2).sum().sqrt())
        assert abs(float(got - slope)) <= spread, (float(got), float(slope), spread)


def test_a_bad_row_stays_with_itself_through_the_experts():
    T, d, F, E = 300, 256, 384, 4
    w, x, off, token = make_experts(T, d, F, E, 1, "even")
    token = torch.arange(T).int().cuda()
    off = off.int().cuda()
    ex = Fp8Experts(w, gradients=True)
    saved = torch.empty(T, 2 * F, dtype=torch.bfloat16, device="cuda")
    want = ex.forward(x, off, token, saved=saved)
    x2 = x.clone()
    x2[5, 7], x2[200, 0] = float("nan"), float("inf")
    got = ex.forward(x2, off, token)
    keep = torch.ones(T, dtype=torch.bool)
    keep[5] = keep[200] = False
    assert torch.equal(got[keep], want[keep]) and got[~keep].isnan().all()
    dy = normal(T, d)
    a = ex.backward(dy, saved, off)
    dy2 = dy.clone()
    dy2[9, 9] = float("nan")
    b = ex.backward(dy2, saved, off)
    keep[:] = True
    keep[9] = False
    assert torch.equal(a[keep], b[keep]) and b[9].isnan().all()


@pytest.mark.parametrize("n", [20, 300, 2600])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ex,ew", [(-80, -60), (116, 18), (60, 60), (-120, 100), (100, -110), (10, -118)])
def test_scales_far_apart(n, dtype, ex, ew):
    """Powers of two whose sum no fp32 holds while the results are ordinary, and the other way round: weights
    2^-8 or 2^-14 of their block's largest, and zeros, where the largest would give infinity."""
    K, M = 640, 1032
    x, w = normal(n, K, std=1.0).float().clamp(-3, 3), normal(1, M, K, dtype=torch.float32).clamp(-3, 3)
    w[:, 1::2] *= 2.0 ** (-14 if ew == 18 else -8)
    w[:, 2::4] = 0.0
    if ew == 18:
        w[:, ::4] *= (torch.arange(K, device="cuda") == 5)            # (the largest alone in its rows)
        x[:, 5] = 0.0
        w[0, ::4, 5] = 3.0
    x, w = (x * 2.0 ** ex).to(torch.bfloat16), w * 2.0 ** ew
    m = Fp8Matrix(w)
    out = torch.full((n, M), 7.0, dtype=dtype, device="cuda")
    m.product(x, out=out)
    off = torch.tensor([0, n])
    xq, wq = R.quantize(x)[0], R.quantize(w, 128)[0]
    ref, bound, _ = R.grouped(xq, wq, off, exact=dtype == torch.float32)
    # numbers below 2^-126 may count as zeros, on either side and in the sums
    bound = bound + 2.0 ** -126 * (K + xq.abs().sum(1)[:, None] + wq[0].abs().sum(1)[None])
    if dtype == torch.bfloat16:
        bound = (1 + 2.0 ** -8) * bound + 2.0 ** -8 * ref.abs() + 2.0 ** -126
    assert ref.isfinite().all() and float(ref.abs().max()) < 2.0 ** 128 * (1 - 2.0 ** -7)   # (bf16 ends at 2^128 (1 - 2^-8))
    within(f"scales {n} {ex} {ew}", out, ref, bound)


def test_an_overflowing_h_is_not_a_number():
    """g and u finite, their product past fp32 (as an infinite h has no 8-bit number): NaN in the
    rows where it happens, in every kind of call; the others keep their bits."""
    d, F, E = 128, 256, 2
    for T in (1, 40, 300, 3000):
        w, x, off, token = make_experts(T, d, F, E, 1, "even")
        token = torch.arange(T).int().cuda()
        x = x.float().clamp(-4, 4)
        off = off.int().cuda()
        ex = Fp8Experts({"w1": w["w1"] * 2.0 ** 20, "w3": w["w3"] * 2.0 ** 60, "w2": w["w2"]})
        quiet = (x * 2.0 ** -30).to(torch.bfloat16)
        want = ex.forward(quiet, off, token)
        assert want.isfinite().all()
        loud = quiet.clone()
        loud[::3] *= 2.0 ** 80                        # g about 2^70, u about 2^110: h past 2^128
        got = ex.forward(loud, off, token)
        bad = torch.zeros(T, dtype=torch.bool, device="cuda")
        bad[::3] = True
        assert got[bad].isnan().all() and torch.equal(got[~bad], want[~bad])
        saved = torch.empty(T, 2 * F, dtype=torch.bfloat16, device="cuda")
        assert torch.equal(ex.forward(loud, off, token, saved=saved)[~bad], want[~bad]) and saved.isfinite().all()


@pytest.mark.parametrize("T,d,F,E", [(20, 256, 192, 2), (300, 256, 384, 4), (3000, 512, 256, 4)])
def test_an_overflowing_gradient_stays_in_its_row(T, d, F, E):
    """dh u past fp32 in every third row: NaN there, the others keep their bits."""
    w, x, off, token = make_experts(T, d, F, E, 1, "even")
    off, token = off.int().cuda(), torch.arange(T).int().cuda()
    ex = Fp8Experts(w, gradients=True)
    saved = torch.empty(T, 2 * F, dtype=torch.bfloat16, device="cuda")
    ex.forward(x, off, token, saved=saved)
    saved[:, F:] *= 2.0 ** 30
    dy = normal(T, d).float().clamp(-3, 3).to(torch.bfloat16)
    want = ex.backward(dy, saved, off)
    assert want.isfinite().all()
    loud = dy.clone()
    loud[::3] *= 2.0 ** 120
    got = ex.backward(loud, saved, off)
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[::3] = True
    assert got[bad].isnan().all() and torch.equal(got[~bad], want[~bad])


def test_streams_and_graphs():
    """Eager, on a named stream behind pending work, and captured and replayed over new inputs."""
    T, d, F, E, k = 60, 256, 320, 8, 2
    w, x, off, token = make_experts(T, d, F, E, k)
    ex, m = Fp8Experts(w, gradients=True), Fp8Matrix(w["w2"])
    off, token = off.int().cuda(), token.int().cuda()
    dy = normal(T * k, d)
    out = {}

    def step(stream=None):
        saved = torch.empty(T * k, 2 * F, dtype=torch.bfloat16, device="cuda")
        out["y"] = ex.forward(x, off, token, saved=saved, stream=stream)
        out["dx"] = ex.backward(dy, saved, off, stream=stream)
        out["p"] = m.product(saved[:, :F].contiguous(), off, stream=stream)

    step()
    first = {a: b.clone() for a, b in out.items()}
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert all(torch.equal(first[a], out[a]) for a in out)
    eager = Fp8Experts(w, gradients=True), Fp8Matrix(w["w2"])
    graph = capture(step)
    for seed in range(3):
        x.copy_(normal(T, d, seed=20 + seed))
        dy.copy_(normal(T * k, d, seed=30 + seed))
        graph.replay()
        torch.cuda.synchronize()
        saved = torch.empty(T * k, 2 * F, dtype=torch.bfloat16, device="cuda")
        assert torch.equal(out["y"], eager[0].forward(x, off, token, saved=saved))
        assert torch.equal(out["dx"], eager[0].backward(dy, saved, off))
        assert torch.equal(out["p"], eager[1].product(saved[:, :F].contiguous(), off))


def test_wrong_tensors_are_refused():
    w, x, off, token = make_experts(20, 128, 192, 4, 1)
    off, token = off.int().cuda(), token.int().cuda()
    ex, m = Fp8Experts(w), Fp8Matrix(w["w1"])
    saved = torch.empty(20, 384, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: ex.forward(x.float(), off, token), lambda: ex.forward(x, off[:-1], token), lambda: ex.forward(x, off, token.long()),
                 lambda: ex.backward(x, saved, off), lambda: Fp8Experts({**w, "w2": w["w1"]}), lambda: m.product_backward(x, off),
                 lambda: m.product(x), lambda: m.product(x.float(), off), lambda: m.product(x[:, :64].contiguous(), off),
                 lambda: m.product(x, off, out=torch.empty(20, 64, device="cuda")), lambda: Fp8Matrix(torch.zeros(8, device="cuda")),
                 lambda: m.product(x, off.cpu()), lambda: m.product(x, off, out=torch.empty(20, 384, device="cuda")[:, ::2]),
                 lambda: Fp8Matrix(torch.zeros(8, 8, dtype=torch.float16, device="cuda"))):
        with pytest.raises((ValueError, L.EatError)):
            call()
    for bad in (torch.zeros(4, 12, device="cuda"), torch.zeros(12, 8, device="cuda"), torch.zeros(257, 8, 8, device="cuda")):
        with pytest.raises(L.EatError):
            Fp8Matrix(bad)
