"""Rows past 2^32 elements through sort, combine, the 8-bit products and experts
(up to 30 GB of them): the last rows and some between, against 64 bits."""
import pytest
import torch

from paper_2609_33614_amd.layer import Fp8Experts, Fp8Matrix
from tests import fp8_reference as R
from tests import test_gpu_fp8 as Q
from tests import test_gpu_sort as S

pytestmark = pytest.mark.gpu


def filled(n, d, std=1.0, seed=0):
    """Random rows, made on the GPU piece by piece."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    for r in range(0, n, 1 << 16):
        out[r: r + (1 << 16)] = std * torch.randn(out[r: r + (1 << 16)].shape, generator=g, device="cuda")
    return out


def some(n, k, seed=0):
    """k rows of n: the first, the last ones and random ones, in order."""
    g = torch.Generator().manual_seed(seed)
    at = torch.cat([torch.arange(2), n - 1 - torch.arange(k // 2), torch.randint(0, n, (k // 2,), generator=g)])
    return torch.unique(at).cuda()


def test_rows_there_and_back():
    T, E, d, k = 65536 + 9, 8, 8192, 8
    lay = S.make_layer(E, d, True, T)
    x = filled(T, d)
    mask = torch.full((T,), 255, dtype=torch.int64, device="cuda")
    rows, off, token, place = lay.sort(x, mask, cap=T * k)
    assert rows.numel() > 2 ** 32 and off.tolist() == [T * e for e in range(E + 1)]
    for e in range(E):
        assert torch.equal(rows[T * e: T * (e + 1)], x)
    g = torch.Generator(device="cuda").manual_seed(1)
    gate = torch.rand(T, E, generator=g, device="cuda")
    gate /= gate.sum(1, keepdim=True)
    rows.mul_(torch.arange(1, T * k + 1, device="cuda").remainder(13)[:, None].to(torch.bfloat16))
    y, dy = lay.combine(rows, mask, gate, place), filled(T, d, seed=2)
    drows, dg = torch.empty_like(rows), torch.empty_like(gate)
    lay.combine_backward(dy, rows, mask, gate, place, drows=drows, dgate=dg)
    at = some(T, 200)
    flat = torch.arange(E, device="cuda") * T + at[:, None]
    own, n = rows[flat].double(), at.numel()
    t = torch.arange(n, device="cuda").repeat_interleave(E)
    S.within("large combine", y[at], *S.sums(t, own.flatten(0, 1), gate[at].double().flatten(), n, 2.0 ** -8))
    want = gate[at].double()[:, :, None] * dy[at].double()[:, None]
    S.within("large drows", drows[flat], want, (2.0 ** -8 + S.U) * want.abs() + 2.0 ** -140)
    dots = dy[at].double()[:, None] * own
    S.within("large dgate", dg[at], dots.sum(2), d * S.U * dots.abs().sum(2) + 2.0 ** -140)
    one = torch.ones(n * E, dtype=torch.float64, device="cuda")
    S.within("large dx", lay.sort_backward(rows, mask, place)[at], *S.sums(t, own.flatten(0, 1), one, n, 2.0 ** -8))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_product(dtype):
    n, K, M = 2 ** 20 + 77, 4096, 4104
    w, x = Q.normal(1, M, K, std=K ** -0.5), filled(n, K)
    out = torch.empty(n, M, dtype=dtype, device="cuda")
    Fp8Matrix(w).product(x, out=out)
    at = some(n, 300)
    off = torch.tensor([0, at.numel()])
    ref, bound, _ = R.grouped(R.quantize(x[at])[0], R.quantize(w, 128)[0], off, exact=dtype == torch.float32)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    Q.within("large product", out[at], ref, (1 + half) * bound + half * ref.abs() + Q.TINY)


def test_experts():
    E, d, F, n = 2, 256, 2112, 2 ** 20 + 77
    w, x, _, _ = Q.make_experts(n, d, F, E, 1)
    cut = n // 3
    off = torch.tensor([0, cut, n])
    token = torch.randperm(n, generator=torch.Generator().manual_seed(0)).int().cuda()
    ex = Fp8Experts(w, gradients=True)
    y, saved = torch.empty(n, d, dtype=torch.bfloat16, device="cuda"), torch.empty(n, 2 * F, dtype=torch.bfloat16, device="cuda")
    ex.forward(x, off.int().cuda(), token, y=y, saved=saved)
    dy = filled(n, d, std=0.01)
    dx = ex.backward(dy, saved, off.int().cuda())
    assert saved.numel() > 2 ** 32
    at = some(n, 300)
    small = torch.tensor([0, int((at < cut).sum()), at.numel()])
    (ry, by, _), (rs, bs) = Q.experts_reference(x, w, small, token[at].long())
    h = 2.0 ** -8
    Q.within("large experts y", y[at], ry, by)
    Q.within("large experts saved", saved[at], rs, (1 + h) * bs + h * rs.abs() + Q.TINY)
    rdx, bdx, _ = Q.backward_reference(dy[at], saved[at], w, small)
    Q.within("large experts dx", dx[at], rdx, bdx)
