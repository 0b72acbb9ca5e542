"""8-bit matrices at the limits of their sizes: the last bytes of 2^31, and the
numbers there."""
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import Fp8Experts, Fp8Matrix
from tests import fp8_reference as R
from tests import test_gpu_fp8 as Q

pytestmark = pytest.mark.gpu


def big(M, K, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    for r in range(0, M, 1 << 16):
        w[r: r + (1 << 16)] = torch.randn(w[r: r + (1 << 16)].shape, generator=g, device="cuda")
    return w


def test_rows_of_the_largest_matrix():
    """2040 x 2^20: rows that pick one column each give that column's 8-bit numbers as they are."""
    M, K = 2040, 1 << 20
    w = big(M, K)
    m = Fp8Matrix(w)
    cols = torch.tensor([0, 5, 127, 128, 77777, K // 2, K - 129, K - 1], device="cuda")
    x = torch.zeros(cols.numel(), K, dtype=torch.bfloat16, device="cuda")
    x[torch.arange(cols.numel()), cols] = 1.0
    y, y32 = m.product(x), m.product(x, out=torch.empty(cols.numel(), M, device="cuda"))
    for r in range(0, M, 128):
        strip = R.quantize(w[r: r + 128], 128)[0][:, cols].T
        assert torch.equal(y[:, r: r + 128].double(), strip) and torch.equal(y32[:, r: r + 128].double(), strip)


def test_the_largest_matrix_transposed():
    """2^20 x 2040 written transposed alone (as it lies it would pass 2^31 bytes)."""
    M, K = 1 << 20, 2040
    w = big(M, K, 1)
    nq, ns = L.eat_fp8_size(1, K, M)
    q = torch.empty(1, K, M, dtype=torch.float8_e4m3fn, device="cuda")
    s = torch.empty(1, -(-K // 128), -(-M // 512) * 4, dtype=torch.uint8, device="cuda")
    assert (q.numel(), s.numel()) == (nq, ns)
    L.eat_fp8_quantize(w, L.EAT_BF16, 1, M, K, 1, q, s)
    with pytest.raises(L.EatError):
        L.eat_fp8_quantize(w, L.EAT_BF16, 1, M, K, 0, q, s)
    for c in (0, 128, 1024, 1920):
        want, k = R.quantize(w[:, c: c + 128].T.contiguous(), 128)
        have = torch.exp2(s[0, c // 128, : M // 128].double() - 127).repeat_interleave(128) * q[0, c: c + 128].double()
        assert torch.equal(have, want) and torch.equal(s[0, c // 128, : M // 128].int() - 127, k[0].int())


@pytest.mark.parametrize("T", [3, 300])
def test_experts_too_wide_for_a_gradient(T):
    """16384 x 65536: 2^30 elements a matrix, whose gradient's [d][2 d_ffn] would have 2^31. Rows of x with
    one element pick the 8-bit numbers of W1 and W3 as g and u, exactly; y as the other tests of the experts."""
    d, F = 16384, 65536
    w = {"w1": big(F, d, 2)[None], "w3": big(F, d, 3)[None], "w2": big(d, F, 4)[None]}
    for n, k in (("w1", 7), ("w3", 7), ("w2", 8)):
        w[n].mul_(2.0 ** -k)
    ex = Fp8Experts(w)
    with pytest.raises(L.EatError):
        Fp8Experts(w, gradients=True)
    x, token, off = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda"), torch.arange(T), torch.tensor([0, T])
    x[token, (d - 1 - 5003 * token) % d] = 128.0
    saved = torch.empty(T, 2 * F, dtype=torch.bfloat16, device="cuda")
    y = ex.forward(x, off.int().cuda(), token.int().cuda(), saved=saved)
    assert torch.equal(ex.forward(x, off.int().cuda(), token.int().cuda()), y)
    (ry, by, vy), (rs, _) = Q.experts_reference(x, w, off, token.cuda())
    assert torch.equal(saved.double(), rs)
    Q.within(f"wide experts {T}", y, ry, by)
    assert (y.double() - ry).square().sum() <= vy.sum()


@pytest.mark.parametrize("n", [5, 100, 2600])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_largest_magnitudes(n, dtype):
    """bf16's largest rounds to 2^128: its row's results are those of that number, or not finite; every other
    row keeps its bits. 1.875 2^127 is held as it is."""
    K, M = 256, 264
    top = torch.finfo(torch.bfloat16).max
    w, x = Q.normal(1, M, K, dtype=torch.float32).clamp(-3, 3) * 2.0 ** -60, Q.normal(n, K)
    m = Fp8Matrix(w)
    want = m.product(x, out=torch.empty(n, M, dtype=dtype, device="cuda"))
    held, big = x.clone(), x.clone()
    held[1], held[1, 7], big[1, 7], big[n - 1, 200] = 0.0, 1.875 * 2.0 ** 127, top, -top
    got = m.product(big, out=torch.empty_like(want))
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[1] = keep[n - 1] = False
    assert torch.equal(got[keep], want[keep])
    wq = R.quantize(w, 128)[0][0]
    for r, c, v in ((1, 7, 2.0 ** 128), (n - 1, 200, -2.0 ** 128)):
        ref = v * wq[:, c]                                # (the block's other numbers lie below 2^-15 of it: zeros)
        bad = ~got[r].isfinite()
        assert ((got[r].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -20 * ref.abs().max())[~bad].all()
    one = m.product(held, out=torch.empty_like(want))
    assert torch.equal(one[1].double(), 1.875 * 2.0 ** 127 * wq[:, 7]) if dtype == torch.float32 else one[1].isfinite().all()
