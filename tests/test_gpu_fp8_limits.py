"""8-bit matrices at the limits of their sizes: the last bytes of 2^31, and the
numbers there."""
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import Fp8Matrix
from tests import fp8_reference as R

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
