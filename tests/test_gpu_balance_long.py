"""Balance losses of more rows or columns than one workgroup each may take."""
import pytest
import torch

from tests.test_gpu_balance import call, check, make_layer, make_valid, reference

pytestmark = pytest.mark.gpu


def inputs(T, E, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    prob = torch.softmax(2 * torch.randn(T, E, generator=g, device="cuda"), 1)
    words = torch.zeros(T, (E + 63) // 64, dtype=torch.int64, device="cuda")
    e = prob.argmax(1)
    words.scatter_(1, (e // 64)[:, None], (torch.ones_like(e) << (e % 64))[:, None])
    return prob, words.view(T) if words.shape[1] == 1 else words, g


@pytest.mark.parametrize("kind", [None, "some"])
def test_more_rows_of_x_than_workgroups(kind):
    """fp32 tokens on bf16 parts: 2^22 workgroups at most write x's parts."""
    T, E, d = (1 << 22) + 777, 65, 64
    layer = make_layer(E, d, False, T, k=1)
    prob, mask, g = inputs(T, E)
    x = torch.randn(T, d, generator=g, device="cuda")
    valid = make_valid(T, kind)
    got, ref = call(layer, x, prob, mask, valid), reference(layer, x, prob, mask, valid, 0.01, 0.002)
    check(f"bal {T} {kind}", got, ref)


def test_more_tiles_of_dx_than_workgroups():
    """fp32 instructions: 2^22 workgroups at most, here of 256 x 16385 tiles."""
    T, E, d = 16383, 2, (1 << 20) + 64
    layer = make_layer(E, d, True, T, k=1)
    prob, mask, _ = inputs(T, E)
    dz, dx = torch.empty_like(prob), torch.full((T, d), 7.0, dtype=torch.bfloat16, device="cuda")
    layer.balance_loss(None, prob, mask, None, dlogits=dz, dx=dx)
    w = layer.w["w_router"]
    for c in range(0, d, 65536):
        want = dz.double() @ w[:, c:c + 65536].double()
        # two products and their sum in fp32 (2^-22 of their absolute sum), then bf16
        bound = 2.0 ** -22 * (dz.abs().double() @ w[:, c:c + 65536].abs().double()) + 2.0 ** -8 * want.abs() + 2.0 ** -120
        assert ((dx[:, c:c + 65536].double() - want).abs() <= 1.01 * bound).all(), c
