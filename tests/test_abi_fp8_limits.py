"""Sizes at the limits of the 8-bit entry points, without a GPU: what the header allows is not refused."""
import os

import pytest

from paper_2609_33614_amd import _lib as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libeat.so not built")

F = 1 << 40           # an aligned address that nothing reads
BAD, UNSUP = L.EAT_ERR_INVALID_ARG, L.EAT_ERR_UNSUPPORTED


def status(fn, *args, **kw):
    try:
        fn(*args, **kw)
    except L.EatError as e:
        return e.status
    return L.EAT_OK


@pytest.mark.parametrize("M,K", [(2040, 1 << 20), (1 << 20, 2040), (2048, (1 << 20) - 128), (1 << 20, 2056), (2056, 1 << 20), ((1 << 20) + 8, 8), (64, 128)])
def test_weights_are_rounded_wherever_a_matrix_of_that_size_is_taken(M, K):
    """M K padded below 2^31 counts for the matrix that is written: as it lies, or transposed."""
    for t, rows, cols in ((0, M, K), (1, K, M)):
        # (w is missing, which is looked at after the sizes)
        want = BAD if status(L.eat_fp8_size, 1, rows, cols) == L.EAT_OK else UNSUP
        assert status(L.eat_fp8_quantize, None, L.EAT_BF16, 1, M, K, t, 2 * F, 3 * F, stream=0) == want, (t, M, K)
        assert (want == BAD) == (rows * -(-cols // 128) * 128 < 1 << 31 and max(rows, cols) <= 1 << 20)
        assert (status(L.eat_fp8_product_workspace_size, 1, 1, 1, rows, cols) == L.EAT_OK) == (want == BAD)


@pytest.mark.parametrize("d,ffn,grads", [(16384, 65536, False), (8192, 131008, False), (64, 1 << 20, False), (64, (1 << 19) + 64, False), (64, 1 << 19, True),
                                         (8192, 65408, True), (16384, 65536 // 2 - 128, True)])
def test_experts_that_only_run_forward_need_no_room_for_the_gradients_matrix(d, ffn, grads):
    """[E][d][2 d_ffn] is the backward's: sizes that pass 2^31 bytes or 2^20 columns there have their forward."""
    h = L.eat_create(L.eat_params_default(mode="topk", E=1, d_model=d, d_ffn=ffn, top_k=1), 5)
    try:
        back = L.EAT_OK if grads else UNSUP
        assert status(L.eat_fp8_experts_size, h, 0) == L.EAT_OK and status(L.eat_fp8_experts_size, h, 1) == back
        assert status(L.eat_fp8_experts_workspace_size, h, 3, 3, 0) == L.EAT_OK and status(L.eat_fp8_experts_workspace_size, h, 3, 3, 1) == back
        # (arrays that are missing are looked at after the sizes)
        missing = lambda st: BAD if st == L.EAT_OK else st
        assert status(L.eat_fp8_experts_quantize, h, None, F, F, 0, F, stream=0) == BAD
        assert status(L.eat_fp8_experts_quantize, h, None, F, F, 1, F, stream=0) == missing(back)
        assert status(L.eat_fp8_experts_forward, h, F, 3, F, F, 3, None, F, None, F, 0, stream=0) == BAD
        assert status(L.eat_fp8_experts_backward, h, F, F, 3, None, F, F, F, 0, stream=0) == missing(back)
    finally:
        L.eat_destroy(h)
