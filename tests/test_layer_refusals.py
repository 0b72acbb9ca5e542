"""What the owner objects refuse by themselves, without a GPU."""
import os

import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import EatLayer

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libeat.so not built")


def test_combine_without_gates_is_no_unweighted_sum(monkeypatch):
    ran = []
    for name in ("eat_combine", "eat_sort_backward"):
        monkeypatch.setattr(L, name, lambda *a: ran.append(a))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: None)
    lay = EatLayer(L.eat_params_default(mode="topk", E=4, d_model=64, d_ffn=64, top_k=1), 8, {}, device="cpu")
    rows, mask, place = torch.zeros(6, 64, dtype=torch.bfloat16), torch.zeros(6, dtype=torch.int64), torch.zeros(6, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        lay.combine(rows, mask, None, place)
    assert not ran


def test_numbers_past_32_bits_are_not_cut():
    """2^32 + 8 rows are no call of 8 rows."""
    big, A = (1 << 32) + 8, 1 << 50
    h = L.eat_create(L.eat_params_default(mode="topk", E=4, d_model=64, d_ffn=64, top_k=1), 100)
    try:
        for call in (lambda: L.eat_fp8_size(1, big, 8), lambda: L.eat_fp8_product_workspace_size(big, big, 1, 64, 64),
                     lambda: L.eat_fp8_product(A, big, None, None, big, 2 * A, 3 * A, 1, 64, 64, 4 * A, L.EAT_BF16, 5 * A, 1 << 40, stream=0),
                     lambda: L.eat_fp8_quantize(A, L.EAT_BF16, big, 64, 64, 0, 2 * A, 3 * A, stream=0),
                     lambda: L.eat_sort_workspace_size(h, big), lambda: L.eat_sort_tokens(h, A, 8, 2 * A, big, 3 * A, 4 * A, 5 * A, 6 * A, stream=0),
                     lambda: L.eat_combine(h, A, big, 8, 2 * A, 3 * A, 4 * A, 5 * A, stream=0),
                     lambda: L.eat_fp8_experts_workspace_size(h, 8, big, 1), lambda: L.eat_create(L.eat_params_default(), big),
                     lambda: L.eat_workspace_size(h, -big), lambda: L.eat_balance_workspace_size(h, big), lambda: L.eat_ce_workspace_size(big, 64, 64, 0)):
            with pytest.raises((ValueError, L.EatError)):
                call()
    finally:
        L.eat_destroy(h)


def test_a_workspace_lies_on_the_calls_device(monkeypatch):
    """A layer's sort runs where its mask is: memory that a call on another device left is no workspace there."""
    from types import SimpleNamespace
    from paper_2609_33614_amd.layer import _Workspace
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    one, two = (SimpleNamespace(cuda_stream=0, device=torch.device(d)) for d in ("cpu", "meta"))
    ws = _Workspace(one.device)
    a = ws.get(1000, one)
    assert a.device == one.device and ws.get(500, one) is a
    b = ws.get(500, two)
    assert b.device == two.device and b.numel() >= 500 and ws.get(500, two) is b
    assert ws.get(500, one).device == one.device
