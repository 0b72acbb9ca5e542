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
