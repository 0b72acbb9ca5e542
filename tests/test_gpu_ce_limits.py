"""The cross entropy at the ends of its sizes: vocabularies past the most columns
a piece has (2^22), and the most positions (2^20)."""
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import CrossEntropy
from tests.test_gpu_ce import IGN, call, check, make, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,n", [(3, 3), (66, 66), (66, 5)])
def test_vocabularies_past_a_pieces_columns(T, n):
    V = (1 << 22) + 4099
    h, w, y = make(T, 64, V)
    y[:3] = torch.tensor([0, V - 1, 1 << 22], dtype=torch.int32)
    y[n:] = IGN
    check(f"ce {T} {V}", call(h, w, y), reference(h, w, y, True, 1.0))


@pytest.mark.parametrize("ignored", [None, 0.9])
def test_the_most_positions(ignored):
    T, V = 1 << 20, 70
    h, w, y = make(T, 64, V, ignored=ignored)
    check(f"ce {T} {V}", call(h, w, y), reference(h, w, y, True, 1.0))
    with pytest.raises(RuntimeError):
        CrossEntropy(w).loss(torch.cat([h, h[:1]]), torch.cat([y, y[:1]]))


@pytest.mark.parametrize("T", [5, 300])
def test_the_widest_rows(T):
    h, w, y = make(T, 65536, 130)
    check(f"ce {T} 65536", call(h, w, y), reference(h, w, y, True, 1.0))


def test_the_default_stream_by_its_address():
    h, w, y = make(300, 192, 1500, ignored=0.2)
    ref = call(h, w, y)
    dh = torch.empty_like(h)
    torch.cuda.synchronize()
    for at in (torch.cuda.default_stream(), torch.cuda.default_stream().cuda_stream):
        ce = CrossEntropy(w)
        loss = ce.loss(h, y, dh=dh, stream=at)
        torch.cuda.synchronize()
        assert torch.equal(loss, ref["loss"]) and torch.equal(dh, ref["dh"])
        assert ce.workspace(300, L.EAT_CE_DH, stream=at).numel() > 0
