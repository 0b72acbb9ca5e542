"""Calls of the losses on a stream that the caller names, while the current one
has work pending: what a call allocates must be memory that its own stream may
use at once."""
import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd.layer import CrossEntropy
from tests.test_gpu_balance import make_valid, routed
from tests.test_gpu_ce import make

pytestmark = pytest.mark.gpu


def cases():
    h, w, y = make(300, 192, 1500, ignored=0.2)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    ce = CrossEntropy(w)
    need = ce.workspace(300, L.EAT_CE_DH | L.EAT_CE_DW).numel()

    def cross(stream=None):
        loss = CrossEntropy(w).loss(h, y, dh=dh, dw=dw, stream=stream)
        return [loss, dh, dw]

    layer, x, prob, mask = routed(60, 128, True, 700)
    valid = make_valid(700, "some")
    grads = [torch.empty_like(prob), torch.empty_like(x), torch.empty(60, 128, device="cuda")]

    def balance(stream=None):
        layer._bws.buf = None
        loss, count, mean = layer.balance_loss(x, prob, mask, valid, 0.01, 0.002, dlogits=grads[0], dx=grads[1],
                                               dw_router=grads[2], stream=stream)
        return [loss, count, mean, *grads]

    return {"ce": (cross, need), "balance": (balance, L.eat_balance_workspace_size(layer.handle, 700))}


@pytest.mark.parametrize("which", ["ce", "balance"])
@pytest.mark.parametrize("how", ["stream", "address"])
def test_the_current_streams_pending_work_and_the_call_do_not_meet(which, how):
    run, size = cases()[which]
    want = [t.clone() for t in run()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    # blocks of the sizes that the call allocates, given back while the current
    # stream has still to read and then to overwrite them
    small = [torch.full((n,), 5, dtype=torch.uint8, device="cuda") for n in (4, 240, 480) for _ in range(64)]
    large = [torch.full((size,), 5, dtype=torch.uint8, device="cuda") for _ in range(4)]
    copies = [torch.empty_like(t) for t in small + large]
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    for t, c in zip(small + large, copies):
        c.copy_(t)
        t.fill_(0xFF)
    del small, large, t
    got = run(side if how == "stream" else side.cuda_stream)
    side.synchronize()
    first = [t.clone() for t in got]
    torch.cuda.synchronize()
    for a, b, r in zip(first, got, want):
        assert torch.equal(a, r) and torch.equal(b, r)
    assert all((c == 5).all() for c in copies)


@pytest.mark.parametrize("which", ["ce", "balance"])
def test_what_a_call_returns_may_be_dropped_while_the_current_stream_reads_it(which):
    run, _ = cases()[which]
    want = [t.clone() for t in run()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = run(side)
    side.synchronize()
    torch.cuda._sleep(200_000_000)
    copy = [t.clone() for t in got]               # (pending)
    with torch.cuda.stream(side):
        del got
        fill = [torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") for n in (4, 240, 480) for _ in range(64)]
    torch.cuda.synchronize()
    assert all(torch.equal(c, r) for c, r in zip(copy, want)) and all((f == 0xFF).all() for f in fill)
