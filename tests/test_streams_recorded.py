"""What a call on a named stream reads or writes is made known to torch's
allocator there, so that dropping it while the stream has work pending does not
give its memory away: shown without a GPU, the library's launches left out."""
import contextlib
import os
import types

import pytest
import torch

from paper_2609_33614_amd import _lib as L
from paper_2609_33614_amd import layer as M

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libeat.so not built")

HOME, SIDE = (types.SimpleNamespace(cuda_stream=n, device=torch.device("cpu")) for n in (1, 2))


@pytest.fixture
def seen(monkeypatch):
    """A list of (tensor, stream) pairs that were recorded; `capturing` makes the calls part of a capture."""
    class Seen(list):
        capturing = False

        def on(self, stream):
            return {t.data_ptr() for t, s in self if s is stream}

    seen, current = Seen(), [HOME]

    @contextlib.contextmanager
    def calling_on(stream, device):
        before, current[0] = current[0], current[0] if stream is None else stream
        yield
        current[0] = before

    monkeypatch.setattr(M, "_calling_on", calling_on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: current[0])
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: seen.capturing)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: seen.append((t, s)))
    for name in ("eat_sort_tokens", "eat_sort_backward", "eat_combine", "eat_combine_backward", "eat_fp8_quantize", "eat_fp8_product",
                 "eat_fp8_experts_quantize", "eat_fp8_experts_forward", "eat_fp8_experts_backward", "eat_balance_loss", "eat_ce_loss"):
        monkeypatch.setattr(L, name, lambda *a, **k: None)
    seen.current = current
    return seen


def bf16(*s):
    return torch.zeros(*s, dtype=torch.bfloat16)


def i32(*s):
    return torch.zeros(*s, dtype=torch.int32)


def experts():
    return {"w1": bf16(4, 128, 64), "w3": bf16(4, 128, 64), "w2": bf16(4, 64, 128)}


def ptrs(*tensors):
    return {t.data_ptr() for t in tensors}


def test_the_weights_given_to_a_constructor(seen):
    w, m = experts(), bf16(2, 64, 64)
    M.Fp8Experts(w, gradients=True, stream=SIDE)
    M.Fp8Matrix(m, gradients=True, stream=SIDE)
    assert ptrs(*w.values(), m) <= seen.on(SIDE)


def own(ex, m):
    return ptrs(ex.buf, m.q, m.scale), ptrs(ex.buf, m.qt, m.scale_t)


@pytest.mark.parametrize("named", [True, False])
def test_the_weights_that_an_object_holds(seen, named):
    """Used on another stream than they were made on, named by the call or the current one."""
    ex, m = M.Fp8Experts(experts(), gradients=True), M.Fp8Matrix(bf16(2, 64, 64), gradients=True)
    x, off, off2, token, saved = bf16(6, 64), i32(5), i32(3), i32(6), bf16(6, 256)
    ex.forward(x, off, token)
    ex.backward(x, saved, off)
    m.product(x, off2)
    m.product_backward(x, off2)
    assert not seen                                       # (the stream that they were made on)
    stream = SIDE if named else None
    if not named:
        seen.current[0] = SIDE
    forward, backward = own(ex, m)
    ex.forward(x, off, token, stream=stream)
    m.product(x, off2, stream=stream)
    assert forward <= seen.on(SIDE)
    seen.clear()
    ex.backward(x, saved, off, stream=stream)
    m.product_backward(x, off2, stream=stream)
    assert backward <= seen.on(SIDE)


def test_what_is_made_on_a_named_stream_belongs_there(seen):
    ex = M.Fp8Experts(experts(), stream=SIDE)
    seen.clear()
    ex.forward(bf16(6, 64), i32(5), i32(6))
    assert ex.buf.data_ptr() in seen.on(HOME)


def test_the_tensors_given_to_a_call(seen):
    ex, m = M.Fp8Experts(experts(), gradients=True), M.Fp8Matrix(bf16(2, 64, 64), gradients=True)
    x, off, off2, token, saved, out = bf16(6, 64), i32(5), i32(3), i32(6), bf16(6, 256), bf16(6, 64)
    lay = M.EatLayer(L.eat_params_default(mode="topk", E=4, d_model=64, d_ffn=64, top_k=1), 8, {"w_router": torch.zeros(4, 64)}, device="cpu")
    mask, gate, prob, place, dz = torch.zeros(6, dtype=torch.int64), torch.zeros(6, 4), torch.zeros(6, 4), i32(6, 4), torch.zeros(6, 4)
    rows, valid, dw = bf16(6, 64), torch.ones(6, dtype=torch.bool), torch.zeros(4, 64)
    ce, target = M.CrossEntropy(bf16(32, 64)), i32(6)
    for call, uses in ((lambda s: ex.forward(x, off, token, y=out, saved=saved, stream=s), (x, off, token, out, saved)),
                       (lambda s: ex.backward(x, saved, off, dx=out, stream=s), (x, saved, off, out)),
                       (lambda s: m.product(x, off2, token=token, out=out, stream=s), (x, off2, token, out)),
                       (lambda s: m.product_backward(x, off2, dx=out, stream=s), (x, off2, out)),
                       (lambda s: lay.sort(x, mask, cap=6, rows=rows, stream=s), (x, mask, rows)),
                       (lambda s: lay.sort_backward(rows, mask, place, dx=out, stream=s), (rows, mask, place, out)),
                       (lambda s: lay.combine(rows, mask, gate, place, y=out, stream=s), (rows, mask, gate, place, out)),
                       (lambda s: lay.combine_backward(x, rows, mask, gate, place, prob=prob, drows=out, dlogits=dz, stream=s),
                        (x, rows, mask, gate, place, prob, out, dz)),
                       (lambda s: lay.balance_loss(x, prob, mask, valid=valid, dlogits=dz, dx=out, dw_router=dw, stream=s),
                        (x, prob, mask, valid, dz, out, dw, lay.w["w_router"])),
                       (lambda s: ce.loss(x, target, dh=out, stream=s), (x, target, out, ce.w))):
        seen.clear()
        call(SIDE)
        assert ptrs(*uses) <= seen.on(SIDE)
        seen.clear()
        call(None)
        assert not ptrs(*uses) & seen.on(HOME)


def test_nothing_is_recorded_in_a_capture(seen):
    w = experts()
    ex = M.Fp8Experts(w)
    seen.capturing = True
    ex.forward(bf16(6, 64), i32(5), i32(6), stream=SIDE)
    M.Fp8Experts(w, stream=SIDE)
    assert not seen.on(SIDE)
