"""A small owner object around one EAT layer handle.

Holds the handle, the caller-owned account tensors and a workspace
allocated with torch (device memory plumbing only), and forwards to the C
entry points of ``_lib``.  All compute runs in libeat.so.
"""
from __future__ import annotations

import contextlib
from typing import Dict, Optional

import torch

from . import _lib as L


def _expect(name: str, t: Optional[torch.Tensor], dtype, shape, device=None) -> None:
    """Refuse a tensor (None passes) whose type, shape or device the library would misread."""
    if t is None:
        return
    if t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)) or t.shape != tuple(shape):
        raise ValueError(f"{name}: expected {dtype} {list(shape)}, got {t.dtype} {list(t.shape)}")
    if device is not None and t.device != device:
        raise ValueError(f"{name}: on {t.device}, the call's other tensors on {device}")


class _Workspace:
    """A growing device buffer.  One that a graph capture used stays alive as
    long as its owner does, so that the graph may be replayed after it grew;
    one that another stream used than it was made on is not given away before
    that stream is done."""

    def __init__(self, device):
        self.device, self.buf, self.home, self.captured = device, None, 0, []

    def get(self, need: int, stream) -> torch.Tensor:
        """At least `need` bytes for a call on `stream`, the current one, on its device
        (a layer's calls run where their tensors are)."""
        if self.buf is None or self.buf.numel() < need or self.device != stream.device:
            self.device = stream.device
            self.buf = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
            self.home = stream.cuda_stream
        if torch.cuda.is_current_stream_capturing():
            if not any(b is self.buf for b in self.captured):
                self.captured.append(self.buf)
        elif stream.cuda_stream != self.home:
            self.buf.record_stream(stream)
        return self.buf


def _calling_on(stream, device):
    """The context of a call: its tensors' device and its stream (None: the
    current one; one of torch's, or an address) are the current ones, so that
    what it allocates is memory which that stream may use at once."""
    if stream is None:
        # (the library launches on the current device)
        index = device.index
        return contextlib.nullcontext() if index is None or index == torch.cuda.current_device() else torch.cuda.device(index)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device)
    if stream.device != device:
        raise ValueError(f"stream: on {stream.device}, the call's tensors on {device}")
    return torch.cuda.stream(stream)


def _hand_out(stream, caller, *tensors) -> None:
    """Tell torch's allocator that the caller's stream uses what a call on `stream` made."""
    if stream is not None:
        for t in tensors:
            t.record_stream(caller)


def _take_in(named: bool, on, *tensors) -> None:
    """Tell torch's allocator that a call uses `tensors` (None passes) on `on`, the
    current stream, where that is `named` (not their own): dropped, their
    memory is not given away before `on` is done.  What a graph reads stays its
    caller's to keep."""
    if named and not torch.cuda.is_current_stream_capturing():
        for t in tensors:
            if t is not None:
                t.record_stream(on)


class EatLayer:
    def __init__(self, params: L.eat_params_t, max_tokens: int, weights: Dict[str, torch.Tensor],
                 device: str = "cuda"):
        self.params = params
        self.max_tokens = int(max_tokens)
        self.device = torch.device(device)
        self.handle = L.eat_create(params, max_tokens)
        self.w = weights
        E = params.E
        self.n = torch.zeros(E, dtype=torch.int64, device=self.device)
        self.p_total = torch.zeros(E, dtype=torch.float32, device=self.device)
        self.c_s = torch.zeros(E, dtype=torch.float32, device=self.device)
        self._ws: Optional[torch.Tensor] = None
        self._bws = _Workspace(self.device)

    # account state -------------------------------------------------------
    @property
    def acc(self) -> L.eat_accounts_t:
        return L.accounts(self.n, self.p_total, self.c_s)

    def reset_accounts(self, stream=None) -> None:
        L.eat_reset_accounts(self.handle, self.acc, stream)

    def load_accounts(self, n, p_total, c_s) -> None:
        self.n.copy_(torch.as_tensor(n, dtype=torch.int64))
        self.p_total.copy_(torch.as_tensor(p_total, dtype=torch.float32))
        self.c_s.copy_(torch.as_tensor(c_s, dtype=torch.float32))

    def accounts_host(self):
        return (self.n.cpu().numpy(), self.p_total.cpu().numpy(), self.c_s.cpu().numpy())

    # workspace -----------------------------------------------------------
    def workspace(self, T: int) -> torch.Tensor:
        need = L.eat_workspace_size(self.handle, T)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        return self._ws

    # calls ---------------------------------------------------------------
    def forward(self, x: torch.Tensor, trend: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                mask_out: Optional[torch.Tensor] = None, load_out: Optional[torch.Tensor] = None,
                stream=None, events=None) -> torch.Tensor:
        T = x.shape[0]
        if y is None:
            y = torch.empty_like(x)
        ws = self.workspace(T)
        w = self.w
        args = (self.handle, x, T, w["w_router"], w["w1"], w["w3"], w["w2"], w.get("ws1"), w.get("ws3"),
                w.get("ws2"), self.acc, trend, y, mask_out, load_out, ws, ws.numel(), stream)
        if events is None:
            L.eat_moe_forward(*args)
        else:
            L.eat_moe_forward_profiled(*args, events=events)
        return y

    def mask_tensor(self, T: int) -> torch.Tensor:
        """Mask output for T tokens: [T] for E <= 64, else [T, words]."""
        W = L.mask_words(self.params.E)
        return torch.empty((T,) if W == 1 else (T, W), dtype=torch.int64, device=self.device)

    def route(self, x: torch.Tensor, trend: Optional[torch.Tensor] = None, stream=None):
        T = x.shape[0]
        E = self.params.E
        mask = self.mask_tensor(T)
        k = torch.empty(T, dtype=torch.int32, device=self.device)
        gate = torch.empty(T, E, dtype=torch.float32, device=self.device)
        prob = torch.empty(T, E, dtype=torch.float32, device=self.device)
        ws = self.workspace(T)
        L.eat_route(self.handle, x, T, self.w["w_router"], self.acc, trend, mask, k, gate, prob,
                    ws, ws.numel(), stream)
        return mask, k, gate, prob

    def balance_loss(self, x: Optional[torch.Tensor], prob: torch.Tensor, mask: torch.Tensor,
                     valid: Optional[torch.Tensor] = None, coef: float = 0.01, entropy_coef: float = 0.0,
                     dlogits: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                     dw_router: Optional[torch.Tensor] = None, stream=None):
        """The router's balance loss (eat_balance_loss) of the ``prob`` and
        ``mask`` that ``route`` returned for ``x``: (loss [1], selections per
        expert [E] int64, mean probabilities [E]).  The gradients are written
        to the tensors given.  ``valid`` [T] (bool or uint8): tokens that count.
        Calls of one layer share a workspace: order them on one stream.
        ``stream``: what the call is enqueued on (the current one); the tensors
        given have to be ready there (outside a capture they may be dropped once the
        call has returned), and what is returned is ready when it is."""
        T, E, d = prob.shape[0], self.params.E, self.params.d_model
        act = torch.bfloat16 if self.params.act_dtype == L.EAT_BF16 else torch.float32
        W = L.mask_words(E)
        dev = prob.device
        _expect("prob", prob, torch.float32, (T, E))
        _expect("w_router", self.w["w_router"], torch.float32, (E, d), dev)
        _expect("mask", mask, (torch.int64, torch.uint64), (T,) if mask.dim() == 1 and W == 1 else (T, W), dev)
        _expect("x", x, act, (T, d), dev)
        _expect("valid", valid, (torch.bool, torch.uint8), (T,), dev)
        _expect("dlogits", dlogits, torch.float32, (T, E), dev)
        _expect("dx", dx, act, (T, d), dev)
        _expect("dw_router", dw_router, torch.float32, (E, d), dev)
        caller = torch.cuda.current_stream(dev) if stream is not None else None
        with _calling_on(stream, dev):
            loss = torch.empty(1, dtype=torch.float32, device=dev)
            count = torch.empty(E, dtype=torch.int64, device=dev)
            mean = torch.empty(E, dtype=torch.float32, device=dev)
            need = L.eat_balance_workspace_size(self.handle, T)
            on = torch.cuda.current_stream(dev)
            ws = self._bws.get(need, on)
            L.eat_balance_loss(self.handle, x, T, self.w["w_router"], prob, mask, valid, coef, entropy_coef, loss, count,
                               mean, dlogits, dx, dw_router, ws, need, on)
            _take_in(stream is not None, on, x, self.w["w_router"], prob, mask, valid, dlogits, dx, dw_router)
        _hand_out(stream, caller, loss, count, mean)
        return loss, count, mean

    # tokens sorted by expert, and back ------------------------------------
    def _act(self):
        return torch.bfloat16 if self.params.act_dtype == L.EAT_BF16 else torch.float32

    def _expect_mask(self, mask: torch.Tensor, T: int, dev) -> None:
        W = L.mask_words(self.params.E)
        _expect("mask", mask, (torch.int64, torch.uint64), (T,) if mask.dim() == 1 and W == 1 else (T, W), dev)

    def sort(self, x: Optional[torch.Tensor], mask: torch.Tensor, cap: Optional[int] = None,
             rows: Optional[torch.Tensor] = None, stream=None):
        """The tokens ``x`` sorted by the experts that ``mask`` (from ``route``)
        selects (eat_sort_tokens): (rows [cap][d], offsets [E+1] int32, token
        [cap] int32, place [T][E] int32); rows is None where ``x`` is.  ``cap``:
        the rows to make room for; pairs past it are left out.  Without it, every
        pair that the layer's mode can select has a row (EAT and Top-P: T E of
        them, many times those there are: give the sum of ``route``'s k, or a bound
        near it, where rows go on to ``Fp8Experts``).  Entries behind the last selected
        pair are not written.  Calls of one layer share a workspace: order them on one
        stream.  ``stream`` as in ``balance_loss``."""
        T, E, d, dev = mask.shape[0], self.params.E, self.params.d_model, mask.device
        self._expect_mask(mask, T, dev)
        _expect("x", x, self._act(), (T, d), dev)
        if cap is None:
            p = self.params
            cap = T * (p.top_k if p.mode == L.EAT_MODE_TOPK else p.top_p_cap if p.mode == L.EAT_MODE_TOPP and p.top_p_cap else E)
        if not 0 <= cap < 1 << 31:
            raise ValueError(f"cap: {cap} rows, their numbers have 31 bits")
        if rows is not None and x is None:
            raise ValueError("rows: nothing to write without x")
        _expect("rows", rows, self._act(), (cap, d), dev)
        caller = torch.cuda.current_stream(dev) if stream is not None else None
        with _calling_on(stream, dev):
            given = rows is not None
            if x is not None and not given:
                rows = torch.empty(cap, d, dtype=x.dtype, device=dev)
            offsets = torch.empty(E + 1, dtype=torch.int32, device=dev)
            token = torch.empty(cap, dtype=torch.int32, device=dev)
            place = torch.empty(T, E, dtype=torch.int32, device=dev)
            need = L.eat_sort_workspace_size(self.handle, T)
            on = torch.cuda.current_stream(dev)
            ws = self._bws.get(need, on) if need else None
            L.eat_sort_tokens(self.handle, x, T, mask, cap, rows, offsets, token, place, ws, need, on)
            _take_in(stream is not None, on, x, mask, rows if given else None)
        _hand_out(stream, caller, offsets, token, place, *(() if given or rows is None else (rows,)))
        return rows, offsets, token, place

    def sort_backward(self, drows: torch.Tensor, mask: torch.Tensor, place: torch.Tensor,
                      dx: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """The gradient of ``sort``'s tokens [T][d] from its rows' (eat_sort_backward)."""
        return self._from_rows(drows, mask, None, place, dx, "drows", "dx", stream)

    def combine(self, rows: torch.Tensor, mask: torch.Tensor, gate: torch.Tensor, place: torch.Tensor,
                y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """The experts' ``rows`` [cap][d] back to their tokens, weighted by
        ``gate`` (from ``route``; eat_combine): y [T][d]."""
        if gate is None:
            raise ValueError("gate: the rows' weights are needed")
        _expect("gate", gate, torch.float32, (mask.shape[0], self.params.E), rows.device)
        return self._from_rows(rows, mask, gate, place, y, "rows", "y", stream)

    def _from_rows(self, rows, mask, gate, place, out, src_name, out_name, stream):
        T, E, d, dev = mask.shape[0], self.params.E, self.params.d_model, rows.device
        cap = rows.shape[0]
        _expect(src_name, rows, self._act(), (cap, d), dev)
        self._expect_mask(mask, T, dev)
        _expect("place", place, torch.int32, (T, E), dev)
        _expect(out_name, out, self._act(), (T, d), dev)
        caller = torch.cuda.current_stream(dev) if stream is not None else None
        with _calling_on(stream, dev):
            given = out is not None
            if not given:
                out = torch.empty(T, d, dtype=rows.dtype, device=dev)
            on = torch.cuda.current_stream(dev)
            if gate is None:
                L.eat_sort_backward(self.handle, rows, cap, T, mask, place, out, on)
            else:
                L.eat_combine(self.handle, rows, cap, T, mask, gate, place, out, on)
            _take_in(stream is not None, on, rows, mask, gate, place, out if given else None)
        if not given:
            _hand_out(stream, caller, out)
        return out

    def combine_backward(self, dy: torch.Tensor, rows: Optional[torch.Tensor], mask: torch.Tensor, gate: torch.Tensor,
                         place: torch.Tensor, prob: Optional[torch.Tensor] = None, drows: Optional[torch.Tensor] = None,
                         dgate: Optional[torch.Tensor] = None, dlogits: Optional[torch.Tensor] = None, stream=None) -> None:
        """The gradients of ``combine`` (eat_combine_backward), written to the
        tensors given: of its rows, of the gates, and through the gates'
        renormalisation and the softmax (``prob`` from ``route``) of the router's
        scaled scores, as ``balance_loss`` gives its own."""
        T, E, d, dev = mask.shape[0], self.params.E, self.params.d_model, dy.device
        some = rows if rows is not None else drows
        cap = 0 if some is None else some.shape[0]
        _expect("dy", dy, self._act(), (T, d), dev)
        _expect("rows", rows, self._act(), (cap, d), dev)
        self._expect_mask(mask, T, dev)
        _expect("gate", gate, torch.float32, (T, E), dev)
        _expect("place", place, torch.int32, (T, E), dev)
        _expect("prob", prob, torch.float32, (T, E), dev)
        _expect("drows", drows, self._act(), (cap, d), dev)
        _expect("dgate", dgate, torch.float32, (T, E), dev)
        _expect("dlogits", dlogits, torch.float32, (T, E), dev)
        if rows is None and (dgate is not None or dlogits is not None):
            raise ValueError("rows: the gates' gradients need them")
        with _calling_on(stream, dev):
            on = torch.cuda.current_stream(dev)
            L.eat_combine_backward(self.handle, dy, rows, cap, T, mask, gate, place, prob, drows, dgate, dlogits, on)
            _take_in(stream is not None, on, dy, rows, mask, gate, place, prob, drows, dgate, dlogits)

    def close(self) -> None:
        if self.handle:
            L.eat_destroy(self.handle)
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class PplSignal:
    """Running perplexity of S sequences through an LM head (Sec. 3.3's
    signal): ``step(h, target)`` returns the int8 trend for the sequences'
    next tokens (eat_ppl_trend)."""

    def __init__(self, S: int, w_vocab: torch.Tensor, device: str = "cuda"):
        self.S, self.w = int(S), w_vocab
        self.V, self.d = w_vocab.shape
        dev = torch.device(device)
        self.nll_sum = torch.zeros(S, dtype=torch.float64, device=dev)
        self.count = torch.zeros(S, dtype=torch.int32, device=dev)
        self.ppl_prev = torch.zeros(S, dtype=torch.float64, device=dev)
        self.trend = torch.zeros(S, dtype=torch.int8, device=dev)
        self.nll = torch.zeros(S, dtype=torch.float32, device=dev)
        self.ws = torch.empty(max(256, L.eat_ppl_workspace_size(S, self.d, self.V)), dtype=torch.uint8, device=dev)

    def reset(self, stream=None) -> None:
        L.eat_ppl_reset(self.S, self.nll_sum, self.count, self.ppl_prev, stream)

    def step(self, h: torch.Tensor, target: torch.Tensor, stream=None) -> torch.Tensor:
        L.eat_ppl_trend(h, self.S, self.d, self.w, self.V, target, self.nll_sum, self.count, self.ppl_prev,
                        self.trend, self.nll, self.ws, self.ws.numel(), stream)
        return self.trend


class CrossEntropy:
    """Cross entropy of an LM head ``w_vocab`` [V][d] bf16 (eat_ce_loss):
    ``loss(h, target)`` returns the loss [1] of the positions whose target is
    not ``ignore``; NLLs, their count and the gradients of ``h`` and of the
    head are written to the tensors given.  ``max_workspace``: bytes of
    workspace to stay under where a call can (the vocabulary is then taken in
    smaller pieces).  Calls of one object share its workspace: order them on
    one stream.  ``stream``: what a call is enqueued on (the current one); the
    tensors given have to be ready there (outside a capture they may be dropped once
    the call has returned), and what is returned is ready when it is."""

    def __init__(self, w_vocab: torch.Tensor, ignore: int = -100, max_workspace: Optional[int] = None):
        if w_vocab.dim() != 2:
            raise ValueError("w_vocab: expected [V][d]")
        _expect("w_vocab", w_vocab, torch.bfloat16, tuple(w_vocab.shape))
        self.w, self.ignore, self.max_workspace = w_vocab, int(ignore), max_workspace
        self.V, self.d = w_vocab.shape
        self._ws = _Workspace(w_vocab.device)

    def _need(self, T: int, grads: int) -> int:
        need, least = L.eat_ce_workspace_size(T, self.d, self.V, grads)
        return need if self.max_workspace is None else min(need, max(least, int(self.max_workspace)))

    def workspace(self, T: int, grads: int, stream=None) -> torch.Tensor:
        """What a call of T positions gets (its size decides the pieces: it does
        not depend on earlier calls)."""
        need = self._need(T, grads)
        with _calling_on(stream, self.w.device):
            return self._ws.get(need, torch.cuda.current_stream(self.w.device))[:need]

    def loss(self, h: torch.Tensor, target: torch.Tensor, mean: bool = True, scale: float = 1.0,
             nll: Optional[torch.Tensor] = None, count: Optional[torch.Tensor] = None,
             dh: Optional[torch.Tensor] = None, dw: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        T = h.shape[0]
        dev = self.w.device
        _expect("h", h, torch.bfloat16, (T, self.d), dev)
        _expect("target", target, torch.int32, (T,), dev)
        _expect("nll", nll, torch.float32, (T,), dev)
        _expect("count", count, torch.int32, (1,), dev)
        _expect("dh", dh, torch.bfloat16, (T, self.d), dev)
        _expect("dw", dw, torch.bfloat16, (self.V, self.d), dev)
        caller = torch.cuda.current_stream(dev) if stream is not None else None
        with _calling_on(stream, dev):
            out = torch.empty(1, dtype=torch.float32, device=dev)
            need = self._need(T, (L.EAT_CE_DH if dh is not None else 0) | (L.EAT_CE_DW if dw is not None else 0))
            on = torch.cuda.current_stream(dev)
            ws = self._ws.get(need, on)
            L.eat_ce_loss(h, T, self.d, self.w, self.V, target, self.ignore, int(mean), scale, out, nll, count, dh, dw, ws,
                          need, on)
            _take_in(stream is not None, on, h, self.w, target, nll, count, dh, dw)
        _hand_out(stream, caller, out)
        return out


class Fp8Matrix:
    """A matrix ``w`` [M][K] or matrices [groups][M][K] (bf16 or fp32) held in 8
    bits with a power of two per 128 x 128 block (eat_fp8_quantize): ``q`` e4m3
    [groups][M][K padded to 128], ``scale`` e8m0 bytes.  ``product(x)`` is x . w^T
    with the rows rounded the same way, a power of two per 128 elements; with
    ``gradients`` the transposed numbers are kept too, for ``product_backward``.
    Calls of one object share its workspace: order them on one stream.
    ``stream``: what a call is enqueued on (the current one); the tensors given
    have to be ready there (and, outside a capture, may be dropped once the call has
    returned, as the object may), and what is returned is ready when it is."""

    def __init__(self, w: torch.Tensor, gradients: bool = False, stream=None):
        if w.dim() not in (2, 3):
            raise ValueError("w: expected [M][K] or [groups][M][K]")
        self.groups, self.M, self.K = (1, *w.shape) if w.dim() == 2 else tuple(w.shape)
        _expect("w", w, (torch.bfloat16, torch.float32), tuple(w.shape))
        self.device = w.device
        dtype = L.EAT_BF16 if w.dtype == torch.bfloat16 else L.EAT_F32
        caller = torch.cuda.current_stream(w.device) if stream is not None else None
        with _calling_on(stream, w.device):
            on = torch.cuda.current_stream(w.device)
            made = []
            for rows, cols in ((self.M, self.K), (self.K, self.M))[:1 + bool(gradients)]:
                L.eat_fp8_size(self.groups, rows, cols)
                q = torch.empty(self.groups, rows, -(-cols // 128) * 128, dtype=torch.float8_e4m3fn, device=w.device)
                s = torch.empty(self.groups, -(-rows // 128), -(-cols // 512) * 4, dtype=torch.uint8, device=w.device)
                L.eat_fp8_quantize(w, dtype, self.groups, self.M, self.K, len(made) // 2, q, s, on)
                made += [q, s]
            _take_in(stream is not None, on, w)
        self._home = on.cuda_stream
        _hand_out(stream, caller, *made)
        self.q, self.scale = made[:2]
        self.qt, self.scale_t = made[2:] if gradients else (None, None)
        self._ws = _Workspace(w.device)

    def _run(self, x, offsets, token, out, q, scale, M, K, names, stream):
        dev, src = self.device, x.shape[0]
        rows = src if token is None else token.shape[0]
        _expect(names[0], x, torch.bfloat16, (src, K), dev)
        _expect("offsets", offsets, torch.int32, (self.groups + 1,), dev)
        _expect("token", token, torch.int32, (rows,), dev)
        _expect(names[1], out, (torch.bfloat16, torch.float32), (rows, M), dev)
        if offsets is None and self.groups != 1:
            raise ValueError("offsets: several matrices need them")
        caller = torch.cuda.current_stream(dev) if stream is not None else None
        with _calling_on(stream, dev):
            given = out is not None
            if not given:
                out = torch.empty(rows, M, dtype=torch.bfloat16, device=dev)
            need = L.eat_fp8_product_workspace_size(src, rows, self.groups, M, K)
            on = torch.cuda.current_stream(dev)
            ws = self._ws.get(need, on)
            L.eat_fp8_product(x, src, token, offsets, rows, q, scale, self.groups, M, K, out,
                              L.EAT_BF16 if out.dtype == torch.bfloat16 else L.EAT_F32, ws, need, on)
            _take_in(on.cuda_stream != self._home, on, q, scale)
            _take_in(stream is not None, on, x, offsets, token, out if given else None)
        if not given:
            _hand_out(stream, caller, out)
        return out

    def product(self, x: torch.Tensor, offsets: Optional[torch.Tensor] = None, token: Optional[torch.Tensor] = None,
                out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """out [rows][M] (bf16, or the type of ``out``) of the rows x [rows][K] bf16,
        or of x[token]; ``offsets`` [groups+1] int32: where each matrix's rows begin
        (``EatLayer.sort``).  Rows outside the groups are not written."""
        return self._run(x, offsets, token, out, self.q, self.scale, self.M, self.K, ("x", "out"), stream)

    def product_backward(self, dy: torch.Tensor, offsets: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                         stream=None) -> torch.Tensor:
        """dx [rows][K] of dy [rows][M] bf16, the weights held constant: dy . w, dy rounded as rows are."""
        if self.qt is None:
            raise ValueError("made without gradients")
        return self._run(dy, offsets, None, dx, self.qt, self.scale_t, self.K, self.M, ("dy", "dx"), stream)


class Fp8Experts:
    """A layer's SwiGLU experts in 8 bits (eat_fp8_experts_*): ``weights`` as
    EatLayer's (w1, w3 [E][F][d], w2 [E][d][F], bf16, row-major), of which the
    object keeps e4m3 numbers with a power of two per 128 x 128 block, with
    ``gradients`` their transposes too.  They are constants: ``backward`` gives
    the rows' gradient.  Tiles, memory and the limit of 2^24 rows go by the length of
    ``token``, not by the rows that ``offsets`` end at.  Streams and workspace as
    Fp8Matrix's."""

    def __init__(self, weights: Dict[str, torch.Tensor], gradients: bool = False, stream=None):
        w1, w3, w2 = weights["w1"], weights["w3"], weights["w2"]
        if w1.dim() != 3:
            raise ValueError("w1: expected [E][F][d]")
        self.E, self.F, self.d = w1.shape
        dev = self.device = w1.device
        _expect("w1", w1, torch.bfloat16, (self.E, self.F, self.d))
        _expect("w3", w3, torch.bfloat16, (self.E, self.F, self.d), dev)
        _expect("w2", w2, torch.bfloat16, (self.E, self.d, self.F), dev)
        self.gradients, self.handle = bool(gradients), 0
        self.handle = L.eat_create(L.eat_params_default(mode="topk", E=self.E, d_model=self.d, d_ffn=self.F, top_k=1), 1 << 24)
        caller = torch.cuda.current_stream(dev) if stream is not None else None
        with _calling_on(stream, dev):
            on = torch.cuda.current_stream(dev)
            self.buf = torch.empty(L.eat_fp8_experts_size(self.handle, int(gradients)), dtype=torch.uint8, device=dev)
            L.eat_fp8_experts_quantize(self.handle, w1, w3, w2, int(gradients), self.buf, on)
            _take_in(stream is not None, on, w1, w3, w2)
        self._home = on.cuda_stream
        _hand_out(stream, caller, self.buf)
        self._ws = _Workspace(dev)

    def forward(self, x: torch.Tensor, offsets: torch.Tensor, token: torch.Tensor, y: Optional[torch.Tensor] = None,
                saved: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """The experts' rows y [rows][d] of the tokens x [T][d], with ``offsets`` and
        ``token`` from ``EatLayer.sort``; what ``backward`` needs is written to
        ``saved`` [rows][2 F] bf16.  Rows behind the last segment are not written."""
        T, rows, dev = x.shape[0], token.shape[0], self.device
        _expect("x", x, torch.bfloat16, (T, self.d), dev)
        _expect("offsets", offsets, torch.int32, (self.E + 1,), dev)
        _expect("token", token, torch.int32, (rows,), dev)
        _expect("y", y, torch.bfloat16, (rows, self.d), dev)
        _expect("saved", saved, torch.bfloat16, (rows, 2 * self.F), dev)
        caller = torch.cuda.current_stream(dev) if stream is not None else None
        with _calling_on(stream, dev):
            given = y is not None
            if not given:
                y = torch.empty(rows, self.d, dtype=torch.bfloat16, device=dev)
            need = L.eat_fp8_experts_workspace_size(self.handle, T, rows, 0)
            on = torch.cuda.current_stream(dev)
            ws = self._ws.get(need, on)
            L.eat_fp8_experts_forward(self.handle, x, T, token, offsets, rows, self.buf, y, saved, ws, need, on)
            _take_in(on.cuda_stream != self._home, on, self.buf)
            _take_in(stream is not None, on, x, offsets, token, saved, y if given else None)
        if not given:
            _hand_out(stream, caller, y)
        return y

    def backward(self, dy: torch.Tensor, saved: torch.Tensor, offsets: torch.Tensor, dx: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
        """dx [rows][d] of the sorted tokens from dy [rows][d] (dx may be dy)."""
        if not self.gradients:
            raise ValueError("made without gradients")
        rows, dev = dy.shape[0], self.device
        _expect("dy", dy, torch.bfloat16, (rows, self.d), dev)
        _expect("saved", saved, torch.bfloat16, (rows, 2 * self.F), dev)
        _expect("offsets", offsets, torch.int32, (self.E + 1,), dev)
        _expect("dx", dx, torch.bfloat16, (rows, self.d), dev)
        caller = torch.cuda.current_stream(dev) if stream is not None else None
        with _calling_on(stream, dev):
            given = dx is not None
            if not given:
                dx = torch.empty(rows, self.d, dtype=torch.bfloat16, device=dev)
            need = L.eat_fp8_experts_workspace_size(self.handle, 0, rows, 1)
            on = torch.cuda.current_stream(dev)
            ws = self._ws.get(need, on)
            L.eat_fp8_experts_backward(self.handle, dy, offsets, rows, self.buf, saved, dx, ws, need, on)
            _take_in(on.cuda_stream != self._home, on, self.buf)
            _take_in(stream is not None, on, dy, saved, offsets, dx if given else None)
        if not given:
            _hand_out(stream, caller, dx)
        return dx

    def close(self) -> None:
        if self.handle:
            L.eat_destroy(self.handle)
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def layerwise_caps(n_layers: int, lower: int, k_lower: int, k_upper: int):
    """Per-layer caps K for layer-wise sparsity: the paper's layer analysis
    (Sec. 4) finds lower layers' experts less critical than higher layers',
    so the lower ``lower`` layers get ``k_lower`` and the rest ``k_upper``."""
    return [k_lower if l < lower else k_upper for l in range(n_layers)]


class EatStack:
    """Stacked layers (one EatLayer each, own accounts) with their d x d
    mixing matrices, run one decode step at a time by eat_stack_forward."""

    def __init__(self, params, max_tokens: int, weights, mixes, device: str = "cuda"):
        self.layers = [EatLayer(p, max_tokens, w, device) for p, w in zip(params, weights)]
        self.mixes = list(mixes)
        self.device = torch.device(device)
        self._ws: Optional[torch.Tensor] = None
        self._arr = None

    def _entries(self):
        out = []
        for lay, m in zip(self.layers, self.mixes):
            w = lay.w
            out.append(L.eat_stack_layer_t(lay.handle, L._ptr(w["w_router"]), L._ptr(w["w1"]), L._ptr(w["w3"]),
                                           L._ptr(w["w2"]), L._ptr(w.get("ws1")), L._ptr(w.get("ws3")),
                                           L._ptr(w.get("ws2")), L._ptr(m), lay.acc))
        return L.stack_layers(out)

    def reset_accounts(self, stream=None) -> None:
        for lay in self.layers:
            lay.reset_accounts(stream)

    def forward(self, x: torch.Tensor, trend: Optional[torch.Tensor] = None, h_out: Optional[torch.Tensor] = None,
                masks_out: Optional[torch.Tensor] = None, probs_out: Optional[torch.Tensor] = None,
                rms_eps: float = 1e-6, stream=None) -> torch.Tensor:
        T = x.shape[0]
        if h_out is None:
            h_out = torch.empty_like(x)
        if self._arr is None:
            self._arr = self._entries()
        n = len(self.layers)
        need = L.eat_stack_workspace_size(self._arr, n, T)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        L.eat_stack_forward(self._arr, n, x, T, trend, rms_eps, h_out, masks_out, probs_out, self._ws,
                            self._ws.numel(), stream)
        return h_out

    def close(self) -> None:
        for lay in self.layers:
            lay.close()


def capture(fn, warmup: int = 2) -> "torch.cuda.CUDAGraph":
    """Capture ``fn()`` -- calls into the library, which only enqueue on the
    current stream and never allocate or synchronise -- into a HIP graph.
    ``warmup`` eager calls first size every workspace (they run the layers,
    so reset accounts afterwards where that matters).  Replay with
    ``graph.replay()`` after copying new inputs into the tensors ``fn``
    reads; account updates inside the graph act on the live account
    tensors, so replays carry the history forward."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(warmup):
            fn()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fn()
    return g


def to_device(weights: Dict, device: str = "cuda") -> Dict[str, torch.Tensor]:
    """Upload generator output (fp32 arrays or bf16 bit patterns as uint16)
    to device tensors (torch.bfloat16 for bf16)."""
    import numpy as np
    out = {}
    for k, v in weights.items():
        t = torch.from_numpy(np.ascontiguousarray(v))
        if v.dtype == np.uint16:
            t = t.view(torch.bfloat16)
        out[k] = t.to(device)
    return out


# expert matrices and the (groups, M, K) view eat_pack_weights takes of each
_PACK_SHAPES = {"w1": ("E", "F", "d"), "w3": ("E", "F", "d"), "w2": ("E", "d", "F"),
                "ws1": (1, "Fs", "d"), "ws3": (1, "Fs", "d"), "ws2": (1, "d", "Fs")}


def pack_weights(weights: Dict[str, torch.Tensor], stream=None) -> Dict[str, torch.Tensor]:
    """Device weight dict -> the same dict with the bf16 expert matrices
    (w1, w3, w2 and the shared ws1, ws3, ws2) in the packed layout (new
    tensors, written by eat_pack_weights); for layers created with
    weight_layout = EAT_LAYOUT_PACKED.  Other entries are passed through."""
    out = dict(weights)
    for name, w in weights.items():
        if name not in _PACK_SHAPES or w is None:
            continue
        if w.dtype != torch.bfloat16 or w.dim() not in (2, 3):
            raise ValueError(f"{name}: packing needs a bf16 [groups][M][K] or [M][K] tensor")
        g, M, K = (1, *w.shape) if w.dim() == 2 else tuple(w.shape)
        dst = torch.empty_like(w)
        L.eat_pack_weights(w.contiguous(), g, M, K, dst, stream)
        out[name] = dst
    return out
