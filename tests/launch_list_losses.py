"""The kernels of the losses' calls, listed on the CPU (tests/launch_list.py
does the same for the layer's): {"kind": "ce", "T", "d", "V", "dh", "dw"
and "least" (1: the smallest workspace)} or {"kind": "balance", "T", "dx",
"dw", "dz", "padded", **eat_params_default overrides}."""
from tests import launch_list as LL

CALLS = r"""
    if kind == "ce":                                  # (arrays far apart: overlaps are refused)
        d, V, A = call["d"], call["V"], 1 << 50
        dh, dw = (5 * A if call["dh"] else None), (6 * A if call["dw"] else None)
        most, least = L.eat_ce_workspace_size(T, d, V, (1 if dh else 0) | (2 if dw else 0))
        n = least if call.get("least") else most
        L.eat_ce_loss(A, T, d, 2 * A, V, 3 * A, -100, 1, 1.0, 4 * A, None, None, dh, dw, 7 * A, n, stream=0)
    elif kind == "balance":
        A = 1 << 50
        dz, dx, dw = (at * A if call.pop(k) else None for at, k in ((5, "dz"), (6, "dx"), (7, "dw")))
        valid = 10 * A if call.pop("padded") else None
        p = L.eat_params_default(**call)
        h = L.eat_create(p, T)
        n = L.eat_balance_workspace_size(h, T)
        L.eat_balance_loss(h, A, T, 2 * A, 3 * A, 4 * A, valid, 0.01, 0.0, 8 * A, None, None, dz, dx, dw, 9 * A, n, stream=0)
        L.eat_destroy(h)
    elif kind == "ppl":
"""
CHILD = LL.CHILD.replace('    if kind == "ppl":\n', CALLS[1:])
assert CHILD != LL.CHILD


def list_launches(tmp_path, calls, monkeypatch):
    monkeypatch.setattr(LL, "CHILD", CHILD)
    return LL.list_launches(tmp_path, calls)
