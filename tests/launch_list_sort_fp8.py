"""The kernels of the sort's, combine's and the 8-bit products' calls, listed on
the CPU (tests/launch_list.py does the same for the layer's): {"kind": "sort",
"T", "cap", "back", **eat_params_default overrides}, {"kind": "combine", "T",
"cap", "back", ...}, {"kind": "quantize", "T" (matrices), "M", "K", "t"}, {"kind":
"product", "T" (rows of x), "rows", "groups", "M", "K", "out"} or {"kind":
"experts", "T", "rows", "saved", "back", ...}."""
from tests import launch_list as LL

CALLS = r"""
    if kind in ("sort", "combine", "experts"):        # (arrays far apart: overlaps are refused)
        A = 1 << 50
        back, cap = call.pop("back"), call.pop("rows")
        saved = 9 * A if call.pop("saved", 0) else None
        p = L.eat_params_default(**call)
        h = L.eat_create(p, T)
        if kind == "sort" and back:
            L.eat_sort_backward(h, A, cap, T, 2 * A, 3 * A, 4 * A, stream=0)
        elif kind == "sort":
            n = L.eat_sort_workspace_size(h, T)
            L.eat_sort_tokens(h, A, T, 2 * A, cap, 3 * A, 4 * A, 5 * A, 6 * A, 7 * A, n, stream=0)
        elif kind == "combine" and back:
            L.eat_combine_backward(h, A, 2 * A, cap, T, 3 * A, 4 * A, 5 * A, 6 * A, 7 * A, 8 * A, 9 * A, stream=0)
        elif kind == "combine":
            L.eat_combine(h, A, cap, T, 2 * A, 3 * A, 4 * A, 5 * A, stream=0)
        elif back:
            n = L.eat_fp8_experts_workspace_size(h, 0, cap, 1)
            L.eat_fp8_experts_backward(h, A, 2 * A, cap, 3 * A, 4 * A, 5 * A, 6 * A, n, stream=0)
        else:
            n = L.eat_fp8_experts_workspace_size(h, T, cap, 0)
            L.eat_fp8_experts_forward(h, A, T, 2 * A, 3 * A, cap, 4 * A, 5 * A, saved, 6 * A, n, stream=0)
        L.eat_destroy(h)
    elif kind == "quantize":
        A = 1 << 50
        L.eat_fp8_quantize(A, call["dtype"], T, call["M"], call["K"], call["t"], 2 * A, 3 * A, stream=0)
    elif kind == "product":
        A = 1 << 50
        n = L.eat_fp8_product_workspace_size(T, call["rows"], call["groups"], call["M"], call["K"])
        L.eat_fp8_product(A, T, 2 * A if T != call["rows"] else None, 3 * A, call["rows"], 4 * A, 5 * A, call["groups"], call["M"], call["K"],
                          6 * A, call["out"], 7 * A, n, stream=0)
    elif kind == "ppl":
"""
CHILD = LL.CHILD.replace('    if kind == "ppl":\n', CALLS[1:])
assert CHILD != LL.CHILD


def list_launches(tmp_path, calls, monkeypatch):
    monkeypatch.setattr(LL, "CHILD", CHILD)
    return LL.list_launches(tmp_path, calls)
