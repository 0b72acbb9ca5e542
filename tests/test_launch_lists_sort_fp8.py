"""What the host code of sort, combine and the 8-bit products launches, listed
on the CPU (tests/launch_list_sort_fp8.py)."""
import os
import shutil

import pytest

from paper_2609_33614_amd import _lib as L
from tests.launch_list_sort_fp8 import list_launches

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH) or shutil.which("g++") is None,
                                reason="needs libeat.so and g++")

LAYER = dict(mode="topk", top_k=1, d_ffn=64)


def test_grids_of_the_longest_calls_can_be_launched(tmp_path, monkeypatch):
    """A grid has fewer than 2^32 threads along x and 65536 workgroups along y and z, up to
    the most tokens, rows and matrices that the entry points take."""
    calls = []
    for T in (1, 256, 257, 16384, 1 << 24, (1 << 24) - 77):
        for E, d in ((1, 64), (65, 64), (256, 64), (256, 8192), (8, 4096)):
            cap = min(T * E, (1 << 31) - 1)
            for kind in ("sort", "combine"):
                for back in (0, 1):
                    calls.append(dict(LAYER, kind=kind, T=T, rows=cap, back=back, E=E, d_model=d))
    for M, K in ((8, 8), (8, 1 << 20), (1 << 20, 8), (1 << 15, 32768), (14336, 4096)):
        for groups in (1, 256):
            for t in (0, 1):
                if M * -(-K // 128) * 128 < 1 << 31 and K * -(-M // 128) * 128 < 1 << 31:
                    calls.append(dict(kind="quantize", T=groups, M=M, K=K, t=t, dtype=L.EAT_BF16))
            for n, rows in ((1, 1), (64, 64), (1 << 24, 1 << 24), (1, 1 << 24), (1 << 24, 7)):
                for out in (L.EAT_BF16, L.EAT_F32):
                    if M * -(-K // 128) * 128 < 1 << 31:
                        calls.append(dict(kind="product", T=n, rows=rows, groups=groups, M=M, K=K, out=out))
    for E, d, F in ((1, 64, 64), (256, 64, 64), (8, 4096, 14336), (256, 8192, 8192)):
        for T, rows in ((1, 2), (300, 600), (1 << 24, 1 << 24), (1 << 20, 1 << 24)):
            for back, saved in ((0, 0), (0, 1), (1, 1)):
                calls.append(dict(LAYER, kind="experts", T=T, rows=rows, saved=saved, back=back, E=E, d_model=d, d_ffn=F))
    for c, g in zip(calls, list_launches(tmp_path, [dict(c) for c in calls], monkeypatch)):
        assert g["kernels"], c
        for name, (x, y, z, threads) in g["kernels"]:
            assert 0 < x * threads < 1 << 32 and 0 < y < 1 << 16 and 0 < z < 1 << 16, (c, name, x, y, z)


def test_few_tokens_are_sorted_by_one_launch(tmp_path, monkeypatch):
    calls = [dict(LAYER, kind="sort", T=T, rows=T * E, back=0, E=E, d_model=128) for T in (1, 64, 256) for E in (1, 64, 256)]
    for c, g in zip(calls, list_launches(tmp_path, [dict(c) for c in calls], monkeypatch)):
        assert len(g["kernels"]) == 1, (c, g)
