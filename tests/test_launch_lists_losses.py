"""What the host code of the losses launches, listed on the CPU (tests/launch_list_losses.py)."""
import os
import shutil

import pytest

from paper_2609_33614_amd import _lib as L
from tests.launch_list_losses import list_launches

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH) or shutil.which("g++") is None,
                                reason="needs libeat.so and g++")


def test_grids_of_the_longest_calls_can_be_launched(tmp_path, monkeypatch):
    """A grid has fewer than 2^32 threads along x and 65536 workgroups along y,
    up to the most tokens and positions that the entry points take."""
    calls = []
    for T in (1 << 24, (1 << 24) - 77, 1 << 23):
        for E, d in ((1, 64), (65, 64), (8, 4096), (64, 4096), (65, 4096), (256, 256), (256, 4096), (8, 8192)):
            for bf16 in (0, 1):
                for padded in (0, 1):
                    calls.append(dict(kind="balance", T=T, dz=1, dx=1, dw=1, padded=padded, mode=1, E=E, top_k=1, d_model=d,
                                      d_ffn=64, act_dtype=bf16, expert_dtype=bf16))
    for T in (1 << 20, (1 << 20) - 77):
        for d, V in ((64, 1), (64, 1 << 24), (65536, 1000), (4096, 128256), (65536, 1 << 22)):
            for least in (0, 1):
                calls.append(dict(kind="ce", T=T, d=d, V=V, dh=1, dw=1, least=least))
    for c, g in zip(calls, list_launches(tmp_path, [dict(c) for c in calls], monkeypatch)):
        assert g["kernels"], c
        for name, (x, y, z, threads) in g["kernels"]:
            assert 0 < x * threads < 1 << 32 and 0 < y < 1 << 16 and z == 1, (c, name, x, y)
