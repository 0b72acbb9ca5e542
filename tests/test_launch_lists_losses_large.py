"""The calls of tests/ce_large.py go to the 256 x 256 tiles."""
import os
import re
import shutil

import pytest

from paper_2609_33614_amd import _lib as L
from tests.ce_large import CALLS
from tests.launch_list_losses import list_launches

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH) or shutil.which("g++") is None,
                                reason="needs libeat.so and g++")
LSE, GRAD, PART, ROWS = 0, 1, 2, 3


def test_large_calls_take_the_large_tiles(tmp_path, monkeypatch):
    names = list(CALLS)
    got = list_launches(tmp_path, [dict(kind="ce", T=T, d=d, V=V, dh=1, dw=1, least=least) for T, d, V, least, _ in CALLS.values()],
                        monkeypatch)
    seen = set()
    for name, g in zip(names, got):
        T, d, V, least, _ = CALLS[name]
        pieces = -(-V // 4096) if least else 1
        tiles = [(int(m[1]), int(m[2])) for k, _ in g["kernels"] if (m := re.search(r"Tile<(\d+).*?>, \w+, \w+, (\d), 0", k))]
        want = [(256, LSE)] + [(256, PART)] * pieces + [(256, GRAD)] * (pieces - 1)
        assert sorted(t for t in tiles if t[1] != ROWS) == sorted(want), (name, tiles)
        assert sum("scale_kernel<256>" in k for k, _ in g["kernels"]) == 1
        seen |= set(tiles)
    assert seen >= {(256, LSE), (256, GRAD), (256, PART), (256, ROWS)}
