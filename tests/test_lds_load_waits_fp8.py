"""The waits before the loads to LDS of the 8-bit products (tests/test_lds_load_waits.py has the rules)."""
import shutil
import os

import pytest

from paper_2609_33614_amd import build as B
from tests import test_lds_load_waits as W

pytestmark = pytest.mark.skipif(not os.path.exists(B.HIPCC) or shutil.which("hipcc") is None, reason="hipcc missing")


def test_loads_to_lds_keep_their_waits(tmp_path):
    W.test_loads_to_lds_keep_their_waits("fp8.hip", tmp_path)
