"""Every load of the losses' GEMM stays in its operands (tests/loss_gemm_loads.py)."""
import shutil

import pytest

from tests.loss_gemm_loads import HEADER, run

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ missing")

CE = """
    for (int n : {0, 1, 40, 64}) ce<Small>(64, n, 320, 1000, 64, 1024, 1024);
    for (int n : {0, 1, 100, 128, 200, 256}) ce<Mid>(256, n, 320, 1000, 256, 1024, 4096);
    for (int n : {0, 1, 255, 257, 513}) {
        ce<Big>(513, n, 512, 1000, 768, 1024, 12288);
        ce<Mid>(513, n, 512, 1000, 768, 1024, 12288);
    }
    ce<Big>(300, 270, 192, 4096 * 4 + 1, 512, 4096, 8192);
    ce<Small>(40, 36, 192, 4096 * 2 + 33, 64, 4096, 1024);
    ce<Big>(2000, 2000, 128, 300, 2048, 512, 16384);
    ce<Mid>(1025, 1025, 256, 2050, 1280, 2304, 16384);
    ce<Big>(5003, 3752, 256, 5003, 5120, 5120, 16384);
    ce<Small>(1, 1, 64, 1, 64, 256, 1024);
    ce<Big>(300, 300, 64, 1, 512, 256, 8192);
"""
BALANCE = """
    for (int n : {1, 0, 63, 64, 65, 700, 2300}) balance(2300, n, 60, 1024, 8, true, 1, 3, 0x010);
    for (int n : {1, 0, 640, 2300}) balance(2300, n, 60, 1024, 8, false, 3, 6, 0x211000);
    for (int n : {0, 1, 770, 1100}) {
        balance(1100, n, 200, 640, 4, true, 1, 3, 0x010);
        balance(1100, n, 200, 640, 4, false, 3, 6, 0x211000);
    }
    balance(2111, 2111, 64, 1024, 8, false, 1, 3, 0x010);
    balance(257, 257, 256, 2112, 1, false, 1, 3, 0x010);
    balance(64, 64, 250, 8640, 1, false, 1, 3, 0x010);
    balance(20000, 20000, 7, 1024, 64, false, 1, 3, 0x010);
    balance(4111, 4111, 130, 320, 16, false, 1, 3, 0x010);
    balance(8000, 6400, 60, 2048, 32, true, 1, 3, 0x010);
"""


@pytest.mark.parametrize("calls", [CE, BALANCE], ids=["ce", "balance"])
def test_every_load_is_in_bounds(tmp_path, calls):
    rc, out = run(tmp_path, calls)
    assert rc == 0 and "ALL IN BOUNDS" in out, out[-500:]


@pytest.mark.parametrize("what,old,new,calls", [
    # a workgroup without chunks loads all the same (one token of 2300, eight slices)
    ("empty items", "    if (!ended) {", "    if (true) {", "    balance(2300, 1, 60, 1024, 8, true, 1, 3, 0x010);"),
    # the last chunk of an operand of 1000 rows reads whole
    ("tail rows", "off[j] -= __umul24(max(k - k_last, 0), ldbytes);", ";", "    ce<Mid>(256, 200, 320, 1000, 256, 1024, 4096);"),
    # the columns of a tile past the operand's width
    ("tail columns", "min(first + 8 * v, count - 8)", "(first + 8 * v)", "    ce<Mid>(256, 200, 320, 1000, 256, 1024, 4096);"),
])
def test_the_check_sees_a_load_out_of_bounds(tmp_path, what, old, new, calls):
    header = open(HEADER).read()
    assert old in header
    rc, out = run(tmp_path, calls, header.replace(old, new))
    assert rc == 1 and "BAD load" in out, out[-500:]
