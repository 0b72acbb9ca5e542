"""Loads of the losses' GEMM for few counted rows in long calls: their second
parts are further rows of dh's product and further reduction elements of dW's."""
import shutil

import pytest

from tests.loss_gemm_loads import run

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ missing")

CALLS = """
    auto few = [](auto tile, int T, int n, int d, int V, int rows_pad, int piece, int pool) {
        using C = decltype(tile);
        int32_t head[4] = {n, (n + 63) / 64 * 64, 0, 0}, slices = 0;
        long total = 0;
        for (int v0 = 0; v0 < V; v0 += piece) {
            const int nv = min(piece, V - v0);
            GemmArgs a{};
            a.a = A; a.lda = d; a.na = d; a.a_rows = nv; a.b = B; a.ldb = piece; a.nb = max(T, 128); a.nb_dev = head; a.K = nv;
            a.planes = 1; a.pool_rows = pool; a.slice_chunks = min(piece, V + 63) / 64; a.slices_out = &slices;
            total += launch<C, true, false, PART>(a, 2ull * nv * d, 2ull * rows_pad * piece);
            GemmArgs w{};
            w.a = A; w.lda = d; w.na = d; w.a_rows = 1 << 30; w.b = B; w.ldb = piece; w.nb = nv;
            w.K = rows_pad; w.k_dev = head + 1; w.k_times = 1; w.planes = 1; w.splits = 1;
            const long here = launch<C, true, true, ROWS>(w, 2ull * rows_pad * d, 2ull * rows_pad * piece);
            if (n && !here) fail("dW without loads", n);
            total += here;
        }
        if (slices * (n <= 64 ? 64 + n : n) > pool) fail("slices past their rows", slices);
        printf("few T %d n %d: %ld loads\\n", T, n, total);
    };
    for (int T : {65, 100, 128, 200, 256})
        for (int n : {0, 1, 2, 63, 64, 65}) {
            few(Mid{}, T, n, 320, 1000, 256, 1024, 4096);
            few(Big{}, T, n, 320, 1000, 256, 1024, 4096);
            few(Mid{}, T, n, 192, 4096 * 2 + 300, 256, 4096, 4096);
            few(Big{}, T, n, 192, 4096 * 2 + 300, 256, 4096, 4096);
        }
    for (int n : {0, 1, 64, 65, 2000}) {
        few(Mid{}, 2100, n, 512, 16387, 2304, 16640, 16384);
        few(Big{}, 2100, n, 512, 16387, 2304, 4096, 16384);
    }
"""


def test_every_load_is_in_bounds(tmp_path):
    rc, out = run(tmp_path, CALLS)
    assert rc == 0 and "ALL IN BOUNDS" in out, out[-500:]


def test_the_check_sees_second_parts_that_are_not_there(tmp_path):
    rc, out = run(tmp_path, CALLS.replace("2ull * rows_pad * d, 2ull * rows_pad * piece", "2ull * 64 * d, 2ull * rows_pad * piece"))
    assert rc == 1 and "BAD load" in out, out[-500:]
