"""How the streaming attention kernel cuts a request into units, as host code: for every mask the units of a block of query rows hold all
keys that its rows see, at any window up to the largest an int holds."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2602_06822_b200")
TOP = 2 ** 31 - 1

SOURCE = r"""
#include <limits.h>
#include "pop_kv_attn.cuh"
template <int ROWS, int TOKENS> static void put(const KvAttnArgs& A, const KvRequest& q, int* out) {
    const Units u = request_units<ROWS, TOKENS>(A, q);
    out[0] = u.first; out[1] = u.count; out[2] = u.row_blocks;
}
extern "C" void units(int rows, int tokens, int ratio, int n, int len, int pos0, int causal, int window, int* out) {
    KvAttnArgs A = {};
    A.ratio = ratio; A.causal = causal; A.window = window; A.prompt_rows = INT_MAX;
    const KvRequest q = {0, n, len, pos0};
    if (rows == 8 && tokens == 32) put<8, 32>(A, q, out);
    else if (rows == 8) put<8, 16>(A, q, out);
    else put<16, 16>(A, q, out);
    out[3] = kv_first(A, pos0);
    out[4] = kv_first(A, pos0 + n - 1);
}
"""


@pytest.fixture(scope="module")
def units(tmp_path_factory):
    d = tmp_path_factory.mktemp("units")
    src, so = str(d / "units.cu"), str(d / "units.so")
    with open(src, "w") as f:
        f.write(SOURCE)
    subprocess.run([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-Xcompiler",
                    "-fPIC", "-shared", "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(PKG, "csrc"), "-o", so, src], check=True)
    fn = C.CDLL(so).units

    def call(rows, tokens, ratio, n, length, pos0, causal, window):
        out = (C.c_int * 5)()
        fn(rows, tokens, ratio, n, length, pos0, int(causal), window, out)
        return list(out)
    return call


@pytest.mark.parametrize("rows,tokens", [(8, 32), (8, 16), (16, 16)])
@pytest.mark.parametrize("ratio", [1, 3, 5, 8])
def test_units_hold_every_visible_key(units, rows, tokens, ratio):
    for length, n in ((517, 517), (300, 64), (64, 200), (0, 40), (5000, 17), (33, 1)):
        for causal in (True, False):
            for window in (0, 1, 31, 256, 4999, 2 ** 30, TOP - tokens - rows, TOP - 38, TOP - 1, TOP):
                pos0 = length - n
                first, count, blocks, at0, at1 = units(rows, tokens, ratio, n, length, pos0, causal, window)
                assert blocks == -(-n * ratio // rows)
                assert at0 == (max(0, pos0 - window + 1) if window else 0) and at1 == (max(0, length - window) if window else 0)
                assert 1 <= count <= max(1, -(-length // tokens))
                for b in range(blocks):
                    p0, p1 = pos0 + b * rows // ratio, pos0 + (min(n * ratio, (b + 1) * rows) - 1) // ratio
                    lo = max(0, p0 - window + 1) if window else 0
                    hi = min(length, max(0, p1 + 1)) if causal else length
                    start = min(lo, length) // tokens if first < 0 else first
                    if lo < hi:
                        assert start * tokens <= lo and hi <= (start + count) * tokens
