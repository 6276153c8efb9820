"""Launch shapes of the projections over 4-bit weights, walked over everything that the calls allow.  The header that chooses them is
plain C++: it is compiled here with the host compiler and called without a GPU."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_27591_b200", "csrc")

SOURCE = r"""
#include "prox_w4_plan.h"
using namespace prox::w4;
static RowsPlan plan_of(int tiles, int K, int tokens, int words, int sms) {
  return plan_rows(tiles, K, tokens, words, (tokens + 1) / 2, sms, [sms](int S) { return sms / S; });
}
extern "C" {
int tokens_of_a_pass(int tiles, int K, int B, int words, int sms) { return linear_pass(B, K, words, [=](int n) { return plan_of(tiles, K, n, words, sms); }); }
int shape(int tiles, int K, int tokens, int words, int sms, int* out) {
  const RowsPlan p = plan_of(tiles, K, tokens, words, sms);
  out[0] = p.S; out[1] = p.WM; out[2] = p.WK; out[3] = p.stages; out[4] = p.R;
  return p.grid;
}
// 0, or the first token count (B >= tokens asked for a pass) for which a launch would be empty or outside its limits
int walk(int tiles, int K, int most, int words, int sms) {
  const int C = (K + 127) / 128;
  for (int B = 1; B <= most; ++B) {
    const int per = tokens_of_a_pass(tiles, K, B, words, sms);
    if (per < 1 || per > kMaxPass || per > B) return B;
    for (int n : {per, B % per ? B % per : per}) {
      const RowsPlan p = plan_of(tiles, K, n, words, sms);
      const int Cs = p.S ? rows_share(C, p.S) : 0;
      if (p.grid < 1 || p.grid > sms || p.S < 1 || p.grid % p.S || p.WM < 1 || p.WK < 1 || p.WM * p.WK > kRowWarps) return B;
      if (p.smem > (size_t)kMaxSmem || (p.S > 1 && (p.R < 1 || Cs * (p.S - 1) >= C)) || (p.stages != 2 && p.stages != 3 && p.stages != kMaxStages)) return B;
    }
  }
  return 0;
}
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    src, out = d / "plan.cpp", d / "plan.so"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(out), str(src)], check=True)
    return C.CDLL(str(out))


@pytest.mark.parametrize("words", [1, 2, 4])
def test_every_projection_has_a_shape(lib, words):
    """Every K (all multiples of 32 up to 65536 share the shape of their number of 128-column chunks) and every number of tokens."""
    for K in range(128, 65536 + 1, 128):
        for tiles in (1, 9, 256, 8192):
            assert lib.walk(tiles, K, 17, words, 148) == 0, (K, tiles)


@pytest.mark.parametrize("sms", [132, 148, 160])
def test_every_ffn_has_a_shape(lib, sms):
    out = (C.c_int * 5)()
    for D in range(128, 16384 + 1, 128):
        for B in range(1, 9):
            for tiles in (1, 100, 8192):
                assert lib.shape(tiles, D, B, 4, sms, out) > 0, (D, B, tiles)


def test_rows_that_fill_neither_four_blocks_nor_eight(lib):
    """Groups of 32, 97 or 98 chunks: seven tokens do not fit in four blocks, and the last of eight would have no columns."""
    out = (C.c_int * 5)()
    for K in range(12320, 12544 + 1, 32):
        assert lib.shape(64, K, 7, 1, 148, out) == 0 and lib.shape(64, K, 8, 1, 148, out) == 0
        assert lib.tokens_of_a_pass(64, K, 8, 1, 148) == 6 and lib.tokens_of_a_pass(64, K, 7, 1, 148) == 6
        assert lib.tokens_of_a_pass(64, K, 3, 1, 148) == 3
