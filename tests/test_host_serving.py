"""Host-side arithmetic of pages and attention, on the CPU: the kernels' index functions, taken
from their source text and built with g++."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2605_31105_amd import build as B

HEAD = r"""
#include <cstdint>
#include <cstdio>
#include <random>
#define __device__
#define __forceinline__ inline
static std::mt19937_64 rng(7);
static int64_t upto(int64_t n) { return (int64_t)(rng() %% (uint64_t)(n + 1)); }
// 0 .. n, spread over its logarithm
static int64_t log_upto(int64_t n) { return upto(n >> upto(40)); }
static long bad = 0;
#define CHECK(x) do { if (!(x) && bad++ < 5) printf("line %%d: %%s\n", __LINE__, #x); } while (0)
%s
int main() {
%s
  printf("bad = %%ld\n", bad);
  return bad != 0;
}
"""


def _function(src, name):
    """The function or struct `name` of a source in csrc, as text."""
    with open(os.path.join(B.CSRC, src)) as f:
        text = f.read()
    m = re.search(r"^(?:__device__ __forceinline__ )?(?:static )?\w[\w ]* %s(?:\([^)]*\))? \{.*?^\};?$" % name, text,
                  re.S | re.M)
    assert m, name
    return m.group(0)


def _run(tmp_path, functions, body):
    if shutil.which("g++") is None:
        pytest.skip("g++ missing")
    src, exe = str(tmp_path / "check.cpp"), str(tmp_path / "check")
    with open(src, "w") as f:
        f.write(HEAD % ("\n".join(functions), body))
    # (signed sums wrap as they do on the GPU)
    subprocess.run(["g++", "-O2", "-std=c++17", "-fwrapv", "-w", src, "-o", exe], check=True)
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert r.returncode == 0, r.stdout


def test_rows_of_a_call_on_pages(tmp_path):
    # every entry and row once, and nothing past them, up to entries * (rows + page size) = 2^31
    fns = [_function("pages.hip", f) for f in ("RowMap", "make_map", "map_row", "new_slot")]
    _run(tmp_path, fns, r"""
  for (int k = 0; k < 3000000; ++k) {
    const int ps = 16 << upto(6);
    const int64_t entries = 1 + log_upto((int64_t(1) << 31) / (ps + 1) - 2);
    const int64_t most_rows = ((int64_t(1) << 31) - 1) / entries - ps;
    if (most_rows < 0) continue;
    const int64_t rows = k % 3 == 0 ? most_rows : log_upto(most_rows);
    const int64_t most = rows + (k & 1 ? ps - 1 : 0);
    const RowMap m = make_map((int)entries, most);
    CHECK((int64_t)m.rows == entries * m.per * (int64_t(1) << m.tile_shift));   // (no wrap)
    CHECK((int64_t)m.rows + 16384 * 32 < int64_t(1) << 32);                     // (nor by a stride)
    CHECK((int64_t)m.per << m.tile_shift >= most);
    if (m.rows == 0) continue;
    // the first, the last, and any other row of the launch
    const uint32_t gs[4] = {0, m.rows - 1, (uint32_t)upto(m.rows - 1), (uint32_t)upto(m.rows - 1)};
    for (uint32_t g : gs) {
      int e, row;
      map_row(m, g, &e, &row);
      CHECK(e >= 0 && e < entries && row >= 0 && row < (int64_t)m.per << m.tile_shift);
      CHECK((((uint32_t)e * m.per + (row >> m.tile_shift)) << m.tile_shift | (row & ((1 << m.tile_shift) - 1))) == g);
      // a unit of up to 2^30 rows, of which the first `first` stay, and a refused one
      const int64_t n1 = log_upto(int64_t(1) << 30), first = upto(n1) / ps * ps;
      const int slot = new_slot((int)first, row, (int)n1);
      CHECK(first + row < n1 ? slot == first + row : slot == -1);
      CHECK(new_slot((int)first, row, -1) == -1);
    }
  }
""")
