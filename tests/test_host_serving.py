"""Host-side arithmetic of pages and attention, on the CPU: the kernels' index functions, taken
from their source text and built with g++."""
import ctypes
import os
import random
import re
import shutil
import subprocess
from types import SimpleNamespace

import pytest

import paper_2605_31105_amd as G
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


def test_division_by_the_group(tmp_path):
    # rows below 2^31 by groups up to 2^30, as launch_attend prepares it
    with open(os.path.join(B.CSRC, "attend.hip")) as f:
        host = re.search(r"  a\.gshift = 0;.*?\n  a\.gmul = [^;]*;", f.read(), re.S).group(0)
    pre = """
struct AttendK { int group, gshift; uint32_t gmul; };
static uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)((uint64_t)a * b >> 32); }
"""
    _run(tmp_path, [pre, _function("attend.h", "group_of")], """
  for (int k = 0; k < 200000; ++k) {
    AttendK a;
    a.group = k < 5000 ? k + 1 : (int)(1 + log_upto((1 << 30) - 1));
    %s
    for (int i = 0; i < 40; ++i) {
      const int64_t near = upto(((int64_t(1) << 31) - 1) / a.group) * a.group + upto(2) - 1;
      const int64_t r = i & 1 ? log_upto((int64_t(1) << 31) - 1) : near < 0 ? 0 : near > 0x7fffffff ? 0x7fffffff : near;
      CHECK(group_of(a, (int)r) == (int)(r / a.group));
    }
  }
""" % host)


def test_blocks_of_an_attention_call(tmp_path):
    # every entry, row group and split is one block's, and the blocks past them leave
    pre = """
struct AttendK { int entries, row_groups, splits, grouped, split_shift; };
static struct { uint32_t x; } blockIdx;
"""
    _run(tmp_path, ["#include <vector>", pre, _function("attend.h", "block_work")], """
  for (int k = 0; k < 4000; ++k) {
    AttendK a;
    a.entries = 1 + (int)log_upto(600);
    a.row_groups = 1 + (int)log_upto(40);
    a.split_shift = (int)upto(6);
    a.splits = 1 << a.split_shift;
    const int64_t w = (int64_t)a.entries * a.splits;
    a.grouped = w % 8 == 0 || w >= 64;
    const int64_t blocks = (a.grouped ? (w + 7) / 8 * 8 : w) * a.row_groups;
    std::vector<int> seen(w * a.row_groups);
    for (int64_t b = 0; b < blocks; ++b) {
      blockIdx.x = (uint32_t)b;
      int e, rg, sp;
      if (!block_work(a, &e, &rg, &sp)) continue;
      CHECK(e >= 0 && e < a.entries && rg >= 0 && rg < a.row_groups && sp >= 0 && sp < a.splits);
      ++seen[((int64_t)e * a.row_groups + rg) * a.splits + sp];
    }
    for (int n : seen) CHECK(n == 1);
  }
""")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if shutil.which("g++") is None or not os.path.isdir(os.path.join(rocm, "include", "hip")):
        pytest.skip("g++ or the HIP headers missing")
    G.lib()
    so = str(tmp_path_factory.mktemp("probe") / "attend_probe.so")
    subprocess.run(["g++", "-shared", "-fPIC", "-O1", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__",
                    "-I" + os.path.join(rocm, "include"), "-I" + os.path.join(B.ROOT, "include"), "-I" + B.CSRC,
                    os.path.join(B.ROOT, "tests", "attend_probe.cpp"), G.lib_path(), "-Wl,-rpath," + B.PKG, "-o", so],
                   check=True)
    fn = ctypes.CDLL(so).attend_probe
    fn.restype = None
    fn.argtypes = [ctypes.c_int32] * 5 + [ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p]
    names = ("rt", "row_groups", "splits", "min_tiles", "rows", "tile_keys", "grouped", "joined", "even", "blocks",
             "opart", "mpart", "flags", "total")

    def probe(*args):
        out = (ctypes.c_int64 * len(names))()
        fn(*args, out)
        return SimpleNamespace(**dict(zip(names, out)))

    return probe


def test_attention_plans_over_random_shapes(plan):
    rng = random.Random(3)

    def log(lo, hi):
        return round(lo * (hi / lo) ** rng.random())

    for _ in range(20000):
        entries, group, tokens = log(1, 5000), rng.choice([1, 4, log(1, 64)]), rng.choice([1, log(1, 64), log(1, 20000)])
        d, dtype, slots, ragged = rng.choice([64, 128]), rng.randrange(2), log(1, 1 << 30), rng.randrange(2)
        p, R = plan(entries, group, tokens, d, dtype, slots, ragged), group * tokens
        case = (entries, group, tokens, d, dtype, slots, ragged, p)
        assert p.rows == (128 if p.rt == 0 else 16 * p.rt) and p.row_groups == -(-R // p.rows), case
        assert 1 <= p.splits <= 256 and p.splits & (p.splits - 1) == 0, case
        assert dtype == G.GRKV_BF16 or p.rt == 1, case
        w = entries * p.splits
        if p.even:
            # one row group; two partial units a block, and a place in the table for each entry
            assert p.row_groups == 1 and ragged and not p.joined and entries <= 4096, case
            rows, extra = 2 * p.blocks * R, 8 * entries
        else:
            assert w * p.row_groups <= p.blocks <= (w + 7) * p.row_groups, case
            assert p.grouped or p.blocks == w * p.row_groups, case
            rows, extra = (w * R if p.splits > 1 else 0), 8 * w * p.row_groups if p.joined else 0
        assert p.opart == 0 and p.mpart >= 4 * d * rows and p.flags - p.mpart >= 16 * rows, case
        assert p.total - p.flags >= extra and not (p.mpart | p.flags | p.total) % 256, case
        # (marks of a joined call are read by one wave)
        assert not p.joined or (p.splits <= 16 and p.rt > 0), case
        # a unit of any length within the plan: its tiles in splits of at least min_tiles
        for n in (0, 1, slots, log(1, slots)):
            nt = -(-n // p.tile_keys)
            chunk = max(p.min_tiles, -(-nt // p.splits))
            assert -(-nt // chunk) <= p.splits, case
