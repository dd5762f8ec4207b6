"""Host-side arithmetic of a step's calls, on the CPU: the kernels' index functions, taken from
their source text and built with g++."""
import re

from tests.test_host_serving import _function, _run

PRE = """
#include <algorithm>
#include <vector>
using std::max; using std::min;
static uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)((uint64_t)a * b >> 32); }
static int64_t min(int a, int64_t b) { return b < a ? b : a; }
static int64_t max(int a, int64_t b) { return b > a ? b : a; }
"""

CHUNK = """
#define __builtin_amdgcn_readfirstlane(x) (x)
static int64_t uniform64(int64_t x) { return x; }
struct AttendK {
  int sequences, heads, group, step_tokens, longest, pool_units, max_pages, shift;
  const int32_t *units, *starts, *lens, *table;
  int64_t unit_stride;
};
typedef %s E;
static const int SHIFT = sizeof(E) == 2 ? 7 : 5;
"""


def _chunk(name):
    text = _function("chunk.hip", name)
    for f in ("tile_of", "find_sequence", "shape_of"):
        text = text.replace(f + "<E>", f)
    return text.replace("kJobShift<E>", "SHIFT")


def _jobs(kind):
    shape = _chunk("Shape")
    return [PRE, CHUNK % kind, _chunk("tile_of"), _chunk("find_sequence"), shape, _chunk("shape_of"), _chunk("Walk")]


JOBS = """
  for (int round = 0; round < 3000; ++round) {
    AttendK a = {};
    a.sequences = 1 + (int)log_upto(60);
    a.heads = 1 + (int)upto(5);
    a.group = 1 + (int)log_upto(40);
    a.step_tokens = (int)log_upto(3000);
    a.longest = round %% 3 == 0 ? 1 + (int)upto(a.step_tokens) : 1 << 29;
    a.pool_units = 1000;
    const bool rising = round %% 4 != 0;
    std::vector<int32_t> starts(a.sequences + 1);
    for (int& x : starts) x = (int)upto(a.step_tokens + 20) - (rising ? 0 : 10);
    if (rising) std::sort(starts.begin(), starts.end());
    a.starts = starts.data();
    const int64_t jobs = (((int64_t)a.step_tokens * a.group >> SHIFT) + a.sequences) * a.heads;
    // rows of each sequence, head: how often a job has them
    std::vector<std::vector<int>> seen(a.sequences * a.heads);
    auto clip = [&](int x) { return min(max(x, 0), a.step_tokens); };
    for (int b = 0; b < a.sequences; ++b)
      for (int h = 0; h < a.heads; ++h)
        seen[b * a.heads + h].resize((size_t)max(0, min(clip(starts[b + 1]) - clip(starts[b]), a.longest)) * a.group);
    // a walk over all jobs, and one that starts at each
    Walk w{a.starts};
    w.start(a, 0);
    for (int64_t j = 0; j < jobs; ++j) {
      w.to(a, j);
      Walk v{a.starts};
      v.start(a, j);
      Shape s = {}, t = {};
      const bool on = shape_of(a, a.starts, j, w.b, w.tile, w.next, &s);
      const bool too = shape_of(a, a.starts, j, v.b, v.tile, v.next, &t);
      CHECK(w.b < a.sequences && v.b < a.sequences);
      for (int k = 0; k < 2; ++k) {   // (whatever the starts: inside the packed rows)
        const Shape& x = k ? t : s;
        if (k ? !too : !on) continue;
        CHECK(x.h >= 0 && x.h < a.heads && x.start >= 0 && x.t >= 1 && x.start + x.t <= a.step_tokens && x.t <= a.longest);
        CHECK(x.r0 >= 0 && x.rows >= 1 && x.rows <= 1 << SHIFT && x.r0 + x.rows <= (int64_t)x.t * a.group);
        CHECK(x.unit >= 0 && x.unit < a.pool_units);
      }
      if (!rising) continue;
      CHECK(on == too && (!on || (s.h == t.h && s.start == t.start && s.r0 == t.r0 && s.rows == t.rows)));
      if (!on) continue;
      CHECK(s.unit == w.b * a.heads + s.h && s.start == clip(starts[w.b]));
      auto& rows = seen[w.b * a.heads + s.h];
      for (int r = s.r0; r < s.r0 + s.rows; ++r) {
        CHECK(r < (int)rows.size());
        if (r < (int)rows.size()) ++rows[r];
      }
    }
    if (rising)
      for (auto& rows : seen)
        for (int n : rows) CHECK(n == 1);
  }
"""


def test_jobs_of_a_chunk_call(tmp_path):
    # every row of every sequence and head is in one job, whether a walk comes from afar or starts there
    for i, kind in enumerate(("uint16_t", "float")):
        (tmp_path / str(i)).mkdir()
        _run(tmp_path / str(i), _jobs(kind), JOBS.replace("%%", "%"))


def test_parts_of_a_chunk_call(tmp_path):
    # jobs cut into equal parts: every tile is in one part, the parts of a cut job follow one another
    # and are as many as its first one says, and no part begins or goes on with two cut jobs
    _run(tmp_path, [PRE, _function("chunk.hip", "Cost")], r"""
  for (int round = 0; round < 20000; ++round) {
    const int jobs = 1 + (int)log_upto(300), blocks = 8 * (1 + (int)upto(63));
    std::vector<Cost> cost(jobs);
    int64_t all = 0;
    for (Cost& c : cost) {
      const int kind = (int)upto(2);
      c = kind == 0 ? Cost{6, 2, 1} : kind == 1 ? Cost{15, 5, 1} : Cost{9, 3, 1};
      c.n = 1 + (int)log_upto(round % 2 ? 3000 : 40);
      all += c.all();
    }
    const int64_t part = max((int64_t)16, (all + blocks - 1) / blocks);
    int64_t at = 0;
    std::vector<int> begun(blocks), gone_on(blocks);
    for (const Cost& c : cost) {
      int next = 0, first = -1, said = 0, have = 0, last = -1;
      for (int64_t b = 0; b < blocks; ++b) {
        const int64_t lo = b * part, hi = min(all, lo + part);
        if (lo >= all || hi <= at || lo >= at + c.all()) continue;
        const int vt0 = c.tiles(lo - at), vt1 = c.tiles(hi - at);
        const bool whole = vt0 == 0 && vt1 == c.n;
        if (vt1 <= vt0) continue;
        CHECK(vt0 == next && vt1 <= c.n);
        next = vt1;
        ++have;
        if (vt0 == 0) {
          first = (int)b;
          said = (int)(min((at + c.all() - c.tile) / part, (int64_t)blocks - 1) - b) + 1;
        }
        CHECK(last < 0 || b == last + 1);
        last = (int)b;
        if (!whole) ++(vt0 == 0 ? begun : gone_on)[b];
      }
      CHECK(next == c.n && first >= 0 && said == have);
      at += c.all();
    }
    for (int b = 0; b < blocks; ++b) CHECK(begun[b] <= 1 && gone_on[b] <= 1);
  }
""")


def test_pieces_of_a_call_of_few_jobs(tmp_path):
    # blocks for each job, as chunk_kernel counts them: all jobs fit, and no tile is left out
    text = open(__file__.replace("tests/test_host_step.py", "paper_2605_31105_amd/csrc/chunk.hip")).read()
    count = re.search(r"const int k = \(int\)\(\(own \+ cost - 1\) / cost\);\s*return a\.flags \? min\(k, kJoined\) : k;", text)
    second = "max((int64_t)a.min_tiles, (all + blocks - a.jobs - 1) / (blocks - a.jobs))"
    assert count and second in text and "cost.n * (i + 1) / pieces" in text
    _run(tmp_path, [PRE, _function("chunk.hip", "Cost")], r"""
  for (int round = 0; round < 40000; ++round) {
    const int jobs = 1 + (int)upto(63), blocks = min(512, (2 * jobs + 8 * (int)log_upto(60) + 7) / 8 * 8);
    const bool joined = round % 3 == 0;
    std::vector<Cost> cost(jobs);
    int64_t all = 0;
    for (Cost& c : cost) {
      c = round % 2 ? Cost{6, 2, 1} : Cost{15, 5, 1};
      c.n = 1 + (int)log_upto(3000);
      if (upto(5) == 0) c = Cost{0, 0, 0};   // (a job without rows)
      all += c.all();
    }
    auto blocks_for = [&](int64_t own, int64_t cost) {
      const int k = (int)((own + cost - 1) / cost);
      return joined ? min(k, 16) : k;
    };
    int64_t p = 16, total = 0;
    for (const Cost& c : cost) total += blocks_for(c.all(), p);
    if (total > blocks) {
      p = max(p, (all + blocks - jobs - 1) / (blocks - jobs));
      total = 0;
      for (const Cost& c : cost) total += blocks_for(c.all(), p);
    }
    CHECK(total <= blocks);
    for (const Cost& c : cost) {
      const int k = blocks_for(c.all(), p);
      CHECK((k == 0) == (c.n == 0));
      int next = 0;
      for (int i = 0; i < k; ++i) {
        const int vt0 = (int)((int64_t)c.n * i / k), vt1 = (int)((int64_t)c.n * (i + 1) / k);
        CHECK(vt0 == next && (vt1 > vt0 || (c.n == 1 && k == 2 && i == 0)));
        next = vt1;
      }
      CHECK(next == c.n);
    }
  }
""")


def test_sequences_of_grown_units(tmp_path):
    # entries to sequences by multiplication, as launch_extend prepares it, and rows to sequences
    with open(__file__.replace("tests/test_host_step.py", "paper_2605_31105_amd/csrc/extend.hip")) as f:
        host = re.search(r"  while \(\(1ll << a\.hshift\) < a\.heads\).*?\n  a\.hmul = [^;]*;", f.read(), re.S).group(0)
    _run(tmp_path, [PRE, "struct ExtendK { int heads, hshift; uint32_t hmul; };", _function("extend.hip", "sequence_at"),
                    _function("extend.hip", "sequence_of")], """
  for (int k = 0; k < 200000; ++k) {
    ExtendK a = {};
    a.heads = k < 5000 ? k + 1 : (int)(1 + log_upto((1 << 24) - 1));
    %s
    for (int i = 0; i < 40; ++i) {
      const int64_t near = upto((1 << 24) / a.heads) * a.heads + upto(2) - 1;
      const int64_t e = i & 1 ? log_upto((1 << 24) - 1) : near < 0 ? 0 : near;
      CHECK(sequence_at(a, (int)e) == (int)(e / a.heads));
    }
  }
  for (int k = 0; k < 20000; ++k) {
    const int n = 1 + (int)log_upto(50);
    std::vector<int> starts(n + 1);
    for (int& x : starts) x = (int)upto(100);
    std::sort(starts.begin(), starts.end());
    starts[0] = 0;
    for (int t = 0; t <= 101; ++t) {
      int b = 0;
      while (b < n && starts[b + 1] <= t) ++b;
      CHECK(sequence_of(starts.data(), n, t) == b);
    }
  }
""" % host)
