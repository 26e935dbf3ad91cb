"""The division of the paged attention's chunks into runs, compiled for the host (no GPU needed): every chunk is taken once and
a shared unit's pieces find each other; with lengths that change between two reads, which a caller must not do, nothing
outside of the entries or of the pieces' places is named, and every run ends."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include "mkv_paged_runs.h"
#include <cstdio>
#include <cstdlib>
#include <map>
#include <set>
#include <vector>
using namespace mkv;
static unsigned long long state = 1;
static unsigned rnd(unsigned n) { state = state * 6364136223846793005ull + 1442695040888963407ull; return (unsigned)(state >> 33) % n; }
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } } while (0)

struct Entries {
  std::vector<int> chunks;
  bool change;                       // between any two reads
  int read(int b) {
    CHECK(b >= 0 && b < (int)chunks.size());
    if (change && rnd(3) == 0) chunks[b] = rnd(2) ? 0 : (int)rnd(1 + 2 * (unsigned)chunks[b] + 5);
    return chunks[b];
  }
};

// One CTA's way through its run, as the loading warp takes it for more entries than its lanes hold.
struct Taken { int unit, c0, c1, place, count; };
static bool run(Entries& e, int Hkv, int grid, int r, std::vector<Taken>& out) {
  const int B = (int)e.chunks.size();
  int total = 0;
  for (int b = 0; b < B; ++b) total += e.read(b) * Hkv;
  const Runs rs(total, grid);
  if (r >= rs.runs) return true;
  int cur = rs.start(r), end = rs.start(r + 1), b = 0, base = 0;
  for (int b0 = 0;; b0 += 32) {      // 32 entries at a time
    int in = 0, before = 0, found = -1;
    for (int i = b0; i < b0 + 32 && i < B && found < 0; ++i) {
      before = in;
      in += e.read(i) * Hkv;
      if (base + in > cur) found = i;
    }
    if (found >= 0) { b = found; base += before; break; }
    if (b0 + 32 >= B) { b = b0; break; }
    base += in;
  }
  int chunks = e.read(b), held = chunks * Hkv;
  while (cur < end) {
    if (!walk_to(cur, B, b, base, held, [&](int i) { chunks = e.read(i); return chunks * Hkv; })) return false;
    CHECK(chunks > 0 && cur >= base);
    const int kvh = (cur - base) / chunks, unit0 = base + kvh * chunks;
    const int c0 = cur - unit0, c1 = chunks < c0 + (end - cur) ? chunks : c0 + (end - cur);
    CHECK(kvh >= 0 && kvh < Hkv && c0 >= 0 && c1 > c0);
    cur += c1 - c0;
    Taken t = {b * Hkv + kvh, c0, c1, -1, 1};
    if (c1 - c0 != chunks) {
      const Shares sh(rs, unit0, chunks);
      t.place = r == sh.first ? sh.place0 : 2 * r;
      t.count = sh.count;
      CHECK(sh.first >= 0 && sh.place0 >= 0 && sh.place0 < 2 * grid && sh.count <= grid - sh.first);
      CHECK(t.place >= 0 && t.place < 2 * grid);
    }
    out.push_back(t);
  }
  return true;
}

int main() {
  long failed = 0;
  for (int round = 0; round < 400; ++round) {
    const int B = 1 + (int)rnd(round % 4 == 0 ? 2048 : 100), Hkv = 1 + (int)rnd(8), grid = 1 + (int)rnd(304), most = 1 + (int)rnd(300);
    Entries e;
    for (int b = 0; b < B; ++b) e.chunks.push_back(rnd(4) ? (int)rnd((unsigned)most) : 0);
    const std::vector<int> chunks = e.chunks;
    e.change = false;
    std::map<int, std::vector<Taken>> units;
    std::set<int> places;
    for (int r = 0; r < grid; ++r) {
      std::vector<Taken> t;
      CHECK(run(e, Hkv, grid, r, t));
      for (const Taken& x : t) {
        units[x.unit].push_back(x);
        if (x.place >= 0) CHECK(places.insert(x.place).second);
      }
    }
    for (int u = 0; u < B * Hkv; ++u) {
      int next = 0;
      for (const Taken& x : units[u]) { CHECK(x.c0 == next); next = x.c1; CHECK(x.count == (int)units[u].size()); }
      CHECK(next == chunks[u / Hkv]);
    }
    e.change = true;
    for (int r = 0; r < grid && round < 100; ++r) {
      std::vector<Taken> t;
      failed += !run(e, Hkv, grid, r, t);
    }
  }
  CHECK(failed > 0);                 // (some walks did come to the last entry)
  return 0;
}
"""


def test_runs(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("needs a host compiler")
    src, exe = tmp_path / "runs.cpp", tmp_path / "runs"
    src.write_text(SOURCE)
    csrc = os.path.join(ROOT, "paper_2609_07966_gb300", "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", csrc, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
