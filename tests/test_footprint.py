"""Whether tensors of a call share memory (csrc/footprint.h) against every byte marked one by one, over random layouts: apart,
interleaved by head, by layer or by row, overlapping by a few bytes.  The header is host-compilable, so the check runs on the
CPU with g++."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
HEADER = os.path.join(HERE, "..", "paper_2609_22158_gb300", "csrc", "footprint.h")

PROGRAM = r"""
#include "%s"
#include <cstdio>
#include <cstdint>
#include <vector>
using namespace stepkv;
static uint64_t x = 88172645463325252ull;
static int rnd(int n) { x ^= x << 13; x ^= x >> 7; x ^= x << 17; return (int)((x >> 20) %% (uint64_t)n); }

struct Group { std::vector<const void*> at; Footprint f; bool written; };

// by the definition: byte -> how many tensors (or pieces of one) have it, and whether one of them is written
static bool truth(const std::vector<Group>& gs, int size) {
  std::vector<int> taken(size, 0), written(size, 0);
  for (auto& g : gs)
    for (auto p : g.at)
      for (int o = 0; o < g.f.outer_n; ++o)
        for (int i = 0; i < g.f.inner_n; ++i)
          for (int b = 0; b < g.f.len; ++b) {
            const int64_t k = (int64_t)(uintptr_t)p - 4096 + o * g.f.outer_step + i * g.f.inner_step + b;
            ++taken[k];
            written[k] |= g.written;
          }
  for (int k = 0; k < size; ++k)
    if (written[k] && taken[k] > 1) return true;
  return false;
}
static bool answer(const std::vector<Group>& gs) {
  Footprints fp;
  for (auto& g : gs) fp.add(g.at.data(), (int)g.at.size(), g.f, g.written);
  return fp.clash();
}

int main() {
  long bad = 0, yes = 0, no = 0;
  const int size = 1 << 16;
  for (int t = 0; t < 20000; ++t) {
    std::vector<Group> gs;
    const int kind = rnd(3);
    if (kind == 0) {  // sources and destinations of caches: one piece a head, own strides; bases anywhere or in a rough order
      const int groups = 1 + rnd(4);
      int64_t at = 4096;
      for (int g = 0; g < groups; ++g) {
        const int len = 1 + rnd(12), heads = 1 + rnd(5), step = len + rnd(3) * rnd(30), n = 1 + rnd(4);
        Group q{{}, make_footprint(heads, step, 1, 0, len), rnd(2) == 0};
        for (int l = 0; l < n; ++l) {
          q.at.push_back((const void*)(uintptr_t)at);
          at += rnd(4) ? q.f.span() + rnd(3) - (rnd(8) == 0) : rnd(40);
          if (at < 4096) at = 4096;
        }
        if (rnd(3) == 0) std::reverse(q.at.begin(), q.at.end());
        if (rnd(4) == 0) at = 4096 + rnd(200);
        gs.push_back(q);
      }
    } else {  // K and V rows of one layout, from one tensor whose axes (K/V, layer, head, row) come in any order
      int dims[4] = {1 + rnd(2), 1 + rnd(4), 1 + rnd(4), 1 + rnd(4)}, order[4] = {0, 1, 2, 3};
      for (int i = 3; i > 0; --i) std::swap(order[i], order[rnd(i + 1)]);
      const int len = 1 + rnd(5);
      int64_t stride[4], s = len;
      for (int i = 3; i >= 0; --i) {
        stride[order[i]] = s;
        s *= dims[order[i]];
        s += rnd(3) ? 0 : rnd(6);
      }
      if (kind == 2) stride[rnd(4)] = rnd(30);  // and then one axis off
      for (int v = 0; v < dims[0]; ++v) {
        Group q{{}, make_footprint(dims[2], stride[2], dims[3], stride[3], len), true};
        for (int l = 0; l < dims[1]; ++l) q.at.push_back((const void*)(uintptr_t)(4096 + v * stride[0] + l * stride[1]));
        gs.push_back(q);
      }
      // rows and heads that do not nest may miss one another all the same: such a layout is refused
      if (gs[0].f.folds()) {
        bad += !answer(gs);
        continue;
      }
    }
    const bool want = truth(gs, size);
    // (sources and destinations have one piece a run: exact for any mixture)
    bad += answer(gs) != want;
    (want ? yes : no)++;
  }
  std::printf("mismatches %%ld, %%ld meet, %%ld do not\n", bad, yes, no);
  return bad != 0 || yes < 3000 || no < 10000;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_footprints_match_every_byte(tmp_path):
    src, exe = tmp_path / "fp.cpp", tmp_path / "fp"
    src.write_text(PROGRAM % os.path.abspath(HEADER))
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-o", str(exe), str(src)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
