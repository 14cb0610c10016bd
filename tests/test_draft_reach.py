"""Which keys a block of rows of a tree of drafted tokens sees (draft_reach, draft_take, draft_sees in zo_decode.cuh, the rules that
the kernels look pages up by), on the host: none that the page table has no column for, none behind a sequence's last, and
none at all where there are more than the table or 31 bits hold."""
import os
import shutil
import subprocess

import pytest

from paper_2609_38095_gb300 import build as zo_build

HARNESS = r"""
#include <algorithm>
#include <cstdio>
#include <random>
#include "zo_decode.cuh"
using namespace zo;
static int bits_up_to(uint64_t m) { return m == 0 ? 0 : 64 - __builtin_clzll(m); }
int main() {
  std::mt19937_64 g(1);
  const auto pick = [&](int64_t n) { return static_cast<int64_t>(g() % static_cast<uint64_t>(n)); };
  long long seen = 0, none = 0, bad = 0;
  for (int round = 0; round < 200000; ++round) {
    DraftParams p = {};
    p.group = 1 + pick(8);
    p.kv_heads = 1;
    p.drafts = 1 + pick(64);
    p.page_size = 1 + pick(round % 3 ? 20 : 300);
    p.max_pages = pick(4) == 0 ? pick(2) : pick(12);
    p.n_pages = pick(10) == 0 ? 0 : 100;
    const int64_t room = p.max_pages * p.page_size;
    uint64_t any = 0, rows = 0;  // nodes that are seen, nodes that see
    for (int i = 0; i < p.drafts; ++i) {
      const uint64_t m = pick(3) == 0 ? 0 : g() & g() & (~UINT64_C(0) >> (64 - p.drafts));
      any |= m;
      if (m != 0) rows |= UINT64_C(1) << i;
    }
    if (pick(6) == 0) any = rows = 0;
    const int lengths[] = {0, 1, static_cast<int>(pick(room + 1)), static_cast<int>(std::max<int64_t>(0, room - pick(70))),
                           static_cast<int>(room + 1 + pick(300)), 0x7FFFFFFF, 0x7FFFFFFF - static_cast<int>(pick(200)),
                           static_cast<int>(pick(0x7FFFFFFF))};
    const int n = lengths[pick(8)];
    const DraftKeys k = draft_reach(p, n, any, bits_up_to(any), bits_up_to(rows));
    const int block = 16 << pick(5), blocks = (p.drafts * p.group + block - 1) / block;
    for (int i = 0; i < blocks; ++i) {
      DraftPlace w = {};
      w.head0 = i * block;
      w.heads = std::min(block, p.drafts * p.group - w.head0);
      draft_take(w, p, k, n);
      const int64_t want = any == 0 ? 0 : static_cast<int64_t>(n) + bits_up_to(any);
      const bool fits = want <= room && (want == 0 || p.n_pages > 0) && want <= 0x7FFFFFFF - 64;
      const int live = fits ? std::max(0, std::min(w.heads, bits_up_to(rows) * p.group - w.head0)) : 0;
      if ((w.bad != 0) == fits || w.live != live || w.len != (live > 0 ? want : 0)) {
        std::printf("round %d: n %d, len %lld, live %d, bad %d\n", round, n, static_cast<long long>(w.len), w.live, w.bad);
        return 1;
      }
      // every key near the ends of the table, of the sequence and of a few tiles from the first and the last
      for (int64_t from : {static_cast<int64_t>(0), static_cast<int64_t>(4096), room - 100, want - 200, static_cast<int64_t>(n) - 100})
        for (int64_t j = std::max<int64_t>(from, 0); j < from + 600; ++j) {
          const bool sees = draft_sees(w, j);
          const bool right = live > 0 && (j < n || (j < want && (any >> (j - n) & 1) != 0));
          if (sees != right || (sees && (j >= w.len || j / p.page_size >= p.max_pages))) {
            std::printf("round %d: key %lld of %lld (n %d) is looked up, in a table of %lld pages of %d\n", round, static_cast<long long>(j),
                        static_cast<long long>(w.len), n, static_cast<long long>(p.max_pages), p.page_size);
            return 1;
          }
        }
      seen += live > 0, none += live == 0, bad += w.bad;
    }
  }
  std::printf("%lld %lld %lld\n", seen, none, bad);
  return seen > 1000 && none > 1000 && bad > 1000 ? 0 : 1;
}
"""


def test_no_key_beyond_the_page_table(tmp_path):
    try:
        nvcc = zo_build.nvcc()
    except RuntimeError:
        pytest.skip("nvcc not found")
    if shutil.which("g++") is None:
        pytest.skip("g++ not found")
    src, exe = tmp_path / "reach.cu", tmp_path / "reach"
    src.write_text(HARNESS)
    root = os.path.dirname(zo_build.CSRC)
    made = subprocess.run([nvcc, "-O2", "-std=c++17", *zo_build.ARCH, "-I", zo_build.CSRC, "-I", zo_build.INCLUDE, str(src), "-o", str(exe)],
                          capture_output=True, text=True, cwd=root)
    assert made.returncode == 0, made.stderr[-2000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout
