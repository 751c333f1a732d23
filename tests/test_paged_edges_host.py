"""The paged cache's lists at the far ends of what they may hold, without a GPU: the oracle, and the kernels' index arithmetic compiled for the host."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import paged
from tests import asm_checks

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
needs_hipcc = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")

PROGRAM = r"""
#include "paged.hpp"
#include <cstdio>
#include <vector>
using namespace tasp;
static unsigned long long state = 88172645463325252ull;
static unsigned rnd() { state ^= state << 13; state ^= state >> 7; state ^= state << 17; return static_cast<unsigned>(state >> 32); }
static long long bad = 0;
static void expect(bool ok, const char* what) { if (!ok && bad++ < 5) std::printf("%s\n", what); }
BODY
"""


def _run(tmp_path, body):
    src, exe = tmp_path / "edges.cpp", tmp_path / "edges"
    src.write_text(PROGRAM.replace("BODY", body))
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-I" + os.path.join(asm_checks.ROOT, "include"), "-I" + asm_checks.CSRC, str(src), "-o", str(exe)],
                   check=True, capture_output=True, text=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True)
    assert got.returncode == 0, got.stdout


PLACES = r"""
int main() {
  for (int round = 0; round < 4000; ++round) {
    const int n_seqs = 1 + rnd() % 4, n_rows = 1 + rnd() % 40, max_pages = 1 + rnd() % 5;
    std::vector<int> table(n_seqs * max_pages), kv(n_seqs), start(n_seqs + 1);
    for (int& x : table) x = static_cast<int>(rnd() % 7) - 1;
    for (int& x : kv) x = static_cast<int>(rnd() % 120) - 10;
    // not falling, from below 0 to beyond the rows
    start[0] = static_cast<int>(rnd() % 8) - 4;
    for (int i = 0; i < n_seqs; ++i) start[i + 1] = start[i] + static_cast<int>(rnd() % 30);
    if (round % 5 == 0) start[n_seqs] = 2147483647;
    PagedView c{};
    c.table = table.data(); c.kv_len = kv.data(); c.row_start = start.data();
    c.n_pages = 6; c.ps_log2 = 4; c.Hkv = 1; c.n_seqs = n_seqs; c.max_pages = max_pages; c.n_rows = n_rows; c.cap = max_pages << 4;
    for (int b = 0; b < n_seqs; ++b) {
      const PagedSeq s = load_seq(c, b);
      for (int j = 0; j < s.n; ++j) {
        const int pos = s.kv - s.n + j;
        const bool inside = pos >= 0 && pos < c.cap;
        const int page = inside ? page_of(c, b, pos) : -1;
        const PagedPlace at = place_of(c, b, s.r0 + j);
        expect(at.page == page && (page < 0 || at.slot == (pos & 15)), "a row is written elsewhere than it attends from");
      }
    }
  }
  return bad != 0;
}
"""


@needs_hipcc
def test_rows_are_written_where_they_attend_from(tmp_path):
    """place_of (write and read) and load_seq (attention) agree for every row, with lists that reach beyond the rows on both sides."""
    _run(tmp_path, PLACES)


WINDOWS = r"""
int main() {
  for (int round = 0; round < 4000; ++round) {
    int table[8] = {0, 1, 2, 3, 0, 1, 2, 3}, start[2] = {0, 1 + static_cast<int>(rnd() % 40)}, kv = 2147483647 - static_cast<int>(rnd() % 100);
    PagedAttn p{};
    p.window = 2147483647 - static_cast<int>(rnd() % 150);
    if (round % 3 == 1) { p.window = (1 << 30) + static_cast<int>(rnd() % 100); kv = p.window + static_cast<int>(rnd() % 100); }
    if (round % 3 == 2) kv = static_cast<int>(rnd() % 60);                  // fewer tokens than rows, too
    p.c.table = table; p.c.kv_len = &kv; p.c.row_start = start;
    p.c.n_pages = 4; p.c.ps_log2 = 4; p.c.Hkv = 1; p.c.n_seqs = 1; p.c.max_pages = 8; p.c.n_rows = start[1]; p.c.cap = 128;
    p.G = 1 + rnd() % 3; p.tile_cost = 1; p.causal = 1; p.sinks = rnd() % 20;
    const PagedSeq s = load_seq(p.c, 0);
    for (int rt = 0; rt * 16 < s.n * p.G; ++rt) {
      const int tok0 = rt * 16 / p.G, tok1 = (lesser(rt * 16 + 16, s.n * p.G) - 1) / p.G;
      const PagedKeys k = keys_of<16, 64>(p, s, tok0, tok1);
      for (int tok = tok0; tok <= tok1; ++tok)
        for (int t = 0; t < lesser(s.kv, 128); ++t) {
          const int64_t pos = static_cast<int64_t>(s.kv) - s.n + tok;
          const bool seen = t <= pos && (t > pos - p.window || t < p.sinks);
          expect(seen == (t <= pos && (t >= window_start(s.kv - s.n + tok, p.window) || t < p.sinks)), "the mask of a row");
          bool in = false;
          for (int u = 0; u < k.n_tiles && !in; ++u) in = t / 64 == k.tile(u);
          expect(!seen || (in && t < k.end), "a key that is seen is in no tile");
        }
    }
  }
  return bad != 0;
}
"""


@needs_hipcc
def test_windows_and_lengths_near_2_31_stay_in_32_bits(tmp_path):
    _run(tmp_path, WINDOWS)


def test_the_oracle_clips_its_lists():
    rng = np.random.default_rng(3)
    table, kv = [[0, 1, 2], [3, 4, 5]], [40, 30]
    assert paged.places(table, kv, [-3, 5, 90], 16, 6, 9) == paged.places(table, kv, [0, 5, 9], 16, 6)
    assert paged.places(table, kv, [0, 5, 90], 16, 6, 9)[5:] == [(5, 4, 10), (6, 4, 11), (7, 4, 12), (8, 4, 13)]
    q, k, v = rng.standard_normal((9, 2, 8)), rng.standard_normal((6, 1, 16, 8)), rng.standard_normal((6, 1, 16, 8))
    for a, b in zip(paged.attention(q, k, v, table, kv, [-3, 5, 90]), paged.attention(q, k, v, table, kv, [0, 5, 9])):
        assert np.array_equal(a, b, equal_nan=True)
