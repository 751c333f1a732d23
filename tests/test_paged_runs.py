"""The long batches in paged_shapes.py without a GPU: how their work is cut, from paged.hpp compiled for the host, so that tests on the GPU that rely on
long pieces do get them; and that their bounds see a single wrong page."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2509_26541_amd import binding as tb
from tests import asm_checks, paged_shapes

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
needs_hipcc = pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")

# prints the workgroups that share the work and the key tiles of every piece
PROGRAM = r"""
#include "paged.hpp"
#include <cstdio>
#include <vector>
using namespace tasp;
template <int BM, int BT>
static void pieces(const PagedAttn& p) {
  int64_t all = 0;
  for (int b = 0; b < p.c.n_seqs; ++b) { const PagedCost c = cost_of<BM>(p, load_seq(p.c, b)); all += cost_upto(c, c.row_tiles) * p.c.Hkv; }
  const int64_t share = share_of_all(p, static_cast<int>(all));
  std::printf("%d\n", p.workers);
  int64_t start = 0;
  for (int b = 0; b < p.c.n_seqs; ++b) {
    const PagedSeq s = load_seq(p.c, b);
    const PagedCost c = cost_of<BM>(p, s);
    for (int i = 0; i < c.row_tiles * p.c.Hkv; ++i) {
      const int rt = i % c.row_tiles, rows = s.n * p.G;
      const int64_t cost = c.first + rt * c.step;
      const PagedKeys k = keys_of<BM, BT>(p, s, rt * BM / p.G, (lesser(rt * BM + BM, rows) - 1) / p.G);
      for (int64_t w = start / share; w <= (start + cost) / share; ++w) {
        const int64_t from = w * share, to = from + share;
        if (to <= start || from >= start + cost) continue;
        const int64_t x0 = snapped(static_cast<int>(larger<int64_t>(from - start, 0)), cost, p.snap), x1 = to - start >= cost ? cost : snapped(static_cast<int>(to - start), cost, p.snap);
        if (x0 < x1) std::printf("%d\n", key_tile_at(x1, cost, k.n_tiles) - key_tile_at(x0, cost, k.n_tiles));
      }
      start += cost;
    }
  }
}
int main() {
  PagedAttn p{};
  int bm, workers, cost, snap, least;
  if (std::scanf("%d %d %d %d %d %d %d %d %d %d %d %d", &bm, &workers, &cost, &snap, &least, &p.c.n_seqs, &p.c.Hkv, &p.G, &p.causal, &p.window, &p.sinks, &p.c.max_pages) != 12) return 2;
  std::vector<int> kv(p.c.n_seqs), start(p.c.n_seqs + 1);
  for (int i = 0; i < p.c.n_seqs; ++i) { int n; if (std::scanf("%d %d", &n, &kv[i]) != 2) return 2; start[i + 1] = start[i] + n; }
  p.c.kv_len = kv.data(); p.c.row_start = start.data(); p.c.n_rows = start.back(); p.c.ps_log2 = 5; p.c.cap = p.c.max_pages << 5;
  if (!set_cut(p, bm, workers, cost, snap, least)) return 3;
  if (bm == 16) pieces<16, 64>(p);
  if (bm == 32) pieces<32, 64>(p);
  if (bm == 128) pieces<128, 64>(p);
  return 0;
}
"""


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    d = tmp_path_factory.mktemp("runs")
    (d / "runs.cpp").write_text(PROGRAM)
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-I" + os.path.join(asm_checks.ROOT, "include"), "-I" + asm_checks.CSRC, str(d / "runs.cpp"),
                    "-o", str(d / "runs")], check=True, capture_output=True, text=True)
    return str(d / "runs")


def _cut_constants(few):
    """The last three arguments of set_cut, as the launchers have them."""
    with open(os.path.join(asm_checks.CSRC, "attn_paged.hip" if few else "attn_paged_tile.hip")) as f:
        found = re.findall(r"return set_cut\(p, .*, (\d+), (\d+), (\d+)\);", f.read())
    assert len(found) == 1
    return found[0]


def _pieces(exe, kind, d, tokens, windowed):
    few = (kind, d, tokens) in paged_shapes.ROWS
    workers = (paged_shapes.ROWS if few else paged_shapes.TILES)[kind, d, tokens]
    new, kv = paged_shapes.batch(kind, d, tokens)
    bm, width = (8 * tokens if few else 128), max(-(-x // paged_shapes.PAGE) for x in kv)
    head = [bm, workers, *_cut_constants(few), len(kv), paged_shapes.HKV, paged_shapes.GROUP, 1 if windowed else 0, paged_shapes.WINDOW if windowed else 0,
            paged_shapes.SINKS if windowed else 0, width]
    got = subprocess.run([exe], input=" ".join(str(x) for x in head + [y for pair in zip(new, kv) for y in pair]), capture_output=True, text=True, check=True)
    lines = [int(x) for x in got.stdout.split()]
    # the library's own number of workgroups: the workspace holds two partial results of (bm, d) and 32 bytes for each
    c = tb.PagedCacheArgs(k=1 << 20, v=2 << 20, k_scale=3 << 20, v_scale=4 << 20, n_pages=paged_shapes.POOL, page_size=paged_shapes.PAGE, Hkv=paged_shapes.HKV, d=d,
                          dtype=tb.DTYPE_BF16 if kind == "bf16" else tb.DTYPE_E4M3)
    b = tb.PagedBatchArgs(page_table=5 << 20, kv_len=6 << 20, row_start=7 << 20, n_rows=sum(new), n_seqs=len(kv), max_pages=width, max_rows=max(new))
    a = tb.PagedAttnArgs(q_stride=0, Hq=paged_shapes.HKV * paged_shapes.GROUP, out_dtype=tb.DTYPE_FP32, mask_mode=tb.MASK_CAUSAL if windowed else tb.MASK_FULL,
                         window=head[9], sinks=head[10], softmax_scale=0.0)
    size = tb.lib.tasp_paged_attn_workspace_bytes(C.byref(c), C.byref(b), C.byref(a))
    assert lines[0] == workers and abs(size / (workers * (2 * bm * (d + 2) * 4 + 32)) - 1) < 0.05
    return lines[1:]


@needs_hipcc
@pytest.mark.parametrize("windowed", [False, True])
@pytest.mark.parametrize("kind,d,tokens", list(paged_shapes.ROWS) + list(paged_shapes.TILES))
def test_pieces_are_long(exe, kind, d, tokens, windowed):
    got = _pieces(exe, kind, d, tokens, windowed)
    if tokens <= 4:
        # the list of pages is taken up again twice, at tiles 128 and 256
        assert max(got) > 260 and sum(x > 130 for x in got) > 100
    else:
        # lists of pages at tiles 8, 16, ...; sums through their second level at 64 and 128; both parities of the last tile
        assert max(got) > 130 and sum(x > 66 for x in got) > 100
        for parity in (0, 1):
            for lo, hi in ((17, 32), (33, 64), (65, 200)):
                assert any(lo <= x <= hi and x % 2 == parity for x in got), (lo, parity)


@pytest.mark.parametrize("d,tokens,few", [(128, 2, True), (64, 2, True), (128, 5, False), (64, 5, False)])
def test_one_wrong_page_is_out_of_bounds(d, tokens, few):
    """Of the 938 pages of a sequence one is taken for another, for K or for V alone: further from the oracle than test_gpu_paged_long.py lets pass."""
    from tests import test_gpu_paged_long as long

    gen = torch.Generator().manual_seed(d + tokens)
    k, v = (torch.randn((paged_shapes.POOL, 2, paged_shapes.PAGE, d), generator=gen).to(torch.bfloat16).double() for _ in range(2))
    kv, starts = [30000], [0, tokens]
    table = paged_shapes.table(kv, 3)
    q = long._queries(k, table, kv, starts, 16, 5).double()
    want = long._exact(q, k, v, table, kv, starts, causal=False)
    o_bound, l_bound = long._bounds(want, d, 300, few)
    for at in (300, 700):
        there = table[0][at]
        assert 0 <= there < paged_shapes.POOL
        wrong = [table[0][:at] + [paged_shapes.POOL] + table[0][at + 1 :]]           # a page that has one of the two from elsewhere
        for k_from, v_from in ((there, (there + 7) % paged_shapes.POOL), ((there + 7) % paged_shapes.POOL, there)):
            out, lse, _, _ = long._exact(q, torch.cat([k, k[k_from][None]]), torch.cat([v, v[v_from][None]]), wrong, kv, starts, causal=False)
            assert float(((out - want[0]).abs() / o_bound).max()) > 1 or float(((lse - want[1]).abs() / l_bound).max()) > 1
