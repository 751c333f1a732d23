"""The paged cache without a GPU: the oracle's pins, the library's refusals, and the index arithmetic of the kernels compiled for the host,
on lists that hold anything."""
import ctypes as C
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2509_26541_amd import binding as tb
from tests import asm_checks

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


# ---- oracle
def test_round_e4m3_is_the_library_cast():
    x = torch.cat([torch.linspace(-448, 448, 20001), torch.randn(5000) * 0.01, torch.tensor([0.0, 2.0**-9, 2.0**-10, 1.5 * 2.0**-9, 17.0, 19.0, 448.0])])
    want = x.to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(paged.round_e4m3(x.numpy()), want)


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.01, 1), (449.0, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.7501, -7), (0.0, -100), (2.0**-120, -100),
                                   (2.0**127, 119), (2.0**127 * 1.999, 120)])
def test_scale_is_the_smallest_that_fits(top, e):
    values, exps = paged.quantise(np.array([[0.0, top, -top / 3, math.inf, math.nan]]))
    assert exps[0] == e and np.isnan(values[0, 3]) and np.isnan(values[0, 4])
    assert np.abs(values[0, 1]) <= 448 and np.isfinite(np.float32(values[0, 1] * 2.0**e))
    assert abs(values[0, 1] * 2.0**e - top) <= top * (2.0**-4 if top < 2.0**127 * 1.9 else 2.0**-3) + 2.0**-110


def test_attention_against_loops_and_library_softmax():
    rng = np.random.default_rng(1)
    ps, n_pages, hkv, hq, d = 16, 9, 2, 6, 8
    k, v = rng.standard_normal((2, n_pages, hkv, ps, d))
    table, kv_len, starts = [[4, 0, 7], [2, -1, 5], [1, 3, 99]], [40, 37, 3], [0, 3, 5, 10]
    q = rng.standard_normal((10, hq, d))
    for causal, window, sinks in ((True, 0, 0), (True, 5, 2), (True, 17, 0), (False, 0, 0)):
        out, lse, _, _ = paged.attention(q, k, v, table, kv_len, starts, causal, window, sinks)
        for b in range(3):
            n = starts[b + 1] - starts[b]
            for j in range(n):
                p = kv_len[b] - n + j
                keys = [t for t in range(kv_len[b]) if 0 <= table[b][t // ps] < n_pages and (not causal or t <= p)
                        and (not window or t > p - window or t < sinks)]
                for h in (0, 2, 3, 5):
                    row = starts[b] + j
                    if not keys:
                        assert lse[row, h] == -np.inf and not out[row, h].any()
                        continue
                    s = torch.tensor([float(q[row, h] @ k[table[b][t // ps], h // 3, t % ps]) / math.sqrt(d) for t in keys], dtype=torch.float64)
                    w = torch.softmax(s, 0).numpy()
                    want = sum(w[i] * v[table[b][t // ps], h // 3, t % ps] for i, t in enumerate(keys))
                    assert np.allclose(out[row, h], want, atol=1e-12) and abs(lse[row, h] - float(torch.logsumexp(s, 0))) < 1e-12


# ---- refusals: every call below returns before it touches a device
def _args(**kw):
    c = tb.PagedCacheArgs(k=1 << 20, v=2 << 20, k_scale=3 << 20, v_scale=4 << 20, n_pages=8, page_size=16, Hkv=2, d=64, dtype=tb.DTYPE_BF16)
    b = tb.PagedBatchArgs(page_table=5 << 20, kv_len=6 << 20, row_start=7 << 20, n_rows=4, n_seqs=2, max_pages=4, max_rows=0)
    a = tb.PagedAttnArgs(q=8 << 20, out=9 << 20, lse=10 << 20, workspace=11 << 20, workspace_bytes=1 << 40, q_stride=0, Hq=4, out_dtype=tb.DTYPE_BF16,
                         mask_mode=tb.MASK_CAUSAL, window=0, sinks=0, softmax_scale=0.0)
    for name, value in kw.items():
        for part in (c, b, a):
            if name in [f[0] for f in part._fields_]:
                setattr(part, name, value)
                break
        else:
            raise KeyError(name)
    return C.byref(c), C.byref(b), C.byref(a)


COMMON = [(dict(k=None), tb.EINVAL), (dict(v=None), tb.EINVAL), (dict(dtype=tb.DTYPE_E4M3, k_scale=None), tb.EINVAL), (dict(dtype=tb.DTYPE_E4M3, v_scale=None), tb.EINVAL),
          (dict(dtype=tb.DTYPE_FP32), tb.EUNSUPPORTED_SHAPE), (dict(dtype=7), tb.EUNSUPPORTED_SHAPE), (dict(d=96), tb.EUNSUPPORTED_SHAPE), (dict(d=0), tb.EUNSUPPORTED_SHAPE),
          (dict(page_size=8), tb.EUNSUPPORTED_SHAPE), (dict(page_size=48), tb.EUNSUPPORTED_SHAPE), (dict(page_size=2048), tb.EUNSUPPORTED_SHAPE), (dict(page_size=0), tb.EINVAL),
          (dict(n_pages=0), tb.EINVAL), (dict(n_pages=(1 << 30) + 1), tb.EUNSUPPORTED_SHAPE), (dict(Hkv=0), tb.EINVAL), (dict(k=(1 << 20) + 8), tb.EALIGN),
          (dict(dtype=tb.DTYPE_E4M3, v_scale=(4 << 20) + 4), tb.EALIGN), (dict(page_table=None), tb.EINVAL), (dict(kv_len=None), tb.EINVAL), (dict(row_start=None), tb.EINVAL),
          (dict(kv_len=(6 << 20) + 2), tb.EALIGN), (dict(n_seqs=-1), tb.EINVAL), (dict(n_rows=-1), tb.EINVAL), (dict(max_pages=0), tb.EINVAL), (dict(max_rows=-1), tb.EINVAL),
          (dict(max_pages=(1 << 26) + 1), tb.EUNSUPPORTED_SHAPE), (dict(n_rows=(1 << 30) + 1), tb.EUNSUPPORTED_SHAPE), (dict(n_rows=1 << 30), tb.EUNSUPPORTED_SHAPE),
          (dict(n_seqs=1 << 30), tb.EUNSUPPORTED_SHAPE), (dict(n_pages=1 << 30, page_size=1024), tb.EUNSUPPORTED_SHAPE),
          (dict(Hkv=1 << 20, page_size=1024), tb.EUNSUPPORTED_SHAPE)]
ATTN = [(dict(n_rows=1 << 29, Hq=16), tb.EUNSUPPORTED_SHAPE), (dict(Hq=0), tb.EINVAL), (dict(Hq=3), tb.EINVAL), (dict(mask_mode=tb.MASK_ZIGZAG_CAUSAL), tb.EINVAL), (dict(mask_mode=3), tb.EINVAL), (dict(window=-1), tb.EINVAL),
        (dict(sinks=-1), tb.EINVAL), (dict(mask_mode=tb.MASK_FULL, window=4), tb.EINVAL), (dict(softmax_scale=-1.0), tb.EINVAL), (dict(softmax_scale=math.inf), tb.EINVAL),
        (dict(softmax_scale=math.nan), tb.EINVAL), (dict(out_dtype=tb.DTYPE_E4M3), tb.EUNSUPPORTED_SHAPE), (dict(q_stride=255), tb.EINVAL), (dict(q_stride=260), tb.EALIGN),
        (dict(q=None), tb.EINVAL), (dict(out=None), tb.EINVAL), (dict(lse=None), tb.EINVAL), (dict(q=(8 << 20) + 8), tb.EALIGN), (dict(out=(9 << 20) + 4), tb.EALIGN),
        (dict(lse=(10 << 20) + 4), tb.EALIGN), (dict(workspace=None), tb.EWORKSPACE), (dict(workspace_bytes=16), tb.EWORKSPACE), (dict(workspace=(11 << 20) + 16), tb.EALIGN)]


@pytest.mark.parametrize("change,status", COMMON, ids=lambda x: str(x).replace(" ", ""))
def test_common_refusals(change, status):
    c, b, a = _args(**change)
    assert tb.lib.tasp_cache_write(c, b, 1 << 22, 1 << 23, 0, 0, tb.DTYPE_BF16, None) == status
    assert tb.lib.tasp_cache_read(c, b, 1 << 22, 1 << 23, tb.DTYPE_BF16, None) == status
    assert tb.lib.tasp_paged_attn(c, b, a, None) == status
    assert tb.lib.tasp_paged_attn_workspace_bytes(c, b, a) == 0


@pytest.mark.parametrize("change,status", ATTN, ids=lambda x: str(x).replace(" ", ""))
def test_attention_refusals(change, status):
    assert tb.lib.tasp_paged_attn(*_args(**change), None) == status


def test_write_and_read_refusals():
    c, b, _ = _args()
    for args, status in [((None, 1 << 22, 0, 0, tb.DTYPE_BF16), tb.EINVAL), ((1 << 22, None, 0, 0, tb.DTYPE_BF16), tb.EINVAL),
                         ((1 << 22, 1 << 23, 0, 0, tb.DTYPE_E4M3), tb.EUNSUPPORTED_SHAPE), ((1 << 22, 1 << 23, 120, 0, tb.DTYPE_BF16), tb.EINVAL),
                         ((1 << 22, 1 << 23, 0, 132, tb.DTYPE_BF16), tb.EALIGN), (((1 << 22) + 8, 1 << 23, 0, 0, tb.DTYPE_BF16), tb.EALIGN)]:
        assert tb.lib.tasp_cache_write(c, b, *args, None) == status
    for args, status in [((None, 1 << 22, tb.DTYPE_BF16), tb.EINVAL), ((1 << 22, 1 << 23, 5), tb.EUNSUPPORTED_SHAPE), ((1 << 22, (1 << 23) + 4, tb.DTYPE_FP32), tb.EALIGN)]:
        assert tb.lib.tasp_cache_read(c, b, *args, None) == status
    assert tb.lib.tasp_cache_write(None, b, 1 << 22, 1 << 23, 0, 0, tb.DTYPE_BF16, None) == tb.EINVAL
    assert tb.lib.tasp_cache_read(c, None, 1 << 22, 1 << 23, tb.DTYPE_BF16, None) == tb.EINVAL
    assert tb.lib.tasp_paged_attn(c, b, None, None) == tb.EINVAL


def test_calls_without_rows_or_sequences_do_nothing():
    for change in (dict(n_rows=0), dict(n_seqs=0)):
        c, b, a = _args(**change)
        assert tb.lib.tasp_cache_write(c, b, 1 << 22, 1 << 23, 0, 0, tb.DTYPE_BF16, None) == tb.OK
        assert tb.lib.tasp_cache_read(c, b, 1 << 22, 1 << 23, tb.DTYPE_BF16, None) == tb.OK
        assert tb.lib.tasp_paged_attn(c, b, a, None) == tb.OK


def test_binding_refuses_what_it_cannot_pass_on():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="device tensor"):
        tb.PagedCache(k, k)
    with pytest.raises(ValueError, match="n_pages"):
        tb.PagedCache(k.half(), k.half())
    with pytest.raises(ValueError, match="need k_scale"):
        tb.PagedCache(k.to(torch.float8_e4m3fn), k.to(torch.float8_e4m3fn))
    with pytest.raises(ValueError, match="no scales"):
        tb.PagedCache(k, k, k, k)
    with pytest.raises(ValueError, match="device tensor"):
        tb.PagedBatch(ints(2, 3), ints(2), ints(3), 1)
    with pytest.raises(ValueError, match="expected page_table"):
        tb.PagedBatch(ints(2, 3), ints(3), ints(3), 1)
    with pytest.raises(ValueError, match="int32"):
        tb.PagedBatch(ints(2, 3).long(), ints(2), ints(3), 1)
    for bad in (torch.zeros(4, 2, 64), torch.zeros(5, 2, 32, dtype=torch.bfloat16), torch.zeros(4, 2, 128, dtype=torch.bfloat16)[..., ::2],
                torch.zeros(4, 4, 64, dtype=torch.bfloat16)[:, ::2], torch.zeros(1, 2, 64, dtype=torch.bfloat16).expand(4, 2, 64)):
        with pytest.raises(ValueError):
            tb._rows("q", bad, 2, 64, 4, (torch.bfloat16,))
    fused = torch.zeros(4, 3 * 128, dtype=torch.bfloat16)
    assert tb._rows("q", fused[:, 128:256].view(4, 2, 64), 2, 64, 4, (torch.bfloat16,)) == 384


# ---- index arithmetic of the kernels on lists that hold anything
PROGRAM = r"""
#include "paged.hpp"
#include <cstdio>
#include <cstdlib>
#include <vector>
using namespace tasp;
static unsigned long long state = 88172645463325252ull;
static unsigned rnd() { state ^= state << 13; state ^= state >> 7; state ^= state << 17; return static_cast<unsigned>(state >> 32); }
static long long bad = 0;
static void expect(bool ok, const char* what) { if (!ok && bad++ < 5) std::printf("%s\n", what); }
template <int BM, int BT>
static void tiles(const PagedAttn& p, const std::vector<int>& seen) {
  for (int b = 0; b < p.c.n_seqs; ++b) {
    const PagedSeq s = load_seq(p.c, b);
    expect(s.r0 >= 0 && s.n >= 0 && s.r0 + s.n <= p.c.n_rows && s.kv >= 0, "sequence");
    const PagedCost c = cost_of<BM>(p, s);
    const int row_tiles = c.row_tiles;
    expect(static_cast<int64_t>(row_tiles) * BM >= static_cast<int64_t>(s.n) * p.G && c.first > 0 && c.step >= 0, "cost");
    for (int i = 0; i < row_tiles; ++i)
      for (int x : {cost_upto(c, i), (cost_upto(c, i) + cost_upto(c, i + 1)) / 2, cost_upto(c, i + 1) - 1}) expect(row_tile_at(c, x) == i, "row tile");
    for (int rt = 0; rt < row_tiles; ++rt) {
      const int rows = s.n * p.G, tok0 = rt * BM / p.G, tok1 = (lesser(rt * BM + BM, rows) - 1) / p.G;
      const PagedKeys k = keys_of<BM, BT>(p, s, tok0, tok1);
      expect(k.end >= 0 && k.end <= p.c.cap && k.n_tiles >= 0, "tiles");
      // every visible key of every row is in a tile, and no tile comes twice
      int last = -1;
      for (int u = 0; u < k.n_tiles; ++u) { expect(k.tile(u) > last && k.tile(u) * BT < k.end, "order"); last = k.tile(u); }
      for (int tok = tok0; tok <= tok1; ++tok)
        for (int t = 0; t < lesser(s.kv, p.c.cap); ++t) {
          const int pos = s.kv - s.n + tok;
          if (p.causal && t > pos) continue;
          if (p.window && !(static_cast<int64_t>(t) > static_cast<int64_t>(pos) - p.window || t < p.sinks)) continue;
          bool in = false;
          for (int u = 0; u < k.n_tiles && !in; ++u) in = t / BT == k.tile(u);
          expect(in && t < k.end, "a visible key is in no tile");
        }
      for (int u = 0; u < k.n_tiles; ++u)
        for (int i = 0; i < BT; i += 16) {
          const int pos = k.tile(u) * BT + i;
          if (pos >= k.end) continue;
          const long long at = static_cast<long long>(b) * p.c.max_pages + (pos >> p.c.ps_log2);
          expect(at >= 0 && at < static_cast<long long>(seen.size()) && (pos >> p.c.ps_log2) < p.c.max_pages, "table");
          const int page = page_of(p.c, b, pos);
          expect(page >= -1 && page < p.c.n_pages, "page");
        }
    }
  }
}
// The runs of all workers: every key tile of every row tile is taken once, by the workers that the sum of the parts goes by.
template <int BM, int BT>
static void runs(const PagedAttn& p) {
  int64_t all = 0;
  for (int b = 0; b < p.c.n_seqs; ++b) { const PagedCost c = cost_of<BM>(p, load_seq(p.c, b)); all += cost_upto(c, c.row_tiles) * p.c.Hkv; }
  expect(all < (1 << 30), "all");
  const int64_t share = share_of_all(p, static_cast<int>(all));
  int64_t start = 0;
  for (int b = 0; b < p.c.n_seqs; ++b) {
    const PagedSeq s = load_seq(p.c, b);
    const PagedCost c = cost_of<BM>(p, s);
    for (int i = 0; i < c.row_tiles * p.c.Hkv; ++i) {
      const int64_t cost = c.first + i % c.row_tiles * c.step;
      const int tiles = rnd() % 50;
      const int64_t first = (start + p.snap + share - 1) / share - 1, last = cost < p.snap ? -1 : (start + cost - p.snap) / share;
      const bool parts = cost >= 2 * p.snap && first < last;
      int upto = 0, takers = 0;
      for (int64_t w = larger<int64_t>(start / share - 1, 0); w <= (start + cost) / share; ++w) {
        const int64_t from = w * share, to = from + share;
        if (to <= start || from >= start + cost) continue;
        const int64_t x0 = snapped(static_cast<int>(larger<int64_t>(from - start, 0)), cost, p.snap), x1 = to - start >= cost ? cost : snapped(static_cast<int>(to - start), cost, p.snap);
        if (x0 >= x1) continue;
        expect(w < p.workers, "worker");
        expect(parts ? w >= first && w <= last && (x0 == 0) == (w == first) : x0 == 0 && x1 == cost, "part");
        expect(key_tile_at(x0, cost, tiles) == upto, "gap");
        upto = key_tile_at(x1, cost, tiles);
        // what the worker that starts a row tile says of the last one
        if (parts && x0 == 0) expect(w + 1 + (start + cost - p.snap - to) / share == last, "last worker");
        ++takers;
      }
      expect(upto == tiles && takers == (parts ? last - first + 1 : 1), "row tile not taken whole");
      start += cost;
    }
  }
}
int main() {
  for (int round = 0; round < 400; ++round) {
    const bool wild = round % 2 == 0;
    const int ps_log2 = 4 + rnd() % 3, max_pages = 1 + rnd() % 6, n_seqs = 1 + rnd() % 5, n_rows = 1 + rnd() % 60;
    std::vector<int> table(n_seqs * max_pages), kv(n_seqs), start(n_seqs + 1);
    for (int& x : table) x = wild ? static_cast<int>(rnd()) : static_cast<int>(rnd() % 8);
    for (int& x : kv) x = wild && rnd() % 2 ? static_cast<int>(rnd()) : static_cast<int>(rnd() % (max_pages << ps_log2));
    for (int i = 0; i <= n_seqs; ++i) start[i] = wild ? (rnd() % 2 ? static_cast<int>(rnd()) : static_cast<int>(rnd() % (n_rows + 1))) : n_rows * i / n_seqs;
    PagedAttn p{};
    p.c.table = table.data(); p.c.kv_len = kv.data(); p.c.row_start = start.data();
    p.c.n_pages = 7; p.c.ps_log2 = ps_log2; p.c.Hkv = 2; p.c.n_seqs = n_seqs; p.c.max_pages = max_pages; p.c.n_rows = n_rows; p.c.cap = max_pages << ps_log2;
    p.G = 1 + rnd() % 9; p.tile_cost = 1; p.causal = rnd() % 4 != 0; p.window = p.causal && rnd() % 2 ? 1 + rnd() % 100 : 0; p.sinks = p.window ? rnd() % 70 : 0;
    if (p.window && rnd() % 5 == 0) { p.window = 1 << 30; p.sinks = 2147483647; }
    for (int bm : {16, 32, 128}) {
      expect(set_cut(p, bm, 1 + rnd() % 300, 1 + rnd() % 50, 1 + rnd() % 100, 1 + rnd() % 200), "cut");
      if (round % 3 == 0) { p.key_shift = rnd() % 4; p.tile_cost = 1 + rnd() % 3; p.snap = 1 + rnd() % 3; }
      if (!wild && bm == 16) runs<16, 64>(p);
      if (!wild && bm == 32) runs<32, 64>(p);
      if (!wild && bm == 128) runs<128, 64>(p);
    }
    tiles<16, 64>(p, table);
    tiles<32, 64>(p, table);
    tiles<128, 64>(p, table);
    for (int b = 0; b < n_seqs; ++b)
      for (int row = 0; row < n_rows; ++row) {
        const PagedPlace at = place_of(p.c, b, row);
        expect(at.page >= -1 && at.page < p.c.n_pages && at.slot >= 0 && at.slot < (1 << ps_log2), "place");
      }
  }
  // the largest batches that are taken keep all work countable
  for (int i = 0; i < 2000; ++i) {
    PagedAttn p{};
    p.c.Hkv = 1 + rnd() % 64; p.G = 1 + rnd() % 64; p.c.cap = 16 << rnd() % 27; p.c.n_seqs = 1 + rnd() % 5000;
    p.c.n_rows = static_cast<int>(lesser<int64_t>(((int64_t{1} << 26) / p.c.Hkv - p.c.n_seqs) * 16 / p.G, rnd() % (1 << rnd() % 31) + 1));
    if (p.c.n_rows < 1) continue;
    for (int bm : {16, 32, 128}) expect(set_cut(p, bm, 512, 128, 256, 256), "not countable");
  }
  // lists that fall, so that sequences share rows, can carry the sum of all work past 32 bits: a run's last worker is one of the call's
  for (int i = 0; i < 2000; ++i) {
    PagedAttn p{};
    p.workers = 1 + rnd() % 1000; p.snap = 1 + rnd() % 16;
    PagedRun<16, true> r{};
    r.share = 1 + rnd() % 100; r.cost = p.snap + rnd() % 1000000; r.at = rnd() % 1000000; r.to = r.at + rnd() % (r.cost - p.snap + 1);
    const int worker = rnd() % p.workers, last = r.last_worker(p, worker);
    expect(last >= worker && last < p.workers, "a worker that is none");
  }
  return bad != 0;
}
"""


@pytest.mark.skipif(shutil.which(HIPCC) is None, reason="hipcc not found")
def test_index_arithmetic_stays_inside(tmp_path):
    src, exe = tmp_path / "paged.cpp", tmp_path / "paged"
    src.write_text(PROGRAM)
    root = os.path.dirname(os.path.dirname(os.path.abspath(asm_checks.__file__)))
    subprocess.run([HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-std=c++17", "-I" + os.path.join(root, "include"), "-I" + os.path.join(root, "paper_2509_26541_amd", "csrc"), str(src), "-o", str(exe)],
                   check=True, capture_output=True, text=True)
    got = subprocess.run([str(exe)], capture_output=True, text=True)
    assert got.returncode == 0, got.stdout
