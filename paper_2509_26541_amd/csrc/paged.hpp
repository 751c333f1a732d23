// A cache of K and V in pages, and a batch of sequences that live in it: what its kernels know, and how their work is cut.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "divider.hpp"
#include "gfx950.hpp"

namespace tasp {

// Row j of sequence b (rows row_start[b] .. row_start[b + 1] - 1 of the dense tensors) has position kv_len[b] - n_b + j.
// The lists are the caller's device memory and are not trusted: whatever they hold, no kernel leaves its buffers.
struct PagedView {
  unsigned char* k;              // [n_pages, Hkv, page_size, d]
  unsigned char* v;
  unsigned char* k_scale;        // [n_pages, Hkv, page_size] exponents of two, biased by 127 (e4m3 only)
  unsigned char* v_scale;
  const int32_t* table;          // [n_seqs, max_pages]
  const int32_t* kv_len;         // [n_seqs]
  const int32_t* row_start;      // [n_seqs + 1]
  int32_t n_pages, ps_log2, Hkv, n_seqs, max_pages, n_rows;
  int32_t cap;                   // positions the table has pages for, at most 2^30
};

template <class T>
__host__ __device__ __forceinline__ constexpr T lesser(T a, T b) { return b < a ? b : a; }
template <class T>
__host__ __device__ __forceinline__ constexpr T larger(T a, T b) { return a < b ? b : a; }

// The lists of a sequence, clipped: n rows from r0 on, kv tokens (of which those at and behind p.cap have no page).
struct PagedSeq { int n, kv, r0; };
__host__ __device__ __forceinline__ PagedSeq load_seq(const PagedView& p, int i) {
  PagedSeq s{0, 0, 0};
  if (i < p.n_seqs) {
    const int a = p.row_start[i], e = p.row_start[i + 1], len = p.kv_len[i];
    s.r0 = lesser(larger(a, 0), p.n_rows);
    s.n = lesser(larger(e, s.r0), p.n_rows) - s.r0;
    s.kv = larger(len, 0);
  }
  return s;
}
// Page of position pos (0 <= pos < cap) of sequence b, or -1.
__host__ __device__ __forceinline__ int page_of(const PagedView& p, int b, int pos) {
  const int page = p.table[static_cast<int64_t>(b) * p.max_pages + (pos >> p.ps_log2)];
  return page >= 0 && page < p.n_pages ? page : -1;
}
// Where a row of sequence b lives: page and slot, or page -1.  (The sequence's last row is the one that load_seq gives it: a list that reaches
// beyond the rows ends with them.)
struct PagedPlace { int page, slot; };
__host__ __device__ __forceinline__ PagedPlace place_of(const PagedView& p, int b, int64_t row) {
  const int64_t pos = static_cast<int64_t>(larger(p.kv_len[b], 0)) - lesser(p.row_start[b + 1], p.n_rows) + row;
  if (pos < 0 || pos >= p.cap) return {-1, 0};
  return {page_of(p, b, static_cast<int>(pos)), static_cast<int>(pos) & ((1 << p.ps_log2) - 1)};
}

// Value of an exponent byte.
__device__ __forceinline__ float scale_value(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }

// ---- attention: the rows (token, query head of the group) of a sequence and KV head in tiles of BM, their keys in tiles of BT
// The row tile that a worker's run ends in, if others go on with it: where its sequence's rows start in the dense tensors, how many they are
// (with the query heads of the group), and the last of those workers (the worker itself: there is none).
struct PagedSplit { int32_t r0, rows, head, rt, last, unused[3]; };

struct PagedAttn {
  PagedView c;
  const void* q;
  void* out;
  float* lse;
  float* part;                   // workspace: partial results, and
  PagedSplit* split;             // of each worker, the row tile that it starts and others end
  int64_t q_stride;              // elements between the tokens of q
  int32_t Hq, G, causal, window, sinks, out_fp32;
  float scale_log2e;
  double by_workers;             // 1 / workers
  int32_t workers;               // workgroups that share the work, and how they do, in parts of 2^key_shift keys (see PagedCost): what a row
  int32_t key_shift, tile_cost, snap, least_share;      // tile costs beside its keys, the least that is split off one, the least that a worker takes
  Divider by_group;
};

// Keys of a row tile: n_first tiles of BT from position 0 on (what the first tokens need, where the window starts behind them), then
// those from tile `from` on; keys at and after `end` do not count.
struct PagedKeys {
  int n_first, from, n_tiles, end;
  __host__ __device__ __forceinline__ int tile(int u) const { return u < n_first ? u : u - n_first + from; }
};
// The first key of the window of a row at `pos` (a key below 0 is none; pos, window and what comes of them are in 32 bits).
__host__ __device__ __forceinline__ int window_start(int pos, int window) { return larger(pos + 1, 0) - window; }
template <int BM, int BT>
__host__ __device__ __forceinline__ PagedKeys keys_of(const PagedAttn& p, const PagedSeq& s, int tok0, int tok1) {
  PagedKeys k{0, 0, 0, 0};
  const int p0 = s.kv - s.n;
  k.end = larger(0, lesser(p.causal ? p0 + tok1 + 1 : s.kv, p.c.cap));
  const int last = (k.end + BT - 1) / BT;
  if (p.window > 0) {
    k.from = lesser(larger(0, window_start(p0 + tok0, p.window)) / BT, last);
    k.n_first = lesser((lesser(p.sinks, k.end) + BT - 1) / BT, k.from);
  }
  k.n_tiles = k.n_first + last - k.from;
  return k;
}

// What the rows of a sequence cost, in parts of 2^key_shift keys (the host sees to it that all of a call stays below 2^30): row tile i of a KV
// head costs first + i step.  Under the causal mask later row tiles see more keys; with a window all are taken for as long as the longest.  Every
// row tile costs something: its rows are written.
struct PagedCost { int row_tiles, first, step; };
template <int BM>
__host__ __device__ __forceinline__ PagedCost cost_of(const PagedAttn& p, const PagedSeq& s) {
  PagedCost c{(s.n * p.G + BM - 1) / BM, 0, 0};
  const int kv = lesser(s.kv, p.c.cap);
  int keys = kv;
  if (p.causal && s.n <= kv) {
    keys = kv - s.n + lesser(s.n, BM / p.G + 1);
    c.step = (BM >> p.key_shift) / p.G;
    const int64_t most = static_cast<int64_t>(p.window) + BM / p.G + 64 + lesser(p.sinks, kv);
    if (p.window > 0 && keys + static_cast<int64_t>(s.n) > most) {
      keys = static_cast<int>(lesser<int64_t>(kv, most));
      c.step = 0;
    }
  }
  c.first = (keys >> p.key_shift) + p.tile_cost;
  // Row tiles that differ little count as equal: where there is one to a worker, no run ends inside.
  if (c.step * c.row_tiles <= c.first / 8) {
    c.first += c.step * c.row_tiles / 2;
    c.step = 0;
  }
  return c;
}
// All of the first n row tiles.
__host__ __device__ __forceinline__ int cost_upto(const PagedCost& c, int n) {
  return n * c.first + (c.step == 0 ? 0 : static_cast<int>(static_cast<int64_t>(n) * (n - 1) / 2 * c.step));
}
// The row tile that x parts into a KV head's work fall in (0 <= x < cost_upto(c, row_tiles)).
__host__ __device__ __forceinline__ int row_tile_at(const PagedCost& c, int x) {
  if (c.row_tiles <= 1) return 0;
  if (c.step == 0) return static_cast<int>(static_cast<uint32_t>(x) / static_cast<uint32_t>(c.first));
  const float b = static_cast<float>(c.first) - 0.5f * static_cast<float>(c.step), s = static_cast<float>(c.step);
  int i = lesser(larger(static_cast<int>(2.f * static_cast<float>(x) / (b + sqrtf(b * b + 2.f * s * static_cast<float>(x)))), 0), c.row_tiles - 1);
  while (i > 0 && cost_upto(c, i) > x) --i;
  while (i + 1 < c.row_tiles && cost_upto(c, i + 1) <= x) ++i;
  return i;
}
// A run that starts or ends x parts into a row tile of cost `cost` does so at a key tile; one that would leave less than `snap` (at least 1) on a
// side takes or leaves the row tile as a whole.
__host__ __device__ __forceinline__ int snapped(int x, int cost, int snap) { return x < snap ? 0 : cost - x < snap ? cost : x; }
__host__ __device__ __forceinline__ double reciprocal(double x) {          // about 1 / x
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_rcp(x);
#else
  return 1.0 / x;
#endif
}
__host__ __device__ __forceinline__ int key_tile_at(int x, int cost, int n_tiles) {
  return x >= cost ? n_tiles : lesser(static_cast<int>(static_cast<double>(x) * reciprocal(static_cast<double>(cost)) * n_tiles), n_tiles);
}
// A worker's share of all work.
__host__ __device__ __forceinline__ int share_of_all(const PagedAttn& p, int all) {
  return larger(static_cast<int>(static_cast<double>(all) * p.by_workers) + 1, p.least_share);
}

// Sums of the lanes up to and with each: lanes of a row of 16 pass theirs on by 1, 2, 4 and 8, then each row's and each half's last lane its own.
template <int CTRL, int ROWS>
__device__ __forceinline__ int passed_on(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_prefix(int x) {
  x += passed_on<0x111, 0xf>(x);
  x += passed_on<0x112, 0xf>(x);
  x += passed_on<0x114, 0xf>(x);
  x += passed_on<0x118, 0xf>(x);
  x += passed_on<0x142, 0xa>(x);
  x += passed_on<0x143, 0xc>(x);
  return x;
}

// 64 sequences, one to a lane, with their work laid end to end: sequence after sequence, KV head after KV head, row tile after row tile.
template <int BM>
struct PagedChunk {
  int base;
  PagedSeq s;
  PagedCost c;
  int upto;                      // work of this sequence and all before it in this chunk
  __device__ __forceinline__ void load(const PagedAttn& p, int first, int lane) { set(p, first, load_seq(p.c, first + lane)); }
  __device__ __forceinline__ void set(const PagedAttn& p, int first, const PagedSeq& seq) {
    base = first;
    s = seq;
    c = cost_of<BM>(p, s);
    upto = wave_prefix(cost_upto(c, c.row_tiles) * p.c.Hkv);
  }
  // work of the chunk's first `i` sequences
  __device__ __forceinline__ int before(int i) const { return i == 0 ? 0 : __builtin_amdgcn_readlane(upto, i - 1); }
};

// A worker's run of the call's work, one row tile (or piece of one) after the other.  KEEP: the lists of the chunk stay in registers;
// otherwise those of a sequence are read again when its turn comes.
template <int BM, bool KEEP>
struct PagedRun {
  PagedChunk<BM> chunk;
  int share, from, to;           // the run, in parts from the start of sequence b
  int b, seq, head, rt;          // (seq: its place in the chunk) the next row tile
  PagedSeq s;
  PagedCost c;
  int at, cost;                  // where it starts, and its cost
  int x0, x1;                    // what the run has of it

  __device__ __forceinline__ void take(const PagedAttn& p) {
    if constexpr (KEEP) {
      s.n = __builtin_amdgcn_readlane(chunk.s.n, seq);
      s.kv = __builtin_amdgcn_readlane(chunk.s.kv, seq);
      s.r0 = __builtin_amdgcn_readlane(chunk.s.r0, seq);
      c.row_tiles = __builtin_amdgcn_readlane(chunk.c.row_tiles, seq);
      c.first = __builtin_amdgcn_readlane(chunk.c.first, seq);
      c.step = __builtin_amdgcn_readlane(chunk.c.step, seq);
    } else {
      const PagedSeq one = load_seq(p.c, b);
      s.n = __builtin_amdgcn_readfirstlane(one.n);
      s.kv = __builtin_amdgcn_readfirstlane(one.kv);
      s.r0 = __builtin_amdgcn_readfirstlane(one.r0);
      c = cost_of<BM>(p, s);
    }
  }
  // false: no work for this worker
  __device__ __forceinline__ bool start(const PagedAttn& p, int worker, int lane) {
    // the sum of all chunks, each one's lists asked for a chunk ahead; lane i keeps the sum of chunk i
    int all = 0, sums = 0;
    PagedSeq ahead = load_seq(p.c, lane);
    for (int first = 0; first < p.c.n_seqs; first += 64) {
      const PagedSeq now = ahead;
      if (first + 64 < p.c.n_seqs) ahead = load_seq(p.c, first + 64 + lane);
      chunk.set(p, first, now);
      const int sum = chunk.before(64);
      sums = lane == first >> 6 ? sum : sums;
      all += sum;
    }
    share = __builtin_amdgcn_readfirstlane(share_of_all(p, all));
    from = share * worker;
    to = from + share;
    if (from >= all) return false;
    if (p.c.n_seqs > 64) {
      // the chunk: found among the sums, or from the first one on where there are more than 64
      int k = 0;
      if (p.c.n_seqs <= 64 * 64) {
        const int upto = wave_prefix(sums);
        k = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > from));
        const int before = k == 0 ? 0 : __builtin_amdgcn_readlane(upto, k - 1);
        from -= before;
        to -= before;
      }
      chunk.load(p, 64 * k, lane);
    }
    while (true) {
      const uint64_t behind = __builtin_amdgcn_ballot_w64(chunk.upto > from);
      seq = behind != 0 ? __builtin_ctzll(behind) : 64;
      const int before = chunk.before(seq);
      from -= before;
      to -= before;
      if (behind != 0) break;
      chunk.load(p, chunk.base + 64, lane);
    }
    b = chunk.base + seq;
    take(p);
    const int one = cost_upto(c, c.row_tiles);
    head = static_cast<int>(static_cast<uint32_t>(from) / static_cast<uint32_t>(one));
    rt = row_tile_at(c, from - head * one);
    at = head * one + cost_upto(c, rt);
    return true;
  }
  // false: the run is over
  __device__ __forceinline__ bool next(const PagedAttn& p, int lane) {
    while (at < to) {
      if (rt >= c.row_tiles) {
        rt = 0;
        ++head;
      }
      if (static_cast<uint32_t>(head) >= static_cast<uint32_t>(p.c.Hkv) || c.row_tiles == 0) {        // (below zero: see last_worker)
        head = rt = 0;
        from -= at;
        to -= at;
        at = 0;
        if (++b >= p.c.n_seqs) return false;
        if constexpr (KEEP)
          if (++seq == 64) {
            chunk.load(p, chunk.base + 64, lane);
            seq = 0;
          }
        take(p);
        continue;
      }
      cost = c.first + rt * c.step;
      x0 = snapped(larger(from - at, 0), cost, p.snap);
      x1 = to - at >= cost ? cost : snapped(to - at, cost, p.snap);
      if (x0 < x1) return true;
      step();
    }
    return false;
  }
  __device__ __forceinline__ void step() {
    at += cost;
    ++rt;
  }
  __device__ __forceinline__ bool whole() const { return x0 == 0 && x1 == cost; }
  // the last worker of a row tile that this one starts, for p.snap <= x1 < cost: runs end at `to` and every `share` behind it.  (Lists that fall, so
  // that sequences share rows, can carry the sum of all work past 32 bits: then the runs end before the row tile does.)
  __host__ __device__ __forceinline__ int last_worker(const PagedAttn& p, int worker) const {
    const int more = static_cast<int>(static_cast<uint32_t>(at + cost - p.snap - to) / static_cast<uint32_t>(share));
    return lesser(worker + 1 + more, p.workers - 1);
  }
};

// The host's part of the cut: up to `workers` of them, as many as can have work, and `tile_cost`, `snap` and `least_share` from keys to parts.
// False: more work than can be counted.
inline bool set_cut(PagedAttn& p, int bm, int workers, int tile_cost, int snap, int least_share) {
  const int64_t tiles = (static_cast<int64_t>(p.c.n_rows) * p.G / bm + p.c.n_seqs) * p.c.Hkv;
  const int64_t keys = static_cast<int64_t>(p.c.cap) + 2 * bm;
  p.workers = static_cast<int>(lesser<int64_t>(workers, tiles * (keys + tile_cost) / least_share + 1));
  p.by_workers = 1.0 / p.workers;
  for (p.key_shift = 0; p.key_shift <= 30; ++p.key_shift) {
    p.tile_cost = larger(1, tile_cost >> p.key_shift);
    p.snap = larger(1, snap >> p.key_shift);
    p.least_share = larger(1, least_share >> p.key_shift);
    if (tiles * ((keys >> p.key_shift) + 2 + p.tile_cost) < (int64_t{1} << 30)) return true;
  }
  return false;
}

// A partial result: BM rows of d normalised sums, their maxima (times c, to base 2), their sums of weights beside those (apart, since the maximum
// of very large scores would swallow the other's logarithm) and what rounding took from large maxima (see rest_of_product).  A worker leaves at most
// two: of the row tile that its run starts in, and of the one that it ends in.
constexpr int64_t part_floats(int bm, int d) { return static_cast<int64_t>(bm) * (d + 3); }
template <int BM, int D>
__device__ __forceinline__ float* part_of(const PagedAttn& p, int64_t worker, bool starts_inside) {
  return p.part + (2 * worker + (starts_inside ? 0 : 1)) * part_floats(BM, D);
}

// Implemented in cache.hip.
hipError_t launch_cache_write(const PagedView& c, bool e4m3, const void* k, const void* v, int64_t k_stride, int64_t v_stride, bool fp32, int d, hipStream_t stream);
hipError_t launch_cache_read(const PagedView& c, bool e4m3, void* k, void* v, bool fp32, int d, hipStream_t stream);
// Implemented in attn_paged.hip and attn_paged_tile.hip: the kernels for up to 32 rows (token, query head of the group) to a sequence and KV
// head (`rows`: the most, a hint), and for more; and the bytes of workspace that each takes.
hipError_t launch_paged_rows(const PagedAttn& p, bool e4m3, int d, int rows, hipStream_t stream);
int64_t paged_rows_workspace(const PagedAttn& p, bool e4m3, int d, int rows);
hipError_t launch_paged_tile(PagedAttn p, bool e4m3, int d, hipStream_t stream);
int64_t paged_tile_workspace(PagedAttn p, bool e4m3, int d);

}  // namespace tasp
