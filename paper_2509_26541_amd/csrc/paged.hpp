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

// The clipped lists of a sequence: n rows from r0 on, kv tokens.
struct PagedSeq { int n, kv, r0; };
__host__ __device__ __forceinline__ PagedSeq load_seq(const PagedView& p, int i) {
  PagedSeq s{0, 0, 0};
  if (i < p.n_seqs) {
    const int a = p.row_start[i], e = p.row_start[i + 1], len = p.kv_len[i];
    s.r0 = lesser(larger(a, 0), p.n_rows);
    s.n = lesser(larger(e, s.r0), p.n_rows) - s.r0;
    s.kv = lesser(larger(len, 0), p.cap);
  }
  return s;
}
// Page of position pos (0 <= pos < cap) of sequence b, or -1.
__host__ __device__ __forceinline__ int page_of(const PagedView& p, int b, int pos) {
  const int page = p.table[static_cast<int64_t>(b) * p.max_pages + (pos >> p.ps_log2)];
  return page >= 0 && page < p.n_pages ? page : -1;
}
// Where a row of sequence b lives: page and slot, or page -1.
struct PagedPlace { int page, slot; };
__host__ __device__ __forceinline__ PagedPlace place_of(const PagedView& p, int b, int64_t row) {
  const int64_t pos = static_cast<int64_t>(lesser(larger(p.kv_len[b], 0), p.cap)) - p.row_start[b + 1] + row;
  if (pos < 0 || pos >= p.cap) return {-1, 0};
  return {page_of(p, b, static_cast<int>(pos)), static_cast<int>(pos) & ((1 << p.ps_log2) - 1)};
}

// Value of an exponent byte.
__device__ __forceinline__ float scale_value(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }

// ---- attention: the rows (token, query head of the group) of a sequence and KV head in tiles of BM, their keys in tiles of BT
struct PagedAttn {
  PagedView c;
  const void* q;
  void* out;
  float* lse;
  float* part;                   // workspace: partial results
  int64_t q_stride;              // elements between the tokens of q
  int32_t Hq, G, causal, window, sinks, out_fp32;
  float scale_log2e;
  int32_t workers;               // workgroups that share the keys
  Divider by_group;
};

// Keys of a row tile: n_first tiles of BT from position 0 on (what the first tokens need, where the window starts behind them), then
// those from tile `from` on; keys at and after `end` do not count.
struct PagedKeys {
  int n_first, from, n_tiles, end;
  __host__ __device__ __forceinline__ int tile(int u) const { return u < n_first ? u : u - n_first + from; }
};
template <int BM, int BT>
__host__ __device__ __forceinline__ PagedKeys keys_of(const PagedAttn& p, const PagedSeq& s, int tok0, int tok1) {
  PagedKeys k{0, 0, 0, 0};
  const int p0 = s.kv - s.n;
  k.end = larger(0, p.causal ? p0 + tok1 + 1 : s.kv);
  const int last = (k.end + BT - 1) / BT;
  if (p.window > 0) {
    k.from = lesser(larger(0, p0 + tok0 - p.window + 1) / BT, last);
    k.n_first = lesser((lesser(p.sinks, k.end) + BT - 1) / BT, k.from);
  }
  k.n_tiles = k.n_first + last - k.from;
  return k;
}

// What a sequence costs, in key tiles: row tiles, and key tiles of each of them at most.  A row tile without keys counts as
// one: its rows are written too.
template <int BM, int BT>
__host__ __device__ __forceinline__ void cost_of(const PagedAttn& p, const PagedSeq& s, int& row_tiles, int& key_tiles) {
  row_tiles = (s.n * p.G + BM - 1) / BM;
  int t = (s.kv + BT - 1) / BT;
  if (p.window > 0) {
    const int64_t w = (static_cast<int64_t>(lesser(p.sinks, s.kv)) + BT - 1) / BT + (static_cast<int64_t>(p.window) + BM / p.G + 1 + BT - 1) / BT + 1;
    t = static_cast<int>(lesser(static_cast<int64_t>(t), w));
  }
  key_tiles = larger(1, t);
}

// A value that all lanes have, in scalar registers.
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<int>(x)), hi = __builtin_amdgcn_readfirstlane(static_cast<int>(x >> 32));
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

__device__ __forceinline__ int64_t wave_prefix(int64_t x, int lane) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const int64_t y = __shfl_up(x, s);
    x += lane >= s ? y : 0;
  }
  return x;
}

// 64 sequences, one to a lane, with their work laid end to end: sequence after sequence, KV head after KV head, row tile after row
// tile, each `key_tiles` long.
template <int BM, int BT>
struct PagedChunk {
  int base;
  PagedSeq s;
  int row_tiles, key_tiles;
  int64_t len, upto;             // of the lane's sequence; with all before it in this chunk
  __device__ __forceinline__ void load(const PagedAttn& p, int first, int lane) {
    base = first;
    s = load_seq(p.c, first + lane);
    cost_of<BM, BT>(p, s, row_tiles, key_tiles);
    len = static_cast<int64_t>(row_tiles) * p.c.Hkv * key_tiles;
    upto = wave_prefix(len, lane);
  }
  __device__ __forceinline__ int64_t total() const { return before(64); }
  // work of the chunk's first `i` sequences
  __device__ __forceinline__ int64_t before(int i) const {
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(upto), i - 1), hi = __builtin_amdgcn_readlane(static_cast<int>(upto >> 32), i - 1);
    return i == 0 ? 0 : static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
  }
};

// All work of a call, and how much of it a worker takes.
template <int BM, int BT>
__device__ __forceinline__ int64_t share_of(const PagedAttn& p, PagedChunk<BM, BT>& c, int lane) {
  int64_t all = 0;
  for (int first = 0; first < p.c.n_seqs; first += 64) {
    c.load(p, first, lane);
    all += c.total();
  }
  if (c.base != 0) c.load(p, 0, lane);
  return uniform((all + p.workers - 1) / p.workers);
}

// Floats of a partial result: BM rows of d sums, their running maxima and their sums of weights.
constexpr int64_t part_floats(int bm, int d) { return static_cast<int64_t>(bm) * (d + 2); }

// Implemented in cache.hip and attn_paged.hip.
hipError_t launch_cache_write(const PagedView& c, bool e4m3, const void* k, const void* v, int64_t k_stride, int64_t v_stride, bool fp32, int d, hipStream_t stream);
hipError_t launch_cache_read(const PagedView& c, bool e4m3, void* k, void* v, bool fp32, int d, hipStream_t stream);
// workgroups that launch_paged_rows deals a call's keys to, and the bytes of their partial results
int paged_rows_workers(bool e4m3, int d);
int64_t paged_rows_workspace(bool e4m3, int d);
hipError_t launch_paged_rows(PagedAttn p, bool e4m3, int d, hipStream_t stream);

}  // namespace tasp
