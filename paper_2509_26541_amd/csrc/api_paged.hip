// C entry points of the paged cache: checks of the arguments, and the launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "internal.hpp"
#include "paged.hpp"
#include "pipeline.hpp"
#include "tasp.h"

namespace {

using tasp::PagedView;
using tasp::larger;

constexpr int64_t kMost = int64_t{1} << 30;          // positions of a table, rows
bool misaligned(const void* p, uintptr_t by) { return (reinterpret_cast<uintptr_t>(p) & (by - 1)) != 0; }

int check_common(const tasp_paged_cache* c, const tasp_paged_batch* b, PagedView* out) {
  if (c == nullptr || b == nullptr) return TASP_EINVAL;
  const bool e4m3 = c->dtype == TASP_DTYPE_E4M3;
  if (c->k == nullptr || c->v == nullptr || (e4m3 && (c->k_scale == nullptr || c->v_scale == nullptr))) return TASP_EINVAL;
  if (c->n_pages < 1 || c->Hkv < 1 || c->page_size < 1) return TASP_EINVAL;
  if (b->n_seqs < 0 || b->n_rows < 0 || b->max_pages < 1 || b->max_rows < 0) return TASP_EINVAL;
  if (b->page_table == nullptr || b->kv_len == nullptr || b->row_start == nullptr) return TASP_EINVAL;
  if (c->dtype != TASP_DTYPE_BF16 && !e4m3) return TASP_EUNSUPPORTED_SHAPE;
  if (c->d != 64 && c->d != 128) return TASP_EUNSUPPORTED_SHAPE;
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0) return TASP_EUNSUPPORTED_SHAPE;
  if (c->n_pages > kMost || b->n_rows > kMost || static_cast<int64_t>(b->max_pages) * c->page_size > kMost) return TASP_EUNSUPPORTED_SHAPE;
  if (static_cast<int64_t>(c->Hkv) * c->page_size * c->d * 2 >= (int64_t{1} << 31)) return TASP_EUNSUPPORTED_SHAPE;      // a page's bytes,
  if (c->n_pages * c->Hkv * c->page_size >= (int64_t{1} << 32)) return TASP_EUNSUPPORTED_SHAPE;                                             // and all rows
  if (misaligned(c->k, 16) || misaligned(c->v, 16)) return TASP_EALIGN;
  if (e4m3 && (misaligned(c->k_scale, 16) || misaligned(c->v_scale, 16))) return TASP_EALIGN;
  if (misaligned(b->page_table, 4) || misaligned(b->kv_len, 4) || misaligned(b->row_start, 4)) return TASP_EALIGN;
  // indexes of (rows, heads), and the launches' grids, in 32 bits
  if (b->n_rows * c->Hkv > kMost || static_cast<int64_t>(b->n_seqs) * c->Hkv > kMost) return TASP_EUNSUPPORTED_SHAPE;
  PagedView v{};
  v.k = static_cast<unsigned char*>(c->k);
  v.v = static_cast<unsigned char*>(c->v);
  v.k_scale = c->k_scale;
  v.v_scale = c->v_scale;
  v.table = b->page_table;
  v.kv_len = b->kv_len;
  v.row_start = b->row_start;
  v.n_pages = static_cast<int32_t>(c->n_pages);
  while ((1 << v.ps_log2) < c->page_size) ++v.ps_log2;
  v.Hkv = c->Hkv;
  v.n_seqs = b->n_seqs;
  v.max_pages = b->max_pages;
  v.n_rows = static_cast<int32_t>(b->n_rows);
  v.cap = b->max_pages * c->page_size;
  *out = v;
  return TASP_OK;
}

bool rows_type(int32_t dtype) { return dtype == TASP_DTYPE_FP32 || dtype == TASP_DTYPE_BF16; }
int status_of(hipError_t e) { return e == hipSuccess ? TASP_OK : TASP_EHIP; }

// Rows (token, query head of the group) of a sequence and KV head, by the hint or the mean.  Up to kFew the kernel for few of them takes the call: it
// keeps more loads on their way, and its wavefronts all have work.  32 sequences of 16 000 tokens, 8 KV heads of 128: 32 rows e4m3 209 us with it,
// 241 with the other, bf16 323 and 365; 64 rows (it would walk the keys twice) e4m3 342 and 277, bf16 504 and 374.  A call runs one kernel for all of its
// sequences: 63 single tokens of 1 000 to 32 000 with a chunk of 2 048 of 16 384 take 857 us e4m3 and 811 bf16, apart 209 + 530 and 399 + 497.
constexpr int64_t kFew = 32;
int64_t rows_of(const tasp::PagedAttn& p, const tasp_paged_batch* b) {
  return (b->max_rows > 0 ? b->max_rows : (b->n_rows + larger(b->n_seqs, 1) - 1) / larger(b->n_seqs, 1)) * p.G;
}

int check_attn(const tasp_paged_cache* c, const tasp_paged_batch* b, const tasp_paged_attn_args* a, tasp::PagedAttn* out) {
  tasp::PagedAttn p{};
  const int st = check_common(c, b, &p.c);
  if (st != TASP_OK) return st;
  if (a == nullptr || a->Hq < 1 || a->Hq % c->Hkv != 0) return TASP_EINVAL;
  if (a->mask_mode != TASP_MASK_FULL && a->mask_mode != TASP_MASK_CAUSAL) return TASP_EINVAL;
  if (a->window < 0 || a->sinks < 0 || (a->window > 0 && a->mask_mode != TASP_MASK_CAUSAL)) return TASP_EINVAL;
  if (!(a->softmax_scale >= 0.f) || !std::isfinite(a->softmax_scale)) return TASP_EINVAL;
  if (!rows_type(a->out_dtype)) return TASP_EUNSUPPORTED_SHAPE;
  p.Hq = a->Hq;
  p.G = a->Hq / c->Hkv;
  if (b->n_rows * p.G > kMost || static_cast<int64_t>(p.G) > kMost || b->n_rows * a->Hq > (int64_t{1} << 36)) return TASP_EUNSUPPORTED_SHAPE;
  if ((b->n_rows * p.G / 16 + b->n_seqs) * c->Hkv > (int64_t{1} << 26)) return TASP_EUNSUPPORTED_SHAPE;           // row tiles, see set_cut
  const int64_t dense = static_cast<int64_t>(a->Hq) * c->d;
  p.q_stride = a->q_stride == 0 ? dense : a->q_stride;
  if (p.q_stride < dense) return TASP_EINVAL;
  if (p.q_stride % 8 != 0) return TASP_EALIGN;
  p.causal = a->mask_mode == TASP_MASK_CAUSAL;
  p.window = a->window;
  p.sinks = a->window > 0 ? a->sinks : 0;
  p.out_fp32 = a->out_dtype == TASP_DTYPE_FP32;
  p.scale_log2e = (a->softmax_scale == 0.f ? 1.f / std::sqrt(static_cast<float>(c->d)) : a->softmax_scale) * tasp::kLog2e;
  p.by_group = tasp::make_divider(static_cast<uint32_t>(p.G));
  p.q = a->q;
  p.out = a->out;
  p.lse = a->lse;
  p.part = static_cast<float*>(a->workspace);
  *out = p;
  return TASP_OK;
}

}  // namespace

extern "C" {

int tasp_cache_write(const tasp_paged_cache* c, const tasp_paged_batch* b, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                     int32_t dtype, void* hip_stream) {
  PagedView p;
  const int st = check_common(c, b, &p);
  if (st != TASP_OK) return st;
  if (k == nullptr || v == nullptr) return TASP_EINVAL;
  if (!rows_type(dtype)) return TASP_EUNSUPPORTED_SHAPE;
  const int64_t dense = static_cast<int64_t>(c->Hkv) * c->d;
  if (k_stride == 0) k_stride = dense;
  if (v_stride == 0) v_stride = dense;
  if (k_stride < dense || v_stride < dense) return TASP_EINVAL;
  if (k_stride % 8 != 0 || v_stride % 8 != 0 || misaligned(k, 16) || misaligned(v, 16)) return TASP_EALIGN;
  if (p.n_rows == 0 || p.n_seqs == 0) return TASP_OK;
  return status_of(tasp::launch_cache_write(p, c->dtype == TASP_DTYPE_E4M3, k, v, k_stride, v_stride, dtype == TASP_DTYPE_FP32, c->d, static_cast<hipStream_t>(hip_stream)));
}

int tasp_cache_read(const tasp_paged_cache* c, const tasp_paged_batch* b, void* k, void* v, int32_t dtype, void* hip_stream) {
  PagedView p;
  const int st = check_common(c, b, &p);
  if (st != TASP_OK) return st;
  if (k == nullptr || v == nullptr) return TASP_EINVAL;
  if (!rows_type(dtype)) return TASP_EUNSUPPORTED_SHAPE;
  if (misaligned(k, 16) || misaligned(v, 16)) return TASP_EALIGN;
  if (p.n_rows == 0 || p.n_seqs == 0) return TASP_OK;
  return status_of(tasp::launch_cache_read(p, c->dtype == TASP_DTYPE_E4M3, k, v, dtype == TASP_DTYPE_FP32, c->d, static_cast<hipStream_t>(hip_stream)));
}

size_t tasp_paged_attn_workspace_bytes(const tasp_paged_cache* c, const tasp_paged_batch* b, const tasp_paged_attn_args* a) {
  tasp::PagedAttn p;
  if (check_attn(c, b, a, &p) != TASP_OK) return 0;
  const int64_t rows = rows_of(p, b);
  const bool e4m3 = c->dtype == TASP_DTYPE_E4M3;
  return static_cast<size_t>(rows <= kFew ? tasp::paged_rows_workspace(p, e4m3, c->d, static_cast<int>(rows)) : tasp::paged_tile_workspace(p, e4m3, c->d));
}

int tasp_paged_attn(const tasp_paged_cache* c, const tasp_paged_batch* b, const tasp_paged_attn_args* a, void* hip_stream) {
  tasp::PagedAttn p;
  const int st = check_attn(c, b, a, &p);
  if (st != TASP_OK) return st;
  if (a->q == nullptr || a->out == nullptr || a->lse == nullptr) return TASP_EINVAL;
  if (misaligned(a->q, 16) || misaligned(a->out, 16) || misaligned(a->lse, 16)) return TASP_EALIGN;
  const size_t need = tasp_paged_attn_workspace_bytes(c, b, a);
  if (need > 0) {
    if (a->workspace == nullptr || a->workspace_bytes < need) return TASP_EWORKSPACE;
    if (misaligned(a->workspace, 256)) return TASP_EALIGN;
  }
  if (p.c.n_rows == 0 || p.c.n_seqs == 0) return TASP_OK;
  const bool e4m3 = c->dtype == TASP_DTYPE_E4M3;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const int64_t rows = rows_of(p, b);
  return status_of(rows <= kFew ? tasp::launch_paged_rows(p, e4m3, c->d, static_cast<int>(rows), stream) : tasp::launch_paged_tile(p, e4m3, c->d, stream));
}

}  // extern "C"
