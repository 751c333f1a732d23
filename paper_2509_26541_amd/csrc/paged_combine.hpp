// The rows of a paged attention call whose keys several workgroups took, from their partial results; and the end of every row.
#pragma once
#include <hip/hip_runtime.h>

#include <climits>

#include "internal.hpp"
#include "paged.hpp"
#include "pipeline.hpp"

namespace tasp {
namespace {

// EL values from `col` on of the row (token, query head) at index rh, and its log-sum-exp (base 2; -inf: no key).
template <int D, int EL>
__device__ __forceinline__ void store_row(const PagedAttn& p, int64_t rh, int col, const float (&x)[EL], float lse2) {
  if (p.out_fp32) {
    float* const dst = static_cast<float*>(p.out) + rh * D + col;
#pragma unroll
    for (int e = 0; e < EL; e += 4) *reinterpret_cast<f32x4*>(dst + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
  } else {
    __bf16* const dst = static_cast<__bf16*>(p.out) + rh * D + col;
#pragma unroll
    for (int e = 0; e < EL; e += 4)
      *reinterpret_cast<bf16x4*>(dst + e) = bf16x4{static_cast<__bf16>(x[e]), static_cast<__bf16>(x[e + 1]), static_cast<__bf16>(x[e + 2]), static_cast<__bf16>(x[e + 3])};
  }
  if (col == 0) p.lse[rh] = lse2 * kLn2;
}

// A row tile whose keys several workgroups took: its partial results, in their order.  One workgroup to 16 rows of a row tile.
template <int D, int BM, int BT>
__global__ __launch_bounds__(256) void paged_combine_kernel(const PagedAttn p) {
  constexpr int EL = D / 16, PER = BM / 16;
  const int thread = threadIdx.x, lane = thread & 63;
  PagedChunk<BM, BT> chunk;
  const int64_t share = share_of<BM, BT>(p, chunk, lane);
  int64_t unit = blockIdx.x / PER, start = 0;
  int seq;
  while (true) {
    const int64_t upto = wave_prefix(static_cast<int64_t>(chunk.c.row_tiles) * p.c.Hkv);
    const uint64_t behind = __builtin_amdgcn_ballot_w64(upto > unit);
    if (behind != 0) {
      seq = __builtin_ctzll(behind);
      if (seq > 0) unit -= of_lane(upto, seq - 1);
      start += chunk.before(seq);
      break;
    }
    unit -= of_lane(upto, 63);
    start += chunk.before(64);
    if (chunk.base + 64 >= p.c.n_seqs) return;
    chunk.load(p, chunk.base + 64, lane);
  }
  const PagedCost c{static_cast<int>(__builtin_amdgcn_readlane(chunk.c.row_tiles, seq)), of_lane(chunk.c.first, seq), of_lane(chunk.c.step, seq)};
  const int n = __builtin_amdgcn_readlane(chunk.s.n, seq), r0 = __builtin_amdgcn_readlane(chunk.s.r0, seq);
  const int head = static_cast<int>(unit) / c.row_tiles, rt = static_cast<int>(unit) - head * c.row_tiles;
  start += head * cost_upto(c, c.row_tiles) + cost_upto(c, rt);
  const int64_t cost = c.first + rt * c.step;
  // runs that end inside the row tile: those of workers first .. last - 1, ends snapped to neither side
  if (cost < 2 * p.snap) return;
  const int64_t first = quotient(start + p.snap + share - 1, share) - 1, last = quotient(start + cost - p.snap, share);
  if (first >= last) return;
  const int jr = blockIdx.x % PER * 16 + thread / 16, je = thread % 16 * EL, m = rt * BM + jr;
  if (m >= n * p.G) return;
  float top = -__builtin_inff(), total = 0.f, acc[EL];
#pragma unroll
  for (int e = 0; e < EL; ++e) acc[e] = 0.f;
  // `N` of them from i0 on, all on their way at once
  auto add = [&](auto nn, int64_t i0) __attribute__((always_inline)) {
    constexpr int N = decltype(nn)::value;
    float l[N];
    f32x4 x[N][EL / 4];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float* const src = part_of<BM, D>(p, i0 + j, i0 + j != first);
      l[j] = src[BM * D + jr];
#pragma unroll
      for (int e = 0; e < EL / 4; ++e) x[j][e] = *reinterpret_cast<const f32x4*>(src + jr * D + je + 4 * e);
    }
    float l_new = top;
#pragma unroll
    for (int j = 0; j < N; ++j) l_new = fmaxf(l_new, l[j]);
    const float a = top == l_new ? 1.f : fast_exp2(top - l_new);
    total *= a;
#pragma unroll
    for (int e = 0; e < EL; ++e) acc[e] *= a;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float w = l[j] == -__builtin_inff() ? 0.f : fast_exp2(l[j] - l_new);       // (parts without keys are zeros)
      total += w;
#pragma unroll
      for (int e = 0; e < EL; ++e) acc[e] += x[j][e / 4][e % 4] * w;
    }
    top = l_new;
  };
  int64_t i = first;
  for (; i + 7 <= last; i += 8) add(std::integral_constant<int, 8>{}, i);
  if (i + 3 <= last) { add(std::integral_constant<int, 4>{}, i); i += 4; }
  for (; i <= last; ++i) add(std::integral_constant<int, 1>{}, i);
  const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
  for (int e = 0; e < EL; ++e) acc[e] *= inv;
  const int tok = divide(m, p.by_group);
  store_row<D, EL>(p, static_cast<int64_t>(r0 + tok) * p.Hq + head * p.G + (m - tok * p.G), je, acc, top + __builtin_amdgcn_logf(total));
}

template <int D, int BM, int BT>
hipError_t launch_paged_combine(const PagedAttn& p, hipStream_t stream) {
  const int64_t blocks = (static_cast<int64_t>(p.c.n_rows) * p.G / BM + p.c.n_seqs) * p.c.Hkv * (BM / 16);
  if (blocks > INT_MAX) return hipErrorInvalidValue;
  return TASP_LAUNCH((paged_combine_kernel<D, BM, BT>), dim3(static_cast<unsigned>(blocks)), dim3(256), stream, p);
}

}  // namespace
}  // namespace tasp
