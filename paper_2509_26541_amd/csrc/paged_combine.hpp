// The rows of a paged attention call whose keys several workgroups took, from their partial results; and the end of every row.
#pragma once
#include <hip/hip_runtime.h>

#include "internal.hpp"
#include "paged.hpp"
#include "pipeline.hpp"

namespace tasp {
namespace {

constexpr float kLeast = -3.0e38f;       // a running maximum before the first key: below any score that is a number

// Whether a running maximum m = score * c (rounded) is so large that the scores have to be taken off it before they are multiplied: fma(s, c, -m)
// is off by what rounding took from m, the same for all keys of the row, so that it cancels unless exp2 of it leaves the floats.
__device__ __forceinline__ bool beyond_fma(float m) { return m != kLeast && __builtin_fabsf(m) > 0x1p29f; }

// Sums with different references are joined by the references' difference.  A reference that is subtracted as the float it is needs nothing more; where
// the scores were taken off the maximum m itself, the reference is m c without rounding: its float and, exactly, what rounding left of it.  Up to 2^30
// that is at most 2^5, and the sums are multiplied by what it stands for; beyond, it goes along as the reference's rest, for joins whose largest reference
// is beyond 2^29 (all others are so far above a reference with a rest that this has no weight).  m: m c afterwards; `times`: what to multiply the sums by.
__device__ __forceinline__ float rest_of_product(float& m, float c, float& times) {
  times = 1.f;
  if (m == kLeast) return 0.f;
  const float product = m * c, rest = __builtin_fabsf(product) < __builtin_inff() ? __builtin_fmaf(m, c, -product) : 0.f;
  m = product;
  if (__builtin_fabsf(product) > 0x1p30f) return rest;
  times = fast_exp2(rest);
  return 0.f;
}
// One reference less another, to 2^-24 of it: where the floats are near each other their difference is exact, and a rest is at most 2^-24 of its float,
// about as far as two scores of that size lie apart.
__device__ __forceinline__ float less(float m, float rest, float of, float of_rest) { return (m - of) + (rest - of_rest); }

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

// What every worker leaves in p.split, once, at its end.
__device__ __forceinline__ void leave_split(const PagedAttn& p, int worker, const PagedSplit& split) {
  if (threadIdx.x == 0) p.split[worker] = split;
}

// A row tile whose keys several workgroups took: its partial results, in their order, 16 rows at a time (and up to 64 to a workgroup).  Where
// there are fewer, the threads of the others take their turn of the parts.
template <int D, int BM>
__global__ __launch_bounds__(256) void paged_combine_kernel(const PagedAttn p) {
  constexpr int EL = D / 16, ROWS = BM < 64 ? BM : 64, PER = BM / ROWS;
  const int worker = blockIdx.x / PER;
  const PagedSplit sp = p.split[worker];
  if (sp.last == worker) return;
  for (int first_row = blockIdx.x % PER * ROWS, end_row = first_row + ROWS; first_row < end_row; first_row += 16) {
    const int m0 = sp.rt * BM + first_row;
    if (m0 >= sp.rows) return;
    const int here = min(sp.rows - m0, 16);                       // rows of this workgroup
    const int turns = here > 8 ? 1 : here > 4 ? 2 : here > 2 ? 4 : here > 1 ? 8 : 16, per_turn = 16 / turns;
    const int group = threadIdx.x / 16, je = threadIdx.x % 16 * EL, turn = group / per_turn, jr = first_row + min(group % per_turn, here - 1);
    float top = kLeast, top_rest = 0.f, total = 0.f, acc[EL];
#pragma unroll
    for (int e = 0; e < EL; ++e) acc[e] = 0.f;
    // `N` parts from i0 on, every turns-th of them, all on their way at once
    auto add = [&](auto nn, int i0) __attribute__((always_inline)) {
      constexpr int N = decltype(nn)::value;
      float m[N], l[N];
      f32x4 x[N][EL / 4];
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int i = i0 + j * turns;
        const float* const src = part_of<BM, D>(p, i, i != worker);
        m[j] = src[BM * D + jr];
        l[j] = src[BM * D + BM + jr];
#pragma unroll
        for (int e = 0; e < EL / 4; ++e) x[j][e] = *reinterpret_cast<const f32x4*>(src + jr * D + je + 4 * e);
      }
      float m_new = top;
#pragma unroll
      for (int j = 0; j < N; ++j) m_new = fmaxf(m_new, m[j]);
      const float a = fast_exp2(top - m_new);
      total *= a;
#pragma unroll
      for (int e = 0; e < EL; ++e) acc[e] *= a;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float w = l[j] * fast_exp2(m[j] - m_new);          // (parts without keys are zeros)
        total += w;
#pragma unroll
        for (int e = 0; e < EL; ++e) acc[e] += x[j][e / 4][e % 4] * w;
      }
      top = m_new;
    };
    int i = worker + turn;
    for (; i + 7 * turns <= sp.last; i += 8 * turns) add(std::integral_constant<int, 8>{}, i);
    if (i + 3 * turns <= sp.last) { add(std::integral_constant<int, 4>{}, i); i += 4 * turns; }
    for (; i <= sp.last; i += turns) add(std::integral_constant<int, 1>{}, i);
    if (turns > 1) {                                              // (the same for the whole workgroup)
      __shared__ float sums[16][D + 4], tops[16], totals[16];
#pragma unroll
      for (int e = 0; e < EL; ++e) sums[group][je + e] = acc[e];
      if (je == 0) { tops[group] = top; totals[group] = total; }
      __syncthreads();
      if (turn > 0) return;                                       // (a row tile's last rows)
      float m_new = top;
      for (int t = 1; t < turns; ++t) m_new = fmaxf(m_new, tops[t * per_turn + group]);
      const float a = fast_exp2(top - m_new);
      total *= a;
#pragma unroll
      for (int e = 0; e < EL; ++e) acc[e] *= a;
      for (int t = 1; t < turns; ++t) {
        const int other = t * per_turn + group;
        const float w = fast_exp2(tops[other] - m_new);
        total += w * totals[other];
#pragma unroll
        for (int e = 0; e < EL; ++e) acc[e] += w * sums[other][je + e];
      }
      top = m_new;
    }
    const int m = m0 + group;
    if (group >= here) return;                                    // (so are these)
    if (__builtin_expect(beyond_fma(top), 0)) {                   // once more, one part after the other, with the references' rests
      top = kLeast; total = 0.f;
#pragma unroll
      for (int e = 0; e < EL; ++e) acc[e] = 0.f;
#pragma nounroll
      for (int part = worker; part <= sp.last; ++part) {
        const float* const src = part_of<BM, D>(p, part, part != worker);
        const float m_part = src[BM * D + jr], rest = src[BM * D + 2 * BM + jr], gap = less(m_part, rest, top, top_rest);
        const float a = gap > 0.f ? fast_exp2(-gap) : 1.f, w = src[BM * D + BM + jr] * (gap > 0.f ? 1.f : fast_exp2(gap));
        total = total * a + w;
#pragma unroll
        for (int e = 0; e < EL; ++e) acc[e] = acc[e] * a + src[jr * D + je + e] * w;
        top = gap > 0.f ? m_part : top;
        top_rest = gap > 0.f ? rest : top_rest;
      }
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
    for (int e = 0; e < EL; ++e) acc[e] *= inv;
    const int tok = divide(m, p.by_group);
    store_row<D, EL>(p, static_cast<int64_t>(sp.r0 + tok) * p.Hq + sp.head * p.G + (m - tok * p.G), je, acc, total == 0.f ? -__builtin_inff() : top + (top_rest + __builtin_amdgcn_logf(total)));
  }
}

template <int D, int BM>
hipError_t launch_paged_combine(const PagedAttn& p, hipStream_t stream) {
  return TASP_LAUNCH((paged_combine_kernel<D, BM>), dim3(static_cast<unsigned>(p.workers * (BM < 64 ? 1 : BM / 64))), dim3(256), stream, p);
}

// Bytes of the partial results of `workers` workgroups and of what they leave beside them, and where in a workspace these are.
constexpr int64_t part_bytes(int workers, int bm, int d) { return (2 * workers * part_floats(bm, d) * 4 + 255) / 256 * 256; }
inline int64_t workspace_of(const PagedAttn& p, int bm, int d) { return part_bytes(p.workers, bm, d) + p.workers * static_cast<int64_t>(sizeof(PagedSplit)); }
inline void place_split(PagedAttn& p, int bm, int d) {
  p.split = reinterpret_cast<PagedSplit*>(reinterpret_cast<unsigned char*>(p.part) + part_bytes(p.workers, bm, d));
}

}  // namespace
}  // namespace tasp
