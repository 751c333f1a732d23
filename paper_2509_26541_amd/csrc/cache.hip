// Rows of K and V into the pages of a cache, and back.
//
// A (token, KV head) pair is d consecutive values on both sides, so both kernels are streams of 16-byte pieces with the pages looked
// up on the way; what bounds them is HBM (few tokens: three dependent loads, the sequence, its page, the row).
// e4m3 rows have one scale, a power of two: the smallest with which the row's largest finite magnitude is at most 448.  Dividing by
// it is exact, so each value is rounded once, and value times scale is exact in bf16 (4 bits and 8 of exponent).
#include <hip/hip_runtime.h>

#include <climits>

#include "internal.hpp"
#include "paged.hpp"

namespace tasp {
namespace {

constexpr int kThreads = 256;
constexpr int kScaleLeast = 27;          // 2^-100: scale times the smallest e4m3 value is still a normal float

// The place of a row of the dense tensors.
__device__ __forceinline__ PagedPlace place_of_row(const PagedView& c, int64_t row, int lane) {
  // the last sequence that starts at or before the wavefront's first row: 64 starts at a time
  const int first = __builtin_amdgcn_readfirstlane(static_cast<int>(row));
  int b = -1;
  for (int i = 0; i <= c.n_seqs; i += 64) {
    const bool in = i + lane <= c.n_seqs && c.row_start[min(i + lane, c.n_seqs)] <= first;
    b += __popcll(__builtin_amdgcn_ballot_w64(in));
  }
  // rows of a wavefront mostly belong to one sequence; the others go on from there
  while (b < c.n_seqs && c.row_start[b + 1] <= row) ++b;
  return b < 0 || b >= c.n_seqs || row >= c.n_rows ? PagedPlace{-1, 0} : place_of(c, b, row);
}

// Both sides are read and written once: no place in the caches is asked for.
template <class T>
__device__ __forceinline__ T once(const T* p) { return __builtin_nontemporal_load(p); }

template <class T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    const f32x4 a = once(reinterpret_cast<const f32x4*>(p)), b = once(reinterpret_cast<const f32x4*>(p) + 1);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
  } else {
    const bf16x8 a = __builtin_bit_cast(bf16x8, once(reinterpret_cast<const u32x4*>(p)));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = static_cast<float>(a[e]);
  }
}

// A lane has eight values of a row, D / 8 neighbouring lanes the whole of it; a wavefront has 512 / D tokens of one KV head.
template <int D, bool F8, class T>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(const PagedView c, const T* k, const T* v, int64_t k_stride, int64_t v_stride) {
  constexpr int LPR = D / 8, TOK = 64 / LPR;
  const int lane = threadIdx.x & 63, piece = lane % LPR;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = static_cast<int>(item % c.Hkv);
  const int64_t row0 = item / c.Hkv * TOK, row = row0 + lane / LPR, rc = min(row, static_cast<int64_t>(c.n_rows) - 1);
  if (row0 >= c.n_rows) return;
  float x[2][8];
  load8(k + rc * k_stride + head * D + piece * 8, x[0]);
  load8(v + rc * v_stride + head * D + piece * 8, x[1]);
  const PagedPlace at = place_of_row(c, row, lane);
  const int64_t out_row = ((static_cast<int64_t>(max(at.page, 0)) * c.Hkv + head) << c.ps_log2) + at.slot;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    unsigned char* const pages = s == 0 ? c.k : c.v;
    if constexpr (F8) {
      float top = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool finite = __builtin_fabsf(x[s][e]) < __builtin_inff();
        top = fmaxf(top, finite ? __builtin_fabsf(x[s][e]) : 0.f);
        x[s][e] = finite ? x[s][e] : __builtin_nanf("");
      }
#pragma unroll
      for (int m = 1; m < LPR; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
      // top = 2^e (1 + f): at most 448 = 2^8 1.75 times 2^(e - 8) if 1 + f <= 1.75, twice that otherwise
      const unsigned bits = __builtin_bit_cast(unsigned, top);
      const int byte = max(static_cast<int>(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), kScaleLeast);
      const float inv = scale_value(254 - byte), most = byte == 247 ? 240.f : 448.f;      // (256 2^120 would be beyond the floats)
      unsigned w[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float z = x[s][4 * j + e] * inv;
          y[e] = z > most ? most : z < -most ? -most : z;            // (NaN stays)
        }
        int u = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        w[j] = static_cast<unsigned>(__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], u, true));
      }
      if (at.page >= 0) {
        *reinterpret_cast<u32x2*>(pages + out_row * D + piece * 8) = u32x2{w[0], w[1]};
        if (piece == 0) (s == 0 ? c.k_scale : c.v_scale)[out_row] = static_cast<unsigned char>(byte);
      }
    } else {
      bf16x8 y;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = static_cast<__bf16>(x[s][e]);
      if (at.page >= 0) *reinterpret_cast<bf16x8*>(pages + (out_row * D + piece * 8) * 2) = y;
    }
  }
}

template <int D, bool F8, class T>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(const PagedView c, T* k, T* v) {
  constexpr int LPR = D / 8, TOK = 64 / LPR;
  const int lane = threadIdx.x & 63, piece = lane % LPR;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = static_cast<int>(item % c.Hkv);
  const int64_t row0 = item / c.Hkv * TOK, row = row0 + lane / LPR;
  if (row0 >= c.n_rows) return;
  const PagedPlace at = place_of_row(c, row, lane);
  const int64_t in_row = ((static_cast<int64_t>(max(at.page, 0)) * c.Hkv + head) << c.ps_log2) + at.slot;
  float x[2][8];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const unsigned char* const pages = s == 0 ? c.k : c.v;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[s][e] = 0.f;
    if (at.page < 0) continue;
    if constexpr (F8) {
      const u32x2 w = once(reinterpret_cast<const u32x2*>(pages + in_row * D + piece * 8));
      const float scale = scale_value((s == 0 ? c.k_scale : c.v_scale)[in_row]);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w[j], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w[j], true);
        x[s][4 * j] = a[0] * scale; x[s][4 * j + 1] = a[1] * scale;
        x[s][4 * j + 2] = b[0] * scale; x[s][4 * j + 3] = b[1] * scale;
      }
    } else {
      load8(reinterpret_cast<const __bf16*>(pages) + in_row * D + piece * 8, x[s]);
    }
  }
  // a row behind the last sequence is left as it is
  if (row >= c.n_rows || row >= c.row_start[c.n_seqs] || row < c.row_start[0]) return;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    T* const dst = (s == 0 ? k : v) + (row * c.Hkv + head) * D + piece * 8;
    if constexpr (sizeof(T) == 4) {
      reinterpret_cast<f32x4*>(dst)[0] = f32x4{x[s][0], x[s][1], x[s][2], x[s][3]};
      reinterpret_cast<f32x4*>(dst)[1] = f32x4{x[s][4], x[s][5], x[s][6], x[s][7]};
    } else {
      bf16x8 y;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = static_cast<__bf16>(x[s][e]);
      *reinterpret_cast<bf16x8*>(dst) = y;
    }
  }
}

int64_t blocks_for(const PagedView& c, int d) {
  const int64_t items = (static_cast<int64_t>(c.n_rows) + 512 / d - 1) / (512 / d) * c.Hkv;
  return (items + kThreads / 64 - 1) / (kThreads / 64);
}

template <int D, bool F8, class T>
hipError_t write_as(const PagedView& c, const void* k, const void* v, int64_t ks, int64_t vs, int64_t blocks, hipStream_t stream) {
  return TASP_LAUNCH((cache_write_kernel<D, F8, T>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), stream, c, static_cast<const T*>(k),
                     static_cast<const T*>(v), ks, vs);
}
template <int D, bool F8, class T>
hipError_t read_as(const PagedView& c, void* k, void* v, int64_t blocks, hipStream_t stream) {
  return TASP_LAUNCH((cache_read_kernel<D, F8, T>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), stream, c, static_cast<T*>(k), static_cast<T*>(v));
}

}  // namespace

hipError_t launch_cache_write(const PagedView& c, bool e4m3, const void* k, const void* v, int64_t ks, int64_t vs, bool fp32, int d, hipStream_t stream) {
  const int64_t blocks = blocks_for(c, d);
  if (blocks == 0) return hipSuccess;
  if (blocks > INT_MAX) return hipErrorInvalidValue;
#define TASP_FORM(D, F8, T) return write_as<D, F8, T>(c, k, v, ks, vs, blocks, stream)
  if (d == 64) {
    if (e4m3) { if (fp32) TASP_FORM(64, true, float); TASP_FORM(64, true, __bf16); }
    if (fp32) TASP_FORM(64, false, float);
    TASP_FORM(64, false, __bf16);
  }
  if (e4m3) { if (fp32) TASP_FORM(128, true, float); TASP_FORM(128, true, __bf16); }
  if (fp32) TASP_FORM(128, false, float);
  TASP_FORM(128, false, __bf16);
#undef TASP_FORM
}

hipError_t launch_cache_read(const PagedView& c, bool e4m3, void* k, void* v, bool fp32, int d, hipStream_t stream) {
  const int64_t blocks = blocks_for(c, d);
  if (blocks == 0) return hipSuccess;
  if (blocks > INT_MAX) return hipErrorInvalidValue;
#define TASP_FORM(D, F8, T) return read_as<D, F8, T>(c, k, v, blocks, stream)
  if (d == 64) {
    if (e4m3) { if (fp32) TASP_FORM(64, true, float); TASP_FORM(64, true, __bf16); }
    if (fp32) TASP_FORM(64, false, float);
    TASP_FORM(64, false, __bf16);
  }
  if (e4m3) { if (fp32) TASP_FORM(128, true, float); TASP_FORM(128, true, __bf16); }
  if (fp32) TASP_FORM(128, false, float);
  TASP_FORM(128, false, __bf16);
#undef TASP_FORM
}

}  // namespace tasp
