// Rows of K and V into the pages of a cache, and back.
//
// A (token, KV head) pair is d consecutive values on both sides, so both kernels are streams of 16-byte pieces with the pages looked
// up on the way; what bounds them is HBM (few tokens: three dependent loads, the sequence, its page, the row: 1.9 us for one token).  Prompts of
// bf16 into e4m3 pages (68 859 tokens of 8 heads of 128) 92 us, 4.6 TB/s; 71 691 back 85 us, 5.2 TB/s; a large copy reaches 4.9 on this card.
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

template <class T, int N>
__device__ __forceinline__ void load_once(const T* p, T (&x)[N]) {
  constexpr int PER = 16 / sizeof(T);
  typedef T Vec __attribute__((ext_vector_type(PER)));
#pragma unroll
  for (int i = 0; i < N / PER; ++i) {
    const Vec y = __builtin_bit_cast(Vec, once(reinterpret_cast<const u32x4*>(p) + i));
#pragma unroll
    for (int e = 0; e < PER; ++e) x[i * PER + e] = y[e];
  }
}

// A lane has eight values of a row, D / 8 neighbouring lanes the whole of it: 16-byte pieces of bf16 that lie side by side.  A wavefront has 512 / D
// tokens and HEADS of their KV heads, so that what it has looked up serves more bytes.  The same calls on two inputs in turn (a part of which the
// caches then hold): writing e4m3 86 us with four heads, 98 with one, reading 86 and 108; from fp32 rows 141 and 148; bf16 pages, where the bytes
// outweigh the look-up, 111 and 109, 107 and 103.  With sixteen values to a lane, 16 bytes of e4m3: writing 86, reading 98, and 194 from fp32 rows,
// whose pieces do not lie side by side then.
constexpr int kPiece = 8;
template <int D>
constexpr int kTokens = 64 * kPiece / D;

template <int D, bool F8, class T, int HEADS>
__global__ __launch_bounds__(kThreads) void cache_write_kernel(const PagedView c, const T* k, const T* v, int64_t k_stride, int64_t v_stride) {
  constexpr int N = kPiece, LPR = D / N;
  const int lane = threadIdx.x & 63, piece = lane % LPR, groups = (c.Hkv + HEADS - 1) / HEADS;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head0 = static_cast<int>(item % groups) * HEADS;
  const int64_t row0 = item / groups * kTokens<D>, row = row0 + lane / LPR, rc = min(row, static_cast<int64_t>(c.n_rows) - 1);
  if (row0 >= c.n_rows) return;
  T x[HEADS][2][N];
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int head = min(head0 + i, c.Hkv - 1);
    load_once(k + rc * k_stride + head * D + piece * N, x[i][0]);
    load_once(v + rc * v_stride + head * D + piece * N, x[i][1]);
  }
  const PagedPlace at = place_of_row(c, row, lane);
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int head = head0 + i;
    if (HEADS > 1 && head >= c.Hkv) break;
    const int64_t out_row = ((static_cast<int64_t>(max(at.page, 0)) * c.Hkv + head) << c.ps_log2) + at.slot;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      unsigned char* const dst = (s == 0 ? c.k : c.v) + (out_row * D + piece * N) * (F8 ? 1 : 2);
      if constexpr (F8) {
        float y[N], top = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const float z = static_cast<float>(x[i][s][e]);
          const bool finite = __builtin_fabsf(z) < __builtin_inff();
          top = fmaxf(top, finite ? __builtin_fabsf(z) : 0.f);
          y[e] = finite ? z : __builtin_nanf("");
        }
#pragma unroll
        for (int m = 1; m < LPR; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
        // top = 2^e (1 + f): at most 448 = 2^8 1.75 times 2^(e - 8) if 1 + f <= 1.75, twice that otherwise
        const unsigned bits = __builtin_bit_cast(unsigned, top);
        const int byte = max(static_cast<int>(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), kScaleLeast);
        const float inv = scale_value(254 - byte), most = byte == 247 ? 240.f : 448.f;      // (256 2^120 would be beyond the floats)
        u32x2 w;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float q[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float z = y[4 * j + e] * inv;
            q[e] = z > most ? most : z < -most ? -most : z;            // (NaN stays)
          }
          const int u = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
          w[j] = static_cast<unsigned>(__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], u, true));
        }
        if (at.page >= 0) {
          *reinterpret_cast<u32x2*>(dst) = w;
          if (piece == 0) (s == 0 ? c.k_scale : c.v_scale)[out_row] = static_cast<unsigned char>(byte);
        }
      } else {
        bf16x8 y;
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = static_cast<__bf16>(x[i][s][e]);
        if (at.page >= 0) *reinterpret_cast<bf16x8*>(dst) = y;
      }
    }
  }
}

template <int D, bool F8, class T, int HEADS>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(const PagedView c, T* k, T* v) {
  constexpr int N = kPiece, LPR = D / N;
  const int lane = threadIdx.x & 63, piece = lane % LPR, groups = (c.Hkv + HEADS - 1) / HEADS;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head0 = static_cast<int>(item % groups) * HEADS;
  const int64_t row0 = item / groups * kTokens<D>, row = row0 + lane / LPR;
  if (row0 >= c.n_rows) return;
  const PagedPlace at = place_of_row(c, row, lane);
  u32x4 x[HEADS][2];
  float scale[HEADS][2];
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int head = min(head0 + i, c.Hkv - 1);
    const int64_t in_row = ((static_cast<int64_t>(max(at.page, 0)) * c.Hkv + head) << c.ps_log2) + at.slot;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      x[i][s] = u32x4{0u, 0u, 0u, 0u};
      scale[i][s] = 0.f;
      if (at.page < 0) continue;
      const unsigned char* const src = (s == 0 ? c.k : c.v) + (in_row * D + piece * N) * (F8 ? 1 : 2);
      if constexpr (F8) {
        const u32x2 y = once(reinterpret_cast<const u32x2*>(src));
        x[i][s][0] = y[0]; x[i][s][1] = y[1];
      } else {
        x[i][s] = once(reinterpret_cast<const u32x4*>(src));
      }
      if constexpr (F8) scale[i][s] = scale_value((s == 0 ? c.k_scale : c.v_scale)[in_row]);
    }
  }
  // a row behind the last sequence is left as it is
  if (row >= c.n_rows || row >= c.row_start[c.n_seqs] || row < c.row_start[0]) return;
#pragma unroll
  for (int i = 0; i < HEADS; ++i) {
    const int head = head0 + i;
    if (HEADS > 1 && head >= c.Hkv) break;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      T* const dst = (s == 0 ? k : v) + (row * c.Hkv + head) * D + piece * N;
      float y[N];
#pragma unroll
      for (int j = 0; j < (F8 ? 2 : 4); ++j) {
        if constexpr (F8) {
          const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(x[i][s][j], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(x[i][s][j], true);
          y[4 * j] = a[0] * scale[i][s]; y[4 * j + 1] = a[1] * scale[i][s];
          y[4 * j + 2] = b[0] * scale[i][s]; y[4 * j + 3] = b[1] * scale[i][s];
        } else {
          y[2 * j] = __builtin_bit_cast(float, x[i][s][j] << 16);
          y[2 * j + 1] = __builtin_bit_cast(float, x[i][s][j] & 0xffff0000u);
        }
      }
      if constexpr (sizeof(T) == 4) {
        reinterpret_cast<f32x4*>(dst)[0] = f32x4{y[0], y[1], y[2], y[3]};
        reinterpret_cast<f32x4*>(dst)[1] = f32x4{y[4], y[5], y[6], y[7]};
      } else {
        bf16x8 z;
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = static_cast<__bf16>(y[e]);
        *reinterpret_cast<bf16x8*>(dst) = z;
      }
    }
  }
}

template <int D>
int64_t items_of(const PagedView& c, int heads) {
  return (static_cast<int64_t>(c.n_rows) + kTokens<D> - 1) / kTokens<D> * ((c.Hkv + heads - 1) / heads);
}
constexpr int kHeads = 4;
constexpr int64_t kFull = 256 * 32;          // wavefronts that the chip holds: as many items keep it busy

template <int D, bool F8, class T, int HEADS>
hipError_t launch_one(const PagedView& c, const void* k, const void* v, int64_t ks, int64_t vs, bool write, hipStream_t stream) {
  const int64_t blocks = (items_of<D>(c, HEADS) + kThreads / 64 - 1) / (kThreads / 64);
  if (blocks > INT_MAX) return hipErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(blocks)), block(kThreads);
  if (write) return TASP_LAUNCH((cache_write_kernel<D, F8, T, HEADS>), grid, block, stream, c, static_cast<const T*>(k), static_cast<const T*>(v), ks, vs);
  return TASP_LAUNCH((cache_read_kernel<D, F8, T, HEADS>), grid, block, stream, c, static_cast<T*>(const_cast<void*>(k)), static_cast<T*>(const_cast<void*>(v)));
}
template <int D, bool F8, class T>
hipError_t launch_form(const PagedView& c, const void* k, const void* v, int64_t ks, int64_t vs, bool write, hipStream_t stream) {
  return items_of<D>(c, kHeads) >= kFull ? launch_one<D, F8, T, kHeads>(c, k, v, ks, vs, write, stream) : launch_one<D, F8, T, 1>(c, k, v, ks, vs, write, stream);
}
template <int D, bool F8>
hipError_t launch_typed(const PagedView& c, const void* k, const void* v, int64_t ks, int64_t vs, bool write, bool fp32, hipStream_t stream) {
  return fp32 ? launch_form<D, F8, float>(c, k, v, ks, vs, write, stream) : launch_form<D, F8, __bf16>(c, k, v, ks, vs, write, stream);
}
hipError_t launch(const PagedView& c, bool e4m3, const void* k, const void* v, int64_t ks, int64_t vs, bool write, bool fp32, int d, hipStream_t stream) {
  if (c.n_rows == 0) return hipSuccess;
  if (d == 64) return e4m3 ? launch_typed<64, true>(c, k, v, ks, vs, write, fp32, stream) : launch_typed<64, false>(c, k, v, ks, vs, write, fp32, stream);
  return e4m3 ? launch_typed<128, true>(c, k, v, ks, vs, write, fp32, stream) : launch_typed<128, false>(c, k, v, ks, vs, write, fp32, stream);
}

}  // namespace

hipError_t launch_cache_write(const PagedView& c, bool e4m3, const void* k, const void* v, int64_t ks, int64_t vs, bool fp32, int d, hipStream_t stream) {
  return launch(c, e4m3, k, v, ks, vs, true, fp32, d, stream);
}
hipError_t launch_cache_read(const PagedView& c, bool e4m3, void* k, void* v, bool fp32, int d, hipStream_t stream) {
  return launch(c, e4m3, k, v, 0, 0, false, fp32, d, stream);
}

}  // namespace tasp
