// Attention of a few new tokens over a paged cache: 16 or 32 (token, query head of the group) rows to a tile.
//
// S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_16x16x32_bf16, softmax in one pass (running maximum and sum).  A grouped head's K and V
// are read once for all 16 rows.  Every wavefront takes keys of its own, in stages of 32, through a part of LDS of its own that loads
// fill directly: no barrier inside the loop, and the loads run ahead of the products by the stages behind the first.
// What bounds it is HBM: per key and KV head 4 d bytes (e4m3: 2 d + 2) for 4 d 16 products.  One token of 500 003, 8 KV heads of 128: 312 us,
// 6.6 TB/s of 7.0 that a kernel that only reads gets; 64 sequences of e4m3, 1 000 to 32 000 tokens, 193 us, 6.2 TB/s.  One token of 700 is latency:
// 6.5 us, and 3.2 for the joining kernel.
//
// The work of a call (sequence after sequence, KV head after KV head, row tile after row tile, in key tiles) is cut into equal runs,
// one for a workgroup; where a run ends inside a row tile, partial results go to the workspace and paged_combine_kernel adds them up,
// always in the same order.  The lengths are on the device, so every workgroup works out its own run.
//
// Rounding: P goes into the second product as two bf16 (its value and what rounding that left, 2^-17 of it), which costs a second
// matrix instruction that HBM hides; everything else is fp32.  e4m3 values are exact in bf16, their scales (powers of two) multiply the
// scores and the probabilities.
#include <hip/hip_runtime.h>

#include <climits>

#include "internal.hpp"
#include "paged.hpp"
#include "paged_combine.hpp"
#include "pipeline.hpp"

namespace tasp {
namespace {

// NR times 16 rows to a tile.
template <int D, bool F8, int NR>
struct RowsCfg {
  static constexpr int BM = 16 * NR, WK = 32;            // rows of a tile; keys of a stage
  static constexpr int RB = D * (F8 ? 1 : 2);            // bytes of a row in the cache
  static constexpr int UNITS = RB / 16, RPL = 64 / UNITS, LOADS = WK / RPL;       // 16-byte units of it; rows to a wavefront's load; loads to a stage's K
  static constexpr int NW = 2;                           // wavefronts
  static constexpr int PER_CU = F8 ? (D == 128 || NR == 2 ? 4 : 6) : (D == 128 ? 2 : 4);      // workgroups that a compute unit holds
  static constexpr int NS = 2;                           // stages in LDS
  static constexpr int BT = NW * WK;
  static constexpr int STAGE = 2 * WK * RB + (F8 ? 256 : 0), PER_STAGE = 2 * LOADS + (F8 ? 1 : 0);
  static constexpr int LIST = 256;                       // pages a wavefront looks up at once, one for every 16 keys
  static constexpr int ROW = D + 4;                      // floats of a row of sums while they are joined
  static constexpr int RING = NW * NS * STAGE, JOIN = NW * 16 * ROW * 4 + NW * 16 * 12, LDS = RING > JOIN ? RING : JOIN;
  static constexpr int NDB = D / 16;
  // 16-byte units of a stage's row are kept at unit ^ swz: the 16 rows that one read takes a unit (K) or two (V) of then lie in different banks
  __device__ static int swz_k(int r) { return (r / (16 / UNITS)) % UNITS; }
  __device__ static int swz_v(int r) {
    if constexpr (!F8) return 2 * ((r / (16 / UNITS)) % (UNITS / 2));
    else if constexpr (D == 128) return ((r >> 1) & 3) | (r >> 4 << 2);
    else return ((r >> 2) & 1) | (r >> 4 << 1);
  }
};

__device__ __forceinline__ bf16x8 widen(u32x2 w) {
  union { bf16x2 p[4]; bf16x8 v; } r;
  r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], 1.0f, false);
  r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[0], 1.0f, true);
  r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], 1.0f, false);
  r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[1], 1.0f, true);
  return r.v;
}

__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

typedef int i32x2v __attribute__((ext_vector_type(2)));
typedef i32x2v __attribute__((address_space(3))) * lds_i32x2_ptr;

template <int D, bool F8, int NR>
__global__ __launch_bounds__((RowsCfg<D, F8, NR>::NW * 64), (RowsCfg<D, F8, NR>::NW * RowsCfg<D, F8, NR>::PER_CU / 4)) void paged_rows_kernel(const PagedAttn p) {
  using C = RowsCfg<D, F8, NR>;
  constexpr int NW = C::NW, NS = C::NS, BT = C::BT, BM = C::BM, NDB = C::NDB, RB = C::RB;
  __shared__ __attribute__((aligned(256))) unsigned char smem[C::LDS];
  __shared__ int pages[NW][C::LIST];
  const int thread = threadIdx.x, w = __builtin_amdgcn_readfirstlane(thread >> 6), lane = thread & 63;
  const int g = lane >> 4, lq = lane & 15;
  const float c = p.scale_log2e;
  unsigned char* const ring = smem + w * NS * C::STAGE;

  PagedRun<BM, true> run;
  const int worker = xcd_contiguous(blockIdx.x, p.workers);
  PagedSplit split{0, 0, 0, 0, worker, {0, 0, 0}};
  if (!run.start(p, worker, lane)) {
    leave_split(p, worker, split);
    return;
  }
  const unsigned page_bytes = (static_cast<unsigned>(p.c.Hkv) << p.c.ps_log2) * RB;            // (below 2^31, the host sees to it)
  const int ps_mask = (1 << p.c.ps_log2) - 1;
  for (; run.next(p, lane); run.step()) {
    const PagedSeq& s = run.s;
    const int b = run.b, head = scalar(run.head), rt = scalar(run.rt);
    const bool whole = run.whole();
    if (run.x0 == 0 && !whole) split = PagedSplit{run.s.r0, run.s.n * p.G, head, rt, run.last_worker(p, worker), {0, 0, 0}};

    // ---- the rows
    const int rows = s.n * p.G;
    const int tok0 = divide(rt * BM, p.by_group), tok1 = divide(min(rt * BM + BM, rows) - 1, p.by_group);
    PagedKeys keys = keys_of<BM, BT>(p, s, tok0, tok1);
    const int p0 = s.kv - s.n;
    const int all_to = min(p.causal ? p0 + tok0 : INT_MAX, keys.end - 1), all_from = p.window > 0 ? window_start(p0 + tok1, p.window) : INT_MIN;
    int see_to[NR], see_from[NR];                  // the lane's rows see keys up to the one, from the other on or among the first
    bf16x8 qf[NR][D / 32];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int m = min(rt * BM + 16 * n + lq, rows - 1), tok = divide(m, p.by_group);
      see_to[n] = min(p.causal ? p0 + tok : INT_MAX, keys.end - 1);
      see_from[n] = p.window > 0 ? window_start(p0 + tok, p.window) : INT_MIN;
      const __bf16* const src = static_cast<const __bf16*>(p.q) + static_cast<int64_t>(s.r0 + tok) * p.q_stride + static_cast<int64_t>(head * p.G + m - tok * p.G) * D;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) qf[n][j] = *reinterpret_cast<const bf16x8*>(src + (F8 ? 64 * (j / 2) + 16 * g + 8 * (j % 2) : 32 * j + 8 * g));
    }
    f32x4 o[NR][NDB];
    float m_run[NR], l_run[NR], l_lo[NR], m_rest[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) m_rest[n] = 0.f;

    // (what the loads and the loop go by is the same in all lanes, and said to be)
    const int t0 = scalar(key_tile_at(run.x0, run.cost, keys.n_tiles)), t1 = scalar(key_tile_at(run.x1, run.cost, keys.n_tiles));
    keys.n_first = scalar(keys.n_first);
    keys.from = scalar(keys.from);
    keys.end = scalar(keys.end);
    const int64_t head_bytes = (static_cast<int64_t>(head) << p.c.ps_log2) * RB;
    const unsigned char* const k_head = p.c.k + head_bytes;
    const unsigned char* const v_head = p.c.v + head_bytes;
    // ---- pages of the wavefront's keys, up to LIST / 2 tiles at a time (as far as the loads go, NS tiles behind the last)
    int listed = t0;
    const int32_t* const table = p.c.table + static_cast<int64_t>(b) * p.c.max_pages;
    auto look_up = [&](int t) {
      listed = t;
#pragma unroll
      for (int i = 0; i < C::LIST / 64; ++i) {
        if (i > 0 && t + 32 * i >= t1 + NS) break;
        const int u = t + 32 * i + lane / 2, pos = keys.tile(u) * BT + w * C::WK + lane % 2 * 16;
        const bool there = u < t1 && pos < keys.end;
        const int page = table[there ? pos >> p.c.ps_log2 : 0];
        pages[w][64 * i + lane] = there && page >= 0 && page < p.c.n_pages ? page : -1;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    auto listed_pages = [&](int u) {
      if (u - listed >= C::LIST / 2) look_up(u);
      return *reinterpret_cast<const i32x2v*>(&pages[w][(u - listed) * 2]);
    };
    // K and V of the wavefront's 32 keys of tile u into stage st; keys behind the end and keys without a page come as zeros.
    // `paged` takes two bits a tile: whether each 16 keys have a page.
    unsigned paged = 0;
    auto fetch = [&](int u, int st, i32x2v listed_at) {
      const int page[2] = {__builtin_amdgcn_readfirstlane(listed_at[0]), __builtin_amdgcn_readfirstlane(listed_at[1])};
      const int pos0 = keys.tile(u) * BT + w * C::WK;
      unsigned char* const dst = ring + st * C::STAGE;
      paged = paged << 2 | (page[0] >= 0 ? 1u : 0u) | (page[1] >= 0 ? 2u : 0u);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int pos = pos0 + 16 * i;
        const int64_t base = static_cast<int64_t>(static_cast<uint64_t>(static_cast<unsigned>(max(page[i], 0))) * page_bytes) + static_cast<unsigned>((pos & ps_mask) * RB);
        const int n = max(0, scalar(min(16, keys.end - pos)));       // (both bounds at once would be a vector instruction)
        const unsigned records = page[i] < 0 ? 0u : static_cast<unsigned>(n) * RB;
        const u32x4 kb = raw_buffer(k_head + base, records), vb = raw_buffer(v_head + base, records);
#pragma unroll
        for (int j = 0; j < C::LOADS / 2; ++j) {
          const int r = 16 * i + j * C::RPL + lane / C::UNITS;       // of the stage's 32
          const unsigned soff = min(static_cast<unsigned>(j * C::RPL * RB), records);
          const unsigned row = static_cast<unsigned>(lane / C::UNITS * RB), un = lane % C::UNITS;
          buffer_to_lds_16_once(kb, soff, row + (un ^ C::swz_k(r)) * 16, dst + (16 * i + j * C::RPL) * RB);
          buffer_to_lds_16_once(vb, soff, row + (un ^ C::swz_v(r)) * 16, dst + (C::WK + 16 * i + j * C::RPL) * RB);
        }
      }
      if constexpr (F8) {
        // the scales: 16 bytes for each 16 keys of K, then of V
        const int pg = max(lane & 4 ? page[1] : page[0], 0), slot = (pos0 + (lane & 4) * 4) & ps_mask;
        const unsigned char* const sc = (lane & 8 ? p.c.v_scale : p.c.k_scale) + ((static_cast<int64_t>(pg) * p.c.Hkv + head) << p.c.ps_log2) + slot + lane % 4 * 4;
        const unsigned to = static_cast<unsigned>(reinterpret_cast<size_t>((lds_void_ptr)(dst + 2 * C::WK * RB)));
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(to), "v"(sc) : "memory");
      }
    };

    // Zero times an infinity or a NaN would carry V's values to rows that do not see them, and what rounding left of a probability,
    // times an infinity, is NaN for those that do.  Sums that are not finite are formed again, with the rows of V that hold
    // such values taken out of the product and added one by one; so are those behind very large scores (see beyond_fma).
    auto pass = [&](auto careful) {
      float m_raise[NR];
#pragma unroll
      for (int n = 0; n < NR; ++n) {
#pragma unroll
        for (int i = 0; i < NDB; ++i) o[n][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_run[n] = m_raise[n] = kLeast;
        l_run[n] = l_lo[n] = 0.f;
      }
      if (t0 < t1) {
        look_up(t0);
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int j = 0; j < D / 32; ++j) asm volatile("" : "+v"(qf[n][j]));     // (the compiler waits for them here, not in the loop)
        for (int i = 0; i < NS; ++i) fetch(t0 + i, i, listed_pages(t0 + i));
      }
      for (int t = t0, st = 0; t < t1; ++t, st = st + 1 == NS ? 0 : st + 1) {
        const i32x2v soon = listed_pages(t + NS);
        asm volatile("s_waitcnt vmcnt(%0)" : : "n"((NS - 1) * C::PER_STAGE) : "memory");
        const unsigned char* const kl = ring + st * C::STAGE;
        unsigned char* const vl = ring + st * C::STAGE + C::WK * RB;
        const int pos0 = keys.tile(t) * BT + w * C::WK;
        const unsigned has = paged >> (2 * (NS - 1)) & 3;
        // ---- scores: those of keys 4 g .. 4 g + 3 and 16 + 4 g .. of the lane's rows
        float x[NR][8], vs[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          f32x4 sc[NR];
#pragma unroll
          for (int n = 0; n < NR; ++n) sc[n] = f32x4{0.f, 0.f, 0.f, 0.f};
          const int r = 16 * i + lq;
          auto product = [&](bf16x8 kf, int j) {
#pragma unroll
            for (int n = 0; n < NR; ++n) sc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[n][j], sc[n], 0, 0, 0);
          };
          if constexpr (!F8) {
#pragma unroll
            for (int j = 0; j < D / 32; ++j) product(*reinterpret_cast<const bf16x8*>(kl + r * RB + ((4 * j + g) ^ C::swz_k(r)) * 16), j);
          } else {
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
              const u32x4 k16 = *reinterpret_cast<const u32x4*>(kl + r * RB + ((4 * j + g) ^ C::swz_k(r)) * 16);
              product(widen(u32x2{k16[0], k16[1]}), 2 * j);
              product(widen(u32x2{k16[2], k16[3]}), 2 * j + 1);
            }
          }
          if constexpr (F8) {
            const unsigned kw = *reinterpret_cast<const unsigned*>(kl + 2 * C::WK * RB + 16 * i + 4 * g);
            const unsigned vw = *reinterpret_cast<const unsigned*>(kl + 2 * C::WK * RB + 32 + 16 * i + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float ks = scale_value(kw >> 8 * e & 255);
#pragma unroll
              for (int n = 0; n < NR; ++n) x[n][4 * i + e] = sc[n][e] * ks;
              vs[4 * i + e] = scale_value(vw >> 8 * e & 255);
            }
          } else {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) x[n][4 * i + e] = sc[n][e];
          }
        }
        unsigned seen[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) seen[n] = 0xff;
        if (!(has == 3 && pos0 + C::WK - 1 <= all_to && (pos0 >= all_from || pos0 + C::WK <= p.sinks))) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int pos = pos0 + 16 * (e / 4) + 4 * g + e % 4;
            const bool there = (has >> (e / 4) & 1) != 0 && pos < keys.end;
#pragma unroll
            for (int n = 0; n < NR; ++n) {
              const bool ok = there && pos <= see_to[n] && (pos >= see_from[n] || pos < p.sinks);
              seen[n] &= ok ? 0xffu : ~(1u << e);
              x[n][e] = ok ? x[n][e] : -__builtin_inff();
            }
            if constexpr (F8) vs[e] = there ? vs[e] : 0.f;       // (a scale behind the end may be anything)
          }
        }
        bf16x8 hi[NR], lo[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          // ---- softmax: the running maximum is only raised when it grew by more than 2^8
          // (careful: m_run is the maximum of the scores themselves, and nothing is rounded before it is taken off)
          constexpr bool EXACT = decltype(careful)::value;
          const float mx = fmaxf(fmaxf(fmaxf(x[n][0], x[n][1]), fmaxf(x[n][2], x[n][3])), fmaxf(fmaxf(x[n][4], x[n][5]), fmaxf(x[n][6], x[n][7])));
          if (__builtin_amdgcn_ballot_w64((EXACT ? mx : mx * c) > m_raise[n]) != 0) {
            float m_new = fmaxf(mx, __shfl_xor(mx, 16));
            m_new = fmaxf(m_new, __shfl_xor(m_new, 32));
            m_new = fmaxf(m_run[n], EXACT ? m_new : m_new * c);
            const float alpha = fast_exp2(EXACT ? (m_run[n] - m_new) * c : m_run[n] - m_new);
            m_run[n] = m_new;
            m_raise[n] = EXACT ? m_new : m_new + kRescaleGap;
            l_run[n] *= alpha; l_lo[n] *= alpha;
#pragma unroll
            for (int i = 0; i < NDB; ++i) o[n][i] *= alpha;
          }
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[n][e] = fast_exp2(EXACT ? (x[n][e] - m_run[n]) * c : __builtin_fmaf(x[n][e], c, -m_run[n]));
            sum += x[n][e];
            if constexpr (F8) x[n][e] *= vs[e];
            hi[n][e] = static_cast<__bf16>(x[n][e]);
            lo[n][e] = static_cast<__bf16>(x[n][e] - static_cast<float>(hi[n][e]));
          }
          // in two levels, so that a few large terms do not swallow many small ones
          l_lo[n] += sum;
          if ((t & 63) == 63) { l_run[n] += l_lo[n]; l_lo[n] = 0.f; }
        }

        if constexpr (decltype(careful)::value) {
          // (places formed here: outside the loop they would take registers from it)
          int ln = lane;
          asm volatile("" : "+v"(ln));
          const int cg = ln >> 4, cq = ln & 15;
          // rows of V with a value that is not finite: two lanes look at each
          bool odd = false;
#pragma unroll
          for (int i = 0; i < RB / 32; ++i) {
            const u32x4 y = *reinterpret_cast<const u32x4*>(vl + ln / 2 * RB + (ln % 2 * (RB / 32) + i) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if constexpr (F8) {
#pragma unroll
                for (int f = 0; f < 4; ++f) odd |= (y[e] >> 8 * f & 0x7f) == 0x7f;
              } else {
                odd |= (y[e] & 0x7f80u) == 0x7f80u || (y[e] & 0x7f800000u) == 0x7f800000u;
              }
            }
          }
          uint64_t rows_odd = __builtin_amdgcn_ballot_w64(odd);
          rows_odd = (rows_odd | rows_odd >> 1) & 0x5555555555555555ull;
          while (rows_odd != 0) {
            const int r = __builtin_ctzll(rows_odd) / 2, at_e = r / 16 * 4 + r % 4, from_lane = r % 16 / 4 * 16 + cq;
            rows_odd &= rows_odd - 1;
            float pr[NR];
            bool sees[NR];
#pragma unroll
            for (int n = 0; n < NR; ++n) {
              float mine = 0.f;
#pragma unroll
              for (int e = 0; e < 8; ++e) mine = e == at_e ? x[n][e] : mine;
              pr[n] = __shfl(mine, from_lane);
              sees[n] = (__shfl(static_cast<int>(seen[n]), from_lane) >> at_e & 1) != 0;
            }
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int col = 16 * db + 4 * cg + e;
                float y;
                if constexpr (F8) {
                  const unsigned byte = vl[r * RB + (db ^ C::swz_v(r)) * 16 + 4 * cg + e];
                  y = __builtin_amdgcn_cvt_f32_fp8(byte, 0);
                } else {
                  y = static_cast<float>(*reinterpret_cast<const __bf16*>(vl + r * RB + ((col / 8) ^ C::swz_v(r)) * 16 + col % 8 * 2));
                }
#pragma unroll
                for (int n = 0; n < NR; ++n) o[n][db][e] += sees[n] ? pr[n] * y : 0.f;
              }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (ln < C::UNITS) *reinterpret_cast<u32x4*>(vl + r * RB + ln * 16) = u32x4{0u, 0u, 0u, 0u};
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          }
        }
        // ---- O^T += V^T P^T
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          bf16x8 vf;
          if constexpr (!F8) {
            const int r = 4 * g + (lq >> 2), un = 2 * db + ((lq & 3) >> 1);
            vf = lds_tr8(vl + r * RB + (un ^ C::swz_v(r)) * 16 + 8 * (lq & 1), vl + (r + 16) * RB + (un ^ C::swz_v(r + 16)) * 16 + 8 * (lq & 1));
          } else {
            const int r8 = lq >> 1, r = 4 * g + (r8 & 3) + (r8 >> 2) * 16;
            vf = widen(__builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2_ptr)(lds_void_ptr)(vl + r * RB + (db ^ C::swz_v(r)) * 16 + 8 * (lq & 1)))));
          }
#pragma unroll
          for (int n = 0; n < NR; ++n) o[n][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, hi[n], o[n][db], 0, 0, 0);
#pragma unroll
          for (int n = 0; n < NR; ++n) o[n][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, lo[n], o[n][db], 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the stage has been read
        fetch(t + NS, st, soon);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (what was fetched past the end lands in LDS too)
      if constexpr (decltype(careful)::value)
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          float times;
          m_rest[n] = rest_of_product(m_run[n], c, times);
          l_run[n] *= times; l_lo[n] *= times;
#pragma unroll
          for (int i = 0; i < NDB; ++i) o[n][i] *= times;
        }
    };
    pass(std::false_type{});
    {
      float z = 0.f;
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int i = 0; i < NDB; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) z = __builtin_fmaf(o[n][i][e], 0.f, z);
      bool again = z != 0.f;                                     // (0 times a number is 0)
#pragma unroll
      for (int n = 0; n < NR; ++n) again |= beyond_fma(m_run[n]);
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(again) != 0, 0)) pass(std::true_type{});
    }

    // ---- the wavefronts' sums are joined, 16 rows at a time
    float* const sums = reinterpret_cast<float*>(smem);
    float* const tops = sums + NW * 16 * C::ROW;                 // references, their rests, sums of weights
    constexpr int TPR = NW * 64 / 16, EL = D / TPR;              // threads to a row, and its values to each
    const int jr = thread / TPR, je = thread % TPR * EL;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      float l = l_run[n] + l_lo[n];
      l += __shfl_xor(l, 16);
      l += __shfl_xor(l, 32);
      __syncthreads();
#pragma unroll
      for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4*>(sums + (w * 16 + lq) * C::ROW + 16 * db + 4 * g) = o[n][db];
      if (g == 0) { tops[w * 16 + lq] = m_run[n]; tops[(NW + w) * 16 + lq] = m_rest[n]; tops[(2 * NW + w) * 16 + lq] = l; }
      __syncthreads();
      float top = kLeast, top_rest = 0.f, weight[NW], total = 0.f, acc[EL];
#pragma unroll
      for (int i = 0; i < NW; ++i) top = fmaxf(top, tops[i * 16 + jr]);
#pragma unroll
      for (int i = 0; i < NW; ++i) weight[i] = fast_exp2(tops[i * 16 + jr] - top);
      if (__builtin_expect(beyond_fma(top), 0)) {
        top = tops[jr]; top_rest = tops[NW * 16 + jr];
#pragma unroll
        for (int i = 1; i < NW; ++i) {
          const float m = tops[i * 16 + jr], rest = tops[(NW + i) * 16 + jr];
          const bool more = less(m, rest, top, top_rest) > 0.f;
          top = more ? m : top;
          top_rest = more ? rest : top_rest;
        }
#pragma unroll
        for (int i = 0; i < NW; ++i) weight[i] = fast_exp2(less(tops[i * 16 + jr], tops[(NW + i) * 16 + jr], top, top_rest));
      }
#pragma unroll
      for (int i = 0; i < NW; ++i) total += weight[i] * tops[(2 * NW + i) * 16 + jr];
#pragma unroll
      for (int e = 0; e < EL; ++e) acc[e] = 0.f;
#pragma unroll
      for (int i = 0; i < NW; ++i)
#pragma unroll
        for (int e = 0; e < EL; ++e) acc[e] += weight[i] * sums[(i * 16 + jr) * C::ROW + je + e];
      const float inv = total == 0.f ? 0.f : 1.f / total, lse2 = total == 0.f ? -__builtin_inff() : top + (top_rest + __builtin_amdgcn_logf(total));
#pragma unroll
      for (int e = 0; e < EL; ++e) acc[e] *= inv;
      const int at = 16 * n + jr, row = rt * BM + at;
      if (row < rows) {
        if (whole) {
          const int tok = divide(row, p.by_group);
          store_row<D, EL>(p, static_cast<int64_t>(s.r0 + tok) * p.Hq + head * p.G + (row - tok * p.G), je, acc, lse2);
        } else {
          float* const dst = part_of<BM, D>(p, worker, run.x0 > 0);
#pragma unroll
          for (int e = 0; e < EL; e += 4) *reinterpret_cast<f32x4*>(dst + at * D + je + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
          if (je == 0) { dst[BM * D + at] = top; dst[BM * D + BM + at] = total; dst[BM * D + 2 * BM + at] = top_rest; }
        }
      }
    }
    __syncthreads();
  }
  leave_split(p, worker, split);
}

// Beside its keys a row tile counts as 64 of them; 16 or more are split off one, and a run has at least 64.  18 calls, geometric mean: 64, 16, 64
// (tile, split, run) 38.4 us; 16, 16, 64 39.2 (64 sequences of e4m3 202 us for 198); 128, 32, 128 39.4; 192, 64, 256 41.3 (one token of 700: 12.1 for
// 9.7).  They are the four cases of perf/operators.py that come here; of its default heads (32 over 8 of 128, bf16 unless said) one token for 8 sequences of
// 300 keys, 1 of 4 000, 32 of 100 to 900 e4m3, 16 of 2 000 e4m3, 4 of 30 000 and 128 of 500 to 1 500; and the first 8 calls of attention with
// at most 32 rows that its draw() gives from random.Random(3).
template <int D, bool F8, int NR>
bool cut(PagedAttn& p) { return set_cut(p, 16 * NR, 256 * RowsCfg<D, F8, NR>::PER_CU, 64, 16, 64); }

template <int D, bool F8, int NR>
hipError_t launch_variant(PagedAttn p, hipStream_t stream) {
  using C = RowsCfg<D, F8, NR>;
  static_assert(C::PER_CU * (C::LDS + 4 * C::NW * C::LIST) <= 160 * 1024, "");
  if (!cut<D, F8, NR>(p)) return hipErrorInvalidValue;
  place_split(p, C::BM, D);
  const hipError_t e = TASP_LAUNCH((paged_rows_kernel<D, F8, NR>), dim3(static_cast<unsigned>(p.workers)), dim3(C::NW * 64), stream, p);
  return e != hipSuccess ? e : launch_paged_combine<D, C::BM>(p, stream);
}

template <int D, bool F8>
hipError_t launch_rows(const PagedAttn& p, int rows, hipStream_t stream) {
  return rows <= 16 ? launch_variant<D, F8, 1>(p, stream) : launch_variant<D, F8, 2>(p, stream);
}
template <int D, bool F8>
int64_t workspace_for(PagedAttn p, int rows) {
  if (rows <= 16) return cut<D, F8, 1>(p) ? workspace_of(p, 16, D) : 0;
  return cut<D, F8, 2>(p) ? workspace_of(p, 32, D) : 0;
}

}  // namespace

int64_t paged_rows_workspace(const PagedAttn& p, bool e4m3, int d, int rows) {
  if (d == 64) return e4m3 ? workspace_for<64, true>(p, rows) : workspace_for<64, false>(p, rows);
  return e4m3 ? workspace_for<128, true>(p, rows) : workspace_for<128, false>(p, rows);
}

hipError_t launch_paged_rows(const PagedAttn& p, bool e4m3, int d, int rows, hipStream_t stream) {
  if (d == 64) return e4m3 ? launch_rows<64, true>(p, rows, stream) : launch_rows<64, false>(p, rows, stream);
  return e4m3 ? launch_rows<128, true>(p, rows, stream) : launch_rows<128, false>(p, rows, stream);
}

}  // namespace tasp
