// Attention of a few new tokens over a paged cache: 16 (token, query head of the group) rows to a tile.
//
// S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_16x16x32_bf16, softmax in one pass (running maximum and sum).  A grouped head's K and V
// are read once for all 16 rows.  Every wavefront takes keys of its own, in stages of 32, through a part of LDS of its own that loads
// fill directly: no barrier inside the loop, and the loads run ahead of the products by the stages behind the first.
// What bounds it is HBM: per key and KV head 4 d bytes (e4m3: 2 d + 2) for 4 d 16 products.
//
// The work of a call (sequence after sequence, KV head after KV head, row tile after row tile, in key tiles) is cut into equal runs,
// one for a workgroup; where a run ends inside a row tile, partial results go to the workspace and paged_rows_combine adds them up,
// always in the same order.  The lengths are on the device, so every workgroup works out its own run.
//
// Rounding: P goes into the second product as two bf16 (its value and what rounding that left, 2^-17 of it), which costs a second
// matrix instruction that HBM hides; everything else is fp32.  e4m3 values are exact in bf16, their scales (powers of two) multiply the
// scores and the probabilities.
#include <hip/hip_runtime.h>

#include "internal.hpp"
#include "paged.hpp"
#include "paged_combine.hpp"
#include "pipeline.hpp"

namespace tasp {
namespace {

template <int D, bool F8>
struct RowsCfg {
  static constexpr int BM = 16, WK = 32;                 // rows of a tile; keys of a stage
  static constexpr int RB = D * (F8 ? 1 : 2);            // bytes of a row in the cache
  static constexpr int UNITS = RB / 16, RPL = 64 / UNITS, LOADS = WK / RPL;       // 16-byte units of it; rows to a wavefront's load; loads to a stage's K
  static constexpr int NW = 2;                           // wavefronts
  static constexpr int PER_CU = F8 ? (D == 128 ? 4 : 6) : (D == 128 ? 2 : 4);      // workgroups that a compute unit holds
  static constexpr int NS = 2;                           // stages in LDS
  static constexpr int BT = NW * WK;
  static constexpr int STAGE = 2 * WK * RB + (F8 ? 256 : 0), PER_STAGE = 2 * LOADS + (F8 ? 1 : 0);
  static constexpr int LIST = 256;                       // pages a wavefront looks up at once, one for every 16 keys
  static constexpr int ROW = D + 4;                      // floats of a row of sums while they are joined
  static constexpr int RING = NW * NS * STAGE, JOIN = NW * BM * ROW * 4 + NW * BM * 8, LDS = RING > JOIN ? RING : JOIN;
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

template <int D, bool F8>
__global__ __launch_bounds__((RowsCfg<D, F8>::NW * 64), (RowsCfg<D, F8>::NW * RowsCfg<D, F8>::PER_CU / 4)) void paged_rows_kernel(const PagedAttn p) {
  using C = RowsCfg<D, F8>;
  constexpr int NW = C::NW, NS = C::NS, BT = C::BT, BM = C::BM, NDB = C::NDB, RB = C::RB;
  __shared__ __attribute__((aligned(256))) unsigned char smem[C::LDS];
  __shared__ int pages[NW][C::LIST];
  const int thread = threadIdx.x, w = __builtin_amdgcn_readfirstlane(thread >> 6), lane = thread & 63;
  const int g = lane >> 4, lq = lane & 15;
  const float c = p.scale_log2e;
  unsigned char* const ring = smem + w * NS * C::STAGE;

  PagedRun<BM, BT, true> run;
  const int worker = xcd_contiguous(blockIdx.x, p.workers);
  PagedSplit split{0, 0, 0, 0, worker, {0, 0, 0}};
  if (!run.start(p, worker, lane)) {
    leave_split<BM, BT>(p, worker, split);
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
    const int rows = s.n * p.G, m = rt * BM + lq, mc = min(m, rows - 1), tok = divide(mc, p.by_group);
    const int tok0 = divide(rt * BM, p.by_group), tok1 = divide(min(rt * BM + BM, rows) - 1, p.by_group);
    PagedKeys keys = keys_of<BM, BT>(p, s, tok0, tok1);
    const int p0 = s.kv - s.n;
    const int see_to = min(p.causal ? p0 + tok : INT_MAX, keys.end - 1);         // the lane's row sees keys up to it,
    const int see_from = p.window > 0 ? p0 + tok - p.window + 1 : INT_MIN;       // from this one on or among the first
    const int all_to = min(p.causal ? p0 + tok0 : INT_MAX, keys.end - 1), all_from = p.window > 0 ? p0 + tok1 - p.window + 1 : INT_MIN;
    bf16x8 qf[D / 32];
    {
      const __bf16* const src = static_cast<const __bf16*>(p.q) + static_cast<int64_t>(s.r0 + tok) * p.q_stride + static_cast<int64_t>(head * p.G + mc - tok * p.G) * D;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) qf[j] = *reinterpret_cast<const bf16x8*>(src + (F8 ? 64 * (j / 2) + 16 * g + 8 * (j % 2) : 32 * j + 8 * g));
    }
    f32x4 o[NDB];
    float m_run, l_run, l_lo;

    // (what the loads and the loop go by is the same in all lanes, and said to be)
    const int t0 = scalar(key_tile_at(run.x0, run.cost, keys.n_tiles)), t1 = scalar(key_tile_at(run.x1, run.cost, keys.n_tiles));
    keys.n_first = scalar(keys.n_first);
    keys.from = scalar(keys.from);
    keys.end = scalar(keys.end);
    const int64_t head_bytes = (static_cast<int64_t>(head) << p.c.ps_log2) * RB;
    const unsigned char* const k_head = p.c.k + head_bytes;
    const unsigned char* const v_head = p.c.v + head_bytes;
    // ---- pages of the wavefront's keys, LIST / 2 tiles at a time
    int listed = t0;
    auto look_up = [&](int t) {
      listed = t;
#pragma unroll
      for (int i = 0; i < C::LIST / 64; ++i) {
        const int e = i * 64 + lane, u = t + e / 2;
        int page = -1;
        if (u < t1) {
          const int pos = keys.tile(u) * BT + w * C::WK + e % 2 * 16;
          if (pos < keys.end) page = page_of(p.c, b, pos);
        }
        pages[w][e] = page;
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
    // such values taken out of the product and added one by one.
    auto pass = [&](auto careful) {
#pragma unroll
      for (int i = 0; i < NDB; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      m_run = kNegBig; l_run = 0.f; l_lo = 0.f;
      float m_raise = kNegBig;
      if (t0 < t1) {
        look_up(t0);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) asm volatile("" : "+v"(qf[j]));          // (the compiler waits for them here, not in the loop)
        for (int i = 0; i < NS; ++i) fetch(t0 + i, i, listed_pages(t0 + i));
      }
      for (int t = t0, st = 0; t < t1; ++t, st = st + 1 == NS ? 0 : st + 1) {
        const i32x2v soon = listed_pages(t + NS);
        asm volatile("s_waitcnt vmcnt(%0)" : : "n"((NS - 1) * C::PER_STAGE) : "memory");
        const unsigned char* const kl = ring + st * C::STAGE;
        unsigned char* const vl = ring + st * C::STAGE + C::WK * RB;
        const int pos0 = keys.tile(t) * BT + w * C::WK;
        const unsigned has = paged >> (2 * (NS - 1)) & 3;
        // ---- scores: those of keys 4 g .. 4 g + 3 and 16 + 4 g .. of the lane's row
        float x[8], vs[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          f32x4 sc = f32x4{0.f, 0.f, 0.f, 0.f};
          const int r = 16 * i + lq;
          if constexpr (!F8) {
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
              sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8*>(kl + r * RB + ((4 * j + g) ^ C::swz_k(r)) * 16), qf[j], sc, 0, 0, 0);
          } else {
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
              const u32x4 k16 = *reinterpret_cast<const u32x4*>(kl + r * RB + ((4 * j + g) ^ C::swz_k(r)) * 16);
              sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(u32x2{k16[0], k16[1]}), qf[2 * j], sc, 0, 0, 0);
              sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(u32x2{k16[2], k16[3]}), qf[2 * j + 1], sc, 0, 0, 0);
            }
          }
          if constexpr (F8) {
            const unsigned kw = *reinterpret_cast<const unsigned*>(kl + 2 * C::WK * RB + 16 * i + 4 * g);
            const unsigned vw = *reinterpret_cast<const unsigned*>(kl + 2 * C::WK * RB + 32 + 16 * i + 4 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              x[4 * i + e] = sc[e] * scale_value(kw >> 8 * e & 255);
              vs[4 * i + e] = scale_value(vw >> 8 * e & 255);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * i + e] = sc[e];
          }
        }
        unsigned seen = 0xff;
        if (!(has == 3 && pos0 + C::WK - 1 <= all_to && (pos0 >= all_from || pos0 + C::WK <= p.sinks))) {
          seen = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int pos = pos0 + 16 * (e / 4) + 4 * g + e % 4;
            const bool ok = (has >> (e / 4) & 1) != 0 && pos <= see_to && (pos >= see_from || pos < p.sinks);
            seen |= ok ? 1u << e : 0u;
            x[e] = ok ? x[e] : -__builtin_inff();
            if constexpr (F8) vs[e] = ok ? vs[e] : 0.f;          // (a scale behind the end may be anything)
          }
        }
        // ---- softmax: the running maximum is only raised when it grew by more than 2^8
        const float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        if (__builtin_amdgcn_ballot_w64(mx * c > m_raise) != 0) {
          float m_new = fmaxf(mx, __shfl_xor(mx, 16));
          m_new = fmaxf(m_run, fmaxf(m_new, __shfl_xor(m_new, 32)) * c);
          const float alpha = fast_exp2(m_run - m_new);
          m_run = m_new;
          m_raise = m_new + kRescaleGap;
          l_run *= alpha; l_lo *= alpha;
#pragma unroll
          for (int i = 0; i < NDB; ++i) o[i] *= alpha;
        }
        bf16x8 hi, lo;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] = fast_exp2(__builtin_fmaf(x[e], c, -m_run));
          sum += x[e];
          if constexpr (F8) x[e] *= vs[e];
          hi[e] = static_cast<__bf16>(x[e]);
          lo[e] = static_cast<__bf16>(x[e] - static_cast<float>(hi[e]));
        }
        // in two levels, so that a few large terms do not swallow many small ones
        l_lo += sum;
        if ((t & 63) == 63) { l_run += l_lo; l_lo = 0.f; }

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
            float pr = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) pr = e == at_e ? x[e] : pr;
            pr = __shfl(pr, from_lane);
            const bool sees = (__shfl(static_cast<int>(seen), from_lane) >> at_e & 1) != 0;
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
                o[db][e] += sees ? pr * y : 0.f;
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
          o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, hi, o[db], 0, 0, 0);
          o[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, lo, o[db], 0, 0, 0);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the stage has been read
        fetch(t + NS, st, soon);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");           // (what was fetched past the end lands in LDS too)
    };
    pass(std::false_type{});
    {
      float z = 0.f;
#pragma unroll
      for (int i = 0; i < NDB; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) z = __builtin_fmaf(o[i][e], 0.f, z);
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(z != 0.f) != 0, 0)) pass(std::true_type{});       // (0 times a number is 0)
    }

    // ---- the wavefronts' sums are joined
    float l = l_run + l_lo;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    float* const sums = reinterpret_cast<float*>(smem);
    float* const tops = sums + NW * BM * C::ROW;
    __syncthreads();
#pragma unroll
    for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4*>(sums + (w * BM + lq) * C::ROW + 16 * db + 4 * g) = o[db];
    if (g == 0) { tops[w * BM + lq] = m_run; tops[(NW + w) * BM + lq] = l; }
    __syncthreads();
    constexpr int TPR = NW * 64 / BM, EL = D / TPR;              // threads to a row, and its values to each
    const int jr = thread / TPR, je = thread % TPR * EL;
    float top = kNegBig, weight[NW], total = 0.f, acc[EL];
#pragma unroll
    for (int i = 0; i < NW; ++i) top = fmaxf(top, tops[i * BM + jr]);
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      weight[i] = fast_exp2(tops[i * BM + jr] - top);
      total += weight[i] * tops[(NW + i) * BM + jr];
    }
#pragma unroll
    for (int e = 0; e < EL; ++e) acc[e] = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i)
#pragma unroll
      for (int e = 0; e < EL; ++e) acc[e] += weight[i] * sums[(i * BM + jr) * C::ROW + je + e];
    const float inv = total == 0.f ? 0.f : 1.f / total, lse2 = total == 0.f ? -__builtin_inff() : top + __builtin_amdgcn_logf(total);
#pragma unroll
    for (int e = 0; e < EL; ++e) acc[e] *= inv;
    if (rt * BM + jr < rows) {
      if (whole) {
        const int jt = divide(rt * BM + jr, p.by_group);
        store_row<D, EL>(p, static_cast<int64_t>(s.r0 + jt) * p.Hq + head * p.G + (rt * BM + jr - jt * p.G), je, acc, lse2);
      } else {
        float* const dst = part_of<BM, D>(p, worker, run.x0 > 0);
#pragma unroll
        for (int e = 0; e < EL; e += 4) *reinterpret_cast<f32x4*>(dst + jr * D + je + e) = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
        if (je == 0) dst[BM * D + jr] = lse2;
      }
    }
    __syncthreads();
  }
  leave_split<BM, BT>(p, worker, split);
}

constexpr int kMostWorkers = 256 * 8;

template <int D, bool F8>
hipError_t launch_variant(PagedAttn p, hipStream_t stream) {
  using C = RowsCfg<D, F8>;
  static_assert(256 * C::PER_CU <= kMostWorkers && C::PER_CU * (C::LDS + 4 * C::NW * C::LIST) <= 160 * 1024, "");
  set_workers(p, 256 * C::PER_CU, C::BM, D);
  const hipError_t e = TASP_LAUNCH((paged_rows_kernel<D, F8>), dim3(static_cast<unsigned>(p.workers)), dim3(C::NW * 64), stream, p);
  return e != hipSuccess ? e : launch_paged_combine<D, C::BM>(p, stream);
}

}  // namespace

int64_t paged_rows_workspace(int d) { return workspace_of(kMostWorkers, 16, d); }

hipError_t launch_paged_rows(PagedAttn p, bool e4m3, int d, hipStream_t stream) {
  p.tile_cost = kParts / 4;
  p.snap = kParts / 4;
  p.least_share = kParts;
  if (d == 64) return e4m3 ? launch_variant<64, true>(p, stream) : launch_variant<64, false>(p, stream);
  return e4m3 ? launch_variant<128, true>(p, stream) : launch_variant<128, false>(p, stream);
}

}  // namespace tasp
