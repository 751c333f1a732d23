// Attention of many new tokens over a paged cache: 128 (token, query head of the group) rows to a workgroup.
//
// S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_32x32x16_bf16, 32 rows to a wavefront, keys in tiles of 64 that all wavefronts share.  The
// loop is that of the joined steps (attn_run.hip), pipelined by hand: the scores of a tile beside the probabilities of the one before.  Only
// where the keys come from differs: a lane of a register holds the page of 16 keys, sixteen tiles ahead at a time, and a load's
// descriptor is made of it by scalar instructions (base, and how many bytes of the 16 rows count: what lies behind, and pages that
// do not exist, come as zeros).  e4m3 rows are loaded into registers a tile ahead, widened (times their scale, exactly) and written to LDS as bf16.
//
// What bounds it: vector issue, as in attn_run.hip.  2 048 new tokens of 65 536, 32 and 8 heads of 128: 1.93 ms, 1.12 PFLOP/s (a large matrix
// product reaches 1.375 on this card).  Few rows of long e4m3 sequences are bound by latency (48 rows, 229 us for 109 of reading).
//
// Rounding: P goes into the second product as one bf16, off by at most 2^-8 of its value, as in the kernels of dense K and V; the largest
// probability of a tile is taken as it was rounded in the sum that the output is divided by.  A second bf16 for what rounding left, as in the kernel for few rows,
// would be half as many matrix instructions again, beside a pipe that is 60 % busy, and as many vector instructions to make it, which are the bound.
//
// The work of a call is cut into equal runs, one for a workgroup (PagedRun), as in attn_paged.hip.
#include <hip/hip_runtime.h>

#include <climits>

#include "internal.hpp"
#include "paged.hpp"
#include "paged_combine.hpp"
#include "pipeline.hpp"

namespace tasp {
namespace {

template <int D, bool F8>
struct PTileCfg {
  static constexpr int BM = 128, NW = 4, NTHREADS = 64 * NW, BT = 64;
  static constexpr int RB = 2 * D, UNITS = RB / 16, RPL = 16 / UNITS;                  // a row in LDS: bytes, 16-byte units; rows to a 256-byte bank line
  static constexpr int CB = F8 ? D : RB, CUNITS = CB / 16;                             // a row in the cache
  static constexpr int RPW = 64 / CUNITS, RPP = NW * RPW, PASSES = BT / RPP;           // rows to a wavefront's load, to a pass of all; loads to a tile
  static constexpr int TILE_BYTES = BT * RB;
  static constexpr int NDB = D / 32, NJ = D / 16;
  // the 16 keys that pass i of a wavefront is in, and its first row there
  __device__ static int block_of(int w, int i) { return (i * RPP + w * RPW) / 16; }
  __device__ static int row_of(int w) { return w * RPW % 16; }
  __device__ static int swz_k(int r, int u) { return u ^ ((r / RPL) % UNITS); }
  __device__ static int swz_v(int r, int u) { return u ^ (4 * ((r / RPL) % (UNITS / 4))); }
};

__device__ __forceinline__ u32x4 widen8(unsigned a, unsigned b, float scale) {
  union { bf16x2 p[4]; u32x4 v; } r;
  r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false);
  r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
  r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
  r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
  return r.v;
}

// Four e4m3 values times 0: NaN stays, the others are 0.
__device__ __forceinline__ unsigned nan_bytes(unsigned w) { return (((w & 0x7f7f7f7fu) + 0x01010101u) >> 7 & 0x01010101u) * 0x7fu; }

// One direct global->LDS load of 16 bytes per lane, as global_to_lds_16 with the fence, to `lds` + TO.
template <int TO>
__device__ __forceinline__ void lds_from(const unsigned char* base, unsigned off, unsigned lds) {
  asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base), "n"(TO) : "memory", "scc");
}

__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <int D, bool F8>
__global__ __launch_bounds__((PTileCfg<D, F8>::NTHREADS), (D == 64 && !F8 ? 3 : 2)) void paged_tile_kernel(const PagedAttn p) {
  using C = PTileCfg<D, F8>;
  constexpr int BM = C::BM, NW = C::NW, BT = C::BT, NDB = C::NDB, NJ = C::NJ, NL = C::PASSES;
  __shared__ __attribute__((aligned(256))) unsigned char smem[4 * C::TILE_BYTES];      // two K tiles, two V tiles
  __shared__ int odd_rows[BT];
  __shared__ int odd_waves[NW];

  const int thread = threadIdx.x, wave_u = __builtin_amdgcn_readfirstlane(thread >> 6);
  const int lane = thread & 63, h = lane >> 5, lq = lane & 31;
  const float c = p.scale_log2e;
  PagedRun<BM, false> run;
  const int worker = xcd_contiguous(blockIdx.x, p.workers);
  PagedSplit split{0, 0, 0, 0, worker, {0, 0, 0}};
  if (!run.start(p, worker, lane)) {
    leave_split(p, worker, split);
    return;
  }

  const unsigned page_rows = static_cast<unsigned>(p.c.Hkv) << p.c.ps_log2;          // (all pages have fewer than 2^32, the host sees to it)
  const int ps_mask = (1 << p.c.ps_log2) - 1;
  const unsigned first_row = static_cast<unsigned>(C::row_of(wave_u) * C::CB);
  const unsigned lane_row = static_cast<unsigned>(lane / C::CUNITS);
  // bf16: the lane's place in a load, so that 16-byte units land where their swizzle wants them (the same in every pass)
  const int fr = C::RPW * wave_u + static_cast<int>(lane_row), fu = lane % C::CUNITS;
  const unsigned k_lane = lane_row * C::CB + (F8 ? fu : C::swz_k(fr, fu)) * 16, v_lane = lane_row * C::CB + (F8 ? fu : C::swz_v(fr, fu)) * 16;
  const unsigned smem_lds = static_cast<unsigned>(reinterpret_cast<size_t>((lds_void_ptr)smem));
  const unsigned k_adr = lq * C::RB + C::swz_k(lq, h) * 16;          // unit 2 j + h sits at k_adr ^ 32 j
  const int vga = lane >> 4, vjj = lane & 15, vrow = 4 * (vga >> 1) + (vjj >> 2);

  // Workers of an XCD mostly have neighbouring row tiles of a KV head, whose keys they find in its L2 if they walk them together: a run starts
  // with the row tiles that it has from their first key on, and a piece that starts inside one comes last.
  bool piece = false, last_piece = false;
  for (bool more = run.next(p, lane);;) {
    if (!more) {
      if (!piece || last_piece) break;
      last_piece = true;
      run.start(p, worker, lane);
      run.next(p, lane);
    } else if (run.x0 > 0 && !piece) {
      piece = true;
      run.step();
      more = run.next(p, lane);
      continue;
    }
    const int head = scalar(run.head), rt = scalar(run.rt), rows = run.s.n * p.G, left = rows - rt * BM;
    const bool whole = run.whole();
    if (run.x0 == 0 && !whole) split = PagedSplit{run.s.r0, rows, head, rt, run.last_worker(p, worker), {0, 0, 0}};
    // The strip of 32 rows that a wavefront takes moves with the row tile: tiles with few rows leave strips without work.
    const int strip = (wave_u + rt) % NW;
    const int m = rt * BM + strip * 32 + lq, mc = min(m, rows - 1), tok = divide(mc, p.by_group);
    const int tok0 = divide(rt * BM, p.by_group), tok1 = divide(min(rt * BM + BM, rows) - 1, p.by_group);
    PagedKeys keys = keys_of<BM, BT>(p, run.s, tok0, tok1);
    const int p0 = run.s.kv - run.s.n;
    const int see_to = min(p.causal ? p0 + tok : INT_MAX, keys.end - 1), see_from = p.window > 0 ? window_start(p0 + tok, p.window) : INT_MIN;
    const int all_to = scalar(min(p.causal ? p0 + tok0 : INT_MAX, keys.end - 1)), all_from = scalar(p.window > 0 ? window_start(p0 + tok1, p.window) : INT_MIN);
    // (what the loader and the loop go by is the same in all lanes, and said to be)
    const int t0 = scalar(key_tile_at(run.x0, run.cost, keys.n_tiles)), n_tiles = scalar(key_tile_at(run.x1, run.cost, keys.n_tiles)) - t0;
    keys.n_first = scalar(keys.n_first);
    keys.from = scalar(keys.from);
    keys.end = scalar(keys.end);

    // ---- loader.  Tiles are counted from t0.  For the 16 tiles from the last multiple of 8 on, one lane to 16 keys: list, the row of the
    // pages where they start; paged, whether they have a page; easy, whether in addition every row sees all of them.
    const uint64_t head_rows = static_cast<uint64_t>(head) << p.c.ps_log2;
    const unsigned char* const k_base = p.c.k + head_rows * C::CB + first_row;
    const unsigned char* const v_base = p.c.v + head_rows * C::CB + first_row;
    const int32_t* const table = p.c.table + static_cast<int64_t>(run.b) * p.c.max_pages;
    auto look_up = [&](int t) __attribute__((always_inline)) {
      const int u = t + lane / 4, pos = keys.tile(t0 + u) * BT + lane % 4 * 16;
      return u < n_tiles && pos < keys.end ? table[pos >> p.c.ps_log2] : -1;
    };
    unsigned list;
    uint64_t paged, easy;
    auto take_list = [&](int t, int page) __attribute__((always_inline)) {
      const int pos = keys.tile(t0 + t + lane / 4) * BT + lane % 4 * 16;
      const bool has = page >= 0 && page < p.c.n_pages;
      list = has ? static_cast<unsigned>(page) * page_rows + (pos & ps_mask) : 0u;
      paged = __builtin_amdgcn_ballot_w64(has);
      easy = __builtin_amdgcn_ballot_w64(has && pos + 15 <= all_to && (pos >= all_from || pos + 16 <= p.sinks));
    };
    take_list(0, look_up(0));
    int next = look_up(8);
    auto turn_list = [&](int t) __attribute__((always_inline)) {
      take_list(t, next);
      next = look_up(t + 8);
    };
    auto is_easy = [&](int t, int listed) __attribute__((always_inline)) { return (static_cast<unsigned>(easy >> ((t - listed) * 4)) & 15) == 15; };
    // Where the loads of a tile find their keys: K's are found first, V's of the same tile lie as far from v_base a body later.  An easy tile
    // needs no more than that; otherwise each 16 keys have a descriptor, with as many records as count.
    unsigned at[NL];
    bool there = false;
    auto find = [&](int t, int listed) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NL; ++i) at[i] = __builtin_amdgcn_readlane(list, (t - listed) * 4 + C::block_of(wave_u, i));
      there = is_easy(t, listed);
    };
    auto records_of = [&](int t, int listed, int i, uint64_t& row) __attribute__((always_inline)) {
      const int place = (t - listed) * 4 + C::block_of(wave_u, i), pos = keys.tile(t0 + t) * BT + 16 * C::block_of(wave_u, i);
      row = __builtin_amdgcn_readlane(list, place);
      const int n = larger(0, scalar(lesser(16, keys.end - pos)));        // (both bounds at once would be a vector instruction)
      return (paged >> place & 1) != 0 ? static_cast<unsigned>(n) : 0u;
    };
    // bf16: straight to LDS, of which the wavefront has the 1 KiB at `mine` of every pass.  (`t` and `listed` are looked at only for tiles that
    // are not easy.)
    const unsigned mine = smem_lds + wave_u * 1024;
    auto fetch = [&](auto vv, auto ss, bool easy_tile, int t, int listed) __attribute__((always_inline)) {
      constexpr bool V = decltype(vv)::value;
      constexpr int TO = (V ? 2 * C::TILE_BYTES : 0) + decltype(ss)::value * C::TILE_BYTES;
      if (__builtin_expect(easy_tile, 1)) {
        static_for<NL>([&](auto i) __attribute__((always_inline)) {
          lds_from<TO + decltype(i)::value * C::NTHREADS * 16>((V ? v_base : k_base) + static_cast<uint64_t>(at[decltype(i)::value]) * C::CB, V ? v_lane : k_lane, mine);
        });
      } else {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          uint64_t row;
          const unsigned records = records_of(t, listed, i, row) * C::CB;
          buffer_to_lds_16<true>(raw_buffer((V ? v_base : k_base) - first_row + row * C::CB, records), lesser(first_row, records), V ? v_lane : k_lane,
                                 smem + TO + wave_u * 1024 + i * C::NTHREADS * 16);
        }
      }
    };
    // e4m3: to registers, and from there, as bf16, to LDS
    u32x4 held[2][F8 ? NL : 1];
    unsigned held_scale[2][F8 ? NL : 1];
    auto load = [&](auto vv, bool easy_tile, int t, int listed) __attribute__((always_inline)) {
      constexpr bool V = decltype(vv)::value;
      const unsigned char* const scales = (V ? p.c.v_scale : p.c.k_scale) + head_rows;
      if (__builtin_expect(easy_tile, 1)) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          held[V][i] = *reinterpret_cast<const u32x4*>((V ? v_base : k_base) + static_cast<uint64_t>(at[i]) * C::CB + k_lane);
          held_scale[V][i] = (scales + at[i] + C::row_of(wave_u))[lane_row];
        }
      } else {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          uint64_t row;
          const unsigned n = records_of(t, listed, i, row);
          const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>((V ? v_base : k_base) - first_row + row * C::CB), 0, static_cast<int>(n * C::CB), 0x00020000);
          held[V][i] = __builtin_amdgcn_raw_buffer_load_b128(rs, static_cast<int>(first_row + k_lane), 0, 0);
          const auto ss = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(scales + row), 0, static_cast<int>(n), 0x00020000);
          held_scale[V][i] = __builtin_amdgcn_raw_buffer_load_b8(ss, static_cast<int>(C::row_of(wave_u) + lane_row), 0, 0);
        }
      }
    };
    auto put = [&](auto vv, int st) __attribute__((always_inline)) {
      constexpr bool V = decltype(vv)::value;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const float scale = scale_value(held_scale[V][i]);
        // (the conversion takes exponent 0 for 2^-127: values times 0 are made here.  A window of 2 048 at d = 64: 107 us, 105 without the test; values
        // masked without a branch 106, and 230 for 229 us of 48 rows at d = 128, where NaN would be lost; mending LDS afterwards 106 and 235.)
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(held_scale[V][i] == 0) != 0, 0))
#pragma unroll
          for (int e = 0; e < 4; ++e) held[V][i][e] = held_scale[V][i] == 0 ? nan_bytes(held[V][i][e]) : held[V][i][e];
        const int r = i * C::RPP + fr;
        unsigned char* const row = smem + (V ? 2 * C::TILE_BYTES : 0) + st * C::TILE_BYTES + r * C::RB;
        const u32x4 x = held[V][i];
        *reinterpret_cast<u32x4*>(row + (V ? C::swz_v(r, 2 * fu) : C::swz_k(r, 2 * fu)) * 16) = widen8(x[0], x[1], scale);
        *reinterpret_cast<u32x4*>(row + (V ? C::swz_v(r, 2 * fu + 1) : C::swz_k(r, 2 * fu + 1)) * 16) = widen8(x[2], x[3], scale);
      }
    };
    constexpr std::false_type K{};
    constexpr std::true_type V{};
    constexpr std::integral_constant<int, 0> stage0{};
    constexpr std::integral_constant<int, 1> stage1{};

    u32x4 qf[NJ];
    {
      const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const __bf16*>(p.q) + static_cast<int64_t>(run.s.r0 + tok) * p.q_stride + static_cast<int64_t>(head * p.G + mc - tok * p.G) * D) + h;
#pragma unroll
      for (int j = 0; j < NJ; ++j) qf[j] = src[2 * j];
    }
    // K of tiles 0 and 1, V of tile 0
    if constexpr (F8) {
      find(0, 0); load(K, there, 0, 0); load(V, there, 0, 0); put(K, 0); put(V, 0);
      find(1, 0); load(K, there, 1, 0); put(K, 1);
      load(V, there, 1, 0);                        // V of tile 1, K of tile 2: written by body 0
      find(2, 0); load(K, there, 2, 0);
    } else {
      find(0, 0); fetch(K, stage0, there, 0, 0); fetch(V, stage0, there, 0, 0);
      find(1, 0); fetch(K, stage1, there, 1, 0);
    }
    unsigned ka[NJ], va[NDB];
#pragma unroll
    for (int j = 0; j < NJ; ++j) ka[j] = smem_lds + (k_adr ^ (32 * j));
#pragma unroll
    for (int db = 0; db < NDB; ++db) va[db] = smem_lds + vrow * C::RB + C::swz_v(vrow, 4 * db + 2 * (vga & 1) + ((vjj & 3) >> 1)) * 16 + 8 * (vjj & 1);
    f32x16 o[NDB];
#pragma unroll
    for (int db = 0; db < NDB; ++db) o[db] = zero16();
    // running max (exp2 domain), this lane's sum in two levels (up to 64 tiles, everything before) and what rounding added to the largest
    // probabilities: as in the kernels of dense K and V
    float m_run = kLeast, m_raise = kLeast, l_run = 0.f, l_lo = 0.f, r_fix = 0.f, mx = kLeast;

    if constexpr (!F8) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int j = 0; j < NJ; ++j) asm volatile("" : "+v"(qf[j]));
    __syncthreads();
    // What body t brings, V(t + 1) and K(t + 2): they go where body t - 1 has read last, and everybody has passed its barrier.
    auto bring_v = [&](int t, auto ss) __attribute__((always_inline)) {
      if constexpr (F8) { put(V, decltype(ss)::value); load(V, there, t + 2, t & ~7); } else fetch(V, ss, there, t + 1, t & ~7);
    };
    auto bring_k = [&](int t, auto ss) __attribute__((always_inline)) {
      if constexpr (F8) { put(K, decltype(ss)::value); find(t + 3, t & ~7); load(K, there, t + 3, t & ~7); }
      else { find(t + 2, t & ~7); fetch(K, ss, there, t + 2, t & ~7); }
    };
    auto brought = [&]() __attribute__((always_inline)) {
      if constexpr (!F8) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
    };
    constexpr int NF = 2 * NJ, NV = 4 * NDB, PD = 4;
    f32x16 Sa[2], Sb[2];
    // The operand fragments of a body as one stream, read PD ahead: NF of K of the next tile, then NV of V^T of this one (of two reads
    // each).  One wait serves an even fragment and the odd one behind it.
    u32x4 fk[PD];
    u32x2 fl[PD], fh[PD];
    auto read = [&](auto ff, auto sk, auto sv) __attribute__((always_inline)) {
      constexpr int F = decltype(ff)::value;
      if constexpr (F < NF) {
        lds_read_b128<F % 2 * 32 * C::RB + decltype(sk)::value * C::TILE_BYTES>(fk[F % PD], ka[F / 2]);
      } else if constexpr (F < NF + NV) {
        constexpr int FV = F - NF, AT = (2 + decltype(sv)::value) * C::TILE_BYTES + FV / NDB * 16 * C::RB;
        lds_read_tr_b64<AT>(fl[F % PD], va[FV % NDB]);
        lds_read_tr_b64<AT + 8 * C::RB>(fh[F % PD], va[FV % NDB]);
      }
    };
    // LDS instructions younger than those of fragments f and f + 1 when f is needed (`end`: fragments of the stream)
    auto younger = [](int f, int end) constexpr {
      if (f % 2 != 0) return -1;
      int n = 0;
      for (int r = f + 2; r < f + PD && r < end; ++r) n += r < NF ? 1 : 2;
      return n;
    };
    auto v_fragment = [&](auto ff) __attribute__((always_inline)) { constexpr int F = decltype(ff)::value % PD; return u32x4{fl[F][0], fl[F][1], fh[F][0], fh[F][1]}; };
    static_assert(NF % PD == 0 && NF % 2 == 0 && NV % 2 == 0 && PD % 2 == 0 && 4 * C::TILE_BYTES <= 65536, "");
    // hide(kb, i) for every score of a tile that its row does not see
    auto for_hidden = [&](int t, int listed, auto hide) __attribute__((always_inline)) {
      if (__builtin_expect(is_easy(t, listed), 1)) return;
      const unsigned has = static_cast<unsigned>(paged >> ((t - listed) * 4)) & 15;
      const int at0 = keys.tile(t0 + t) * BT + 4 * h;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int pos = at0 + 32 * kb + 8 * (i / 4) + i % 4;
          if (!((has >> (2 * kb + i / 8) & 1) != 0 && pos <= see_to && (pos >= see_from || pos < p.sinks))) hide(kb, i);
        }
    };
    auto mask = [&](int t, int listed, f32x16 (&S)[2]) __attribute__((always_inline)) {
      for_hidden(t, listed, [&](int kb, int i) __attribute__((always_inline)) { S[kb][i] = -__builtin_inff(); });
    };
    auto max_step = [&](auto ii, f32x16 (&S)[2]) __attribute__((always_inline)) {      // scores 2 I, 2 I + 1 of the 32 a lane holds
      constexpr int I = decltype(ii)::value;
      const float a = S[I / 8][2 * I % 16], b = S[I / 8][2 * I % 16 + 1];
      mx = I == 0 ? fmaxf(a, b) : fmaxf(fmaxf(mx, a), b);
    };
    u32x4 pf[4];
    float late[2], sum[4];
    auto exp_one = [&](auto ee, f32x16 (&S)[2]) __attribute__((always_inline)) {
      constexpr int E = decltype(ee)::value;
      const float x = fast_exp2(__builtin_fmaf(S[E / 16][E % 16], c, -m_run));
      sum[E % 4] = E < 4 ? x : sum[E % 4] + x;
      asm volatile("" : "+v"(sum[E % 4]));           // (here, not in a later block)
      late[E % 2] = x;
      if constexpr (E % 2 == 1) {
        const bf16x2 pk = {static_cast<__bf16>(late[0]), static_cast<__bf16>(late[1])};
        unsigned u = __builtin_bit_cast(unsigned, pk);
        asm volatile("" : "+v"(u));
        pf[E / 8][E % 8 / 2] = u;
      }
    };
    auto exps = [&](auto lo, auto hi, f32x16 (&S)[2]) __attribute__((always_inline)) {
      constexpr int LO = decltype(lo)::value;
      static_for<decltype(hi)::value - LO>([&](auto i) __attribute__((always_inline)) { exp_one(std::integral_constant<int, LO + decltype(i)::value>{}, S); });
    };
    // a tile's probabilities are summed for themselves and then added to the sum, so that this is rounded once a tile
    auto add_up = [&]() __attribute__((always_inline)) {
      l_lo += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      asm volatile("" : "+v"(l_lo));
    };
    // the output can be read by vector instructions from here on
    auto fence_o = [&]() __attribute__((always_inline)) {
      if constexpr (NDB == 2) asm volatile("s_nop 15\n\ts_nop 3" : "+v"(o[0]), "+v"(o[1]));
      else asm volatile("s_nop 15\n\ts_nop 3" : "+v"(o[0]), "+v"(o[1]), "+v"(o[NDB - 2]), "+v"(o[NDB - 1]));
    };
    // Before the probabilities of a tile whose maxima are in mx: raises the running max where it grew by more than the gap (a lane
    // tests the scores it holds; a row has grown iff one of its two lanes has), and takes down what rounding adds to the largest of them.
    auto raise = [&]() __attribute__((always_inline)) {
      if (__builtin_amdgcn_ballot_w64(mx * c > m_raise) != 0) {
        const float m_new = fmaxf(m_run, max_of_halves(mx) * c);     // both halves of a row agree
        const float alpha = fast_exp2(m_run - m_new);
        m_run = m_new;
        m_raise = m_new + kRescaleGap;
        fence_o();
        l_run *= alpha; l_lo *= alpha; r_fix *= alpha;
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          o[db] *= alpha;
          asm volatile("s_nop 1" : "+v"(o[db]));
        }
      }
      const float p_top = fast_exp2(__builtin_fmaf(mx, c, -m_run));
      r_fix += static_cast<float>(static_cast<__bf16>(p_top)) - p_top;
    };
    constexpr int PRE = 2, EK = 20, VE = 3 * NV / 4, VS = NV / 4;
    // Tile t (stage t % 2): scores of tile t + 1 beside the first probabilities of S, then the second product beside the others and
    // the maxima of S_next.
    auto body = [&](auto ss, int t, f32x16 (&S)[2], f32x16 (&S_next)[2]) __attribute__((always_inline)) {
      constexpr int ST = decltype(ss)::value;
      constexpr std::integral_constant<int, ST ^ 1> sk{};
      static_for<PD>([&](auto f) __attribute__((always_inline)) { read(f, sk, ss); });
      __builtin_amdgcn_sched_barrier(0);
      raise();
      exps(std::integral_constant<int, 0>{}, std::integral_constant<int, PRE>{}, S);
      __builtin_amdgcn_sched_barrier(0);
      static_for<NF>([&](auto ff) __attribute__((always_inline)) {
        constexpr int F = decltype(ff)::value, ks = F / 2, kb = F % 2;
        if constexpr (ks == 0) mfma_s_first<false, younger(F, NF + NV)>(S_next[kb], fk[F % PD], qf[ks]);
        else mfma_s<false, younger(F, NF + NV)>(S_next[kb], fk[F % PD], qf[ks]);
        read(std::integral_constant<int, F + PD>{}, sk, ss);
        exps(std::integral_constant<int, PRE + (EK - PRE) * F / NF>{}, std::integral_constant<int, PRE + (EK - PRE) * (F + 1) / NF>{}, S);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (F == 1) bring_v(t, sk);
        if constexpr (F == NF / 2 + 1) bring_k(t, ss);
        __builtin_amdgcn_sched_barrier(0);
      });
      static_for<NV>([&](auto ff) __attribute__((always_inline)) {
        constexpr int F = decltype(ff)::value, gg = F / NDB, db = F % NDB;
        if constexpr (F == VS) { fence_s(S_next[0], S_next[1]); mask(t + 1, t & ~7, S_next); }
        if constexpr (db == 0) fence_p(pf[gg]);
        mfma_s<false, younger(NF + F, NF + NV)>(o[db], v_fragment(std::integral_constant<int, NF + F>{}), pf[gg]);
        read(std::integral_constant<int, NF + F + PD>{}, sk, ss);
        if constexpr (F < VE) exps(std::integral_constant<int, EK + (32 - EK) * F / VE>{}, std::integral_constant<int, EK + (32 - EK) * (F + 1) / VE>{}, S);
        if constexpr (F == VE) add_up();
        if constexpr (F >= VS) {
          constexpr int lo = 16 * (F - VS) / (NV - VS), hi = 16 * (F + 1 - VS) / (NV - VS);
          static_for<hi - lo>([&](auto i) __attribute__((always_inline)) { max_step(std::integral_constant<int, lo + decltype(i)::value>{}, S_next); });
        }
        __builtin_amdgcn_sched_barrier(0);
      });
      brought();
    };
    // The last tile.
    auto tail = [&](auto ss, f32x16 (&S)[2]) __attribute__((always_inline)) {
      static_for<PD>([&](auto f) __attribute__((always_inline)) { read(std::integral_constant<int, NF + decltype(f)::value>{}, ss, ss); });
      __builtin_amdgcn_sched_barrier(0);
      raise();
      exps(std::integral_constant<int, 0>{}, std::integral_constant<int, 8>{}, S);
      __builtin_amdgcn_sched_barrier(0);
      static_for<NV>([&](auto ff) __attribute__((always_inline)) {
        constexpr int F = decltype(ff)::value, gg = F / NDB, db = F % NDB;
        if constexpr (db == 0) fence_p(pf[gg]);
        mfma_s<false, younger(NF + F, NF + NV)>(o[db], v_fragment(std::integral_constant<int, NF + F>{}), pf[gg]);
        read(std::integral_constant<int, NF + F + PD>{}, ss, ss);
        if constexpr (gg < 3) exps(std::integral_constant<int, 8 + 8 * F / NDB>{}, std::integral_constant<int, 8 + 8 * (F + 1) / NDB>{}, S);
        __builtin_amdgcn_sched_barrier(0);
      });
      add_up();
      fence_o();               // (here: the compiler may copy registers where the ways join)
    };
    const bool idle = strip * 32 >= left;
    if (idle) {                        // no rows: the loads only, with the barriers of the others
      if (n_tiles > 1) __syncthreads();
      for (int t = 0; t + 1 < n_tiles; ++t) {
        if ((t & 7) == 0 && t > 0) turn_list(t);
        if (t % 2 == 0) { bring_v(t, stage1); bring_k(t, stage0); }
        else { bring_v(t, stage0); bring_k(t, stage1); }
        brought();
      }
    } else if (n_tiles > 0) {
      static_for<PD>([&](auto f) __attribute__((always_inline)) { read(f, stage0, stage0); });
      static_for<NF>([&](auto ff) __attribute__((always_inline)) {
        constexpr int F = decltype(ff)::value, ks = F / 2, kb = F % 2;
        if constexpr (ks == 0) mfma_s_first<false, younger(F, NF)>(Sa[kb], fk[F % PD], qf[ks]);
        else mfma_s<false, younger(F, NF)>(Sa[kb], fk[F % PD], qf[ks]);
        if constexpr (F + PD < NF) read(std::integral_constant<int, F + PD>{}, stage0, stage0);
      });
      fence_s(Sa[0], Sa[1]);
      mask(0, 0, Sa);
      static_for<16>([&](auto i) __attribute__((always_inline)) { max_step(i, Sa); });
      if (n_tiles > 1) __syncthreads();          // everybody has read K(0)
      int t = 0;
      for (; t + 2 < n_tiles; t += 2) {
        if ((t & 7) == 0 && t > 0) turn_list(t);
        body(stage0, t, Sa, Sb);
        body(stage1, t + 1, Sb, Sa);
        if ((t & 62) == 62) { l_run += l_lo; l_lo = 0.f; }
      }
      if (t + 1 < n_tiles) {             // (a second way out of the loop would make the compiler copy the output in every round)
        if ((t & 7) == 0 && t > 0) turn_list(t);
        body(stage0, t, Sa, Sb);
        Sa[0] = Sb[0];
        Sa[1] = Sb[1];
#pragma unroll
        for (int db = 0; db < NDB; ++db) va[db] += C::TILE_BYTES;
      }
      tail(stage0, Sa);
    }
    // ---- Zero times an infinity or a NaN would carry V's values to rows that do not see them.  Where sums are not finite, all are formed again,
    // a step at a time, with the rows of V that hold such values taken out of the product and added one by one, and with the scores taken off their
    // maximum as they are (see beyond_fma; m_run is the maximum of the scores themselves here).
    {
      float z = 0.f;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) z = __builtin_fmaf(o[db][i], 0.f, z);
      const bool bad = __builtin_amdgcn_ballot_w64(z != 0.f || beyond_fma(m_run)) != 0;       // (0 times a number is 0)
      if (lane == 0) odd_waves[wave_u] = bad;
    }
    float m_rest = 0.f;
    __syncthreads();                     // everybody has read the last tile, too
    if (__builtin_expect((odd_waves[0] | odd_waves[1] | odd_waves[2] | odd_waves[3]) != 0, 0)) {
#pragma unroll
      for (int db = 0; db < NDB; ++db) o[db] = zero16();
      // (places formed here: outside the loop they would take registers from it)
      int th = thread;
      asm volatile("" : "+v"(th));
      const int ch = th >> 5 & 1, cq = th & 31, cga = th >> 4 & 3, cjj = th & 15, crow = 4 * (cga >> 1) + (cjj >> 2);
      const unsigned c_adr = cq * C::RB + C::swz_k(cq, ch) * 16;
      m_run = kLeast; m_raise = kLeast; l_run = 0.f; l_lo = 0.f; r_fix = 0.f;
      for (int t = 0; t < n_tiles; ++t) {
        if (t % 16 == 0) {
          take_list(t, look_up(t));
        }
        find(t, t & ~15);
        if constexpr (F8) { load(K, there, t, t & ~15); load(V, there, t, t & ~15); put(K, 0); put(V, 0); }
        else { fetch(K, stage0, there, t, t & ~15); fetch(V, stage0, there, t, t & ~15); asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
        if (thread < BT) odd_rows[thread] = 0;
        __syncthreads();
        unsigned char* const mine = smem + 2 * C::TILE_BYTES + th * (C::TILE_BYTES / C::NTHREADS);      // a quarter of row thread / 4
        bool odd = false;
#pragma unroll
        for (int i = 0; i < C::TILE_BYTES / C::NTHREADS / 16; ++i) {
          const u32x4 y = reinterpret_cast<const u32x4*>(mine)[i];
#pragma unroll
          for (int e = 0; e < 4; ++e) odd |= (y[e] & 0x7f80u) == 0x7f80u || (y[e] & 0x7f800000u) == 0x7f800000u;
        }
        if (odd) odd_rows[th / 4] = 1;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          Sa[kb] = zero16();
#pragma unroll
          for (int j = 0; j < NJ; ++j)
            Sa[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(smem + kb * 32 * C::RB + (c_adr ^ (32 * j))), __builtin_bit_cast(bf16x8, qf[j]), Sa[kb], 0, 0, 0);
        }
        unsigned hidden = 0;             // of the 32 scores (a score that is seen can be -inf, too)
        for_hidden(t, t & ~15, [&](int kb, int i) __attribute__((always_inline)) { Sa[kb][i] = -__builtin_inff(); hidden |= 1u << (16 * kb + i); });
        static_for<16>([&](auto i) __attribute__((always_inline)) { max_step(i, Sa); });
        const float m_new = fmaxf(m_run, max_of_halves(mx)), alpha = fast_exp2((m_run - m_new) * c);
        m_run = m_new;
        l_run *= alpha; l_lo *= alpha; r_fix *= alpha;
#pragma unroll
        for (int db = 0; db < NDB; ++db) o[db] *= alpha;
        const float p_top = fast_exp2((mx - m_run) * c);
        r_fix += static_cast<float>(static_cast<__bf16>(p_top)) - p_top;
        float tile_sum = 0.f;
        static_for<16>([&](auto ii) __attribute__((always_inline)) {
          constexpr int I = decltype(ii)::value;
          float y[2];
#pragma unroll
          for (int f = 0; f < 2; ++f) {
            y[f] = fast_exp2((Sa[I / 8][2 * I % 16 + f] - m_run) * c);
            tile_sum += y[f];
          }
          pf[I / 4][I % 4] = __builtin_bit_cast(unsigned, bf16x2{static_cast<__bf16>(y[0]), static_cast<__bf16>(y[1])});
        });
        l_lo += tile_sum;
        if ((t & 63) == 63) { l_run += l_lo; l_lo = 0.f; }
        __syncthreads();
        for (int j = 0; j < BT; ++j) {
          if (odd_rows[j] == 0) continue;
          // key j is element 16 (j / 32) + 4 (j % 32 / 8) + j % 4 of the half j / 4 % 2
          const int e = j / 32 * 16 + j % 32 / 8 * 4 + j % 4, from = (j / 4 % 2) * 32 + cq;
          unsigned w = 0;
          static_for<16>([&](auto ii) __attribute__((always_inline)) { constexpr int I = decltype(ii)::value; w = I == e / 2 ? pf[I / 4][I % 4] : w; });
          const float pr = __builtin_bit_cast(float, __shfl(static_cast<int>(e % 2 != 0 ? w & 0xffff0000u : w << 16), from));
          const bool sees = __shfl(static_cast<int>(hidden >> e & 1), from) == 0;
#pragma unroll
          for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int col = 32 * db + 8 * (i / 4) + 4 * ch + i % 4;
              const float y = static_cast<float>(*reinterpret_cast<const __bf16*>(smem + 2 * C::TILE_BYTES + j * C::RB + C::swz_v(j, col / 8) * 16 + col % 8 * 2));
              o[db][i] += sees ? pr * y : 0.f;
            }
        }
        __syncthreads();
        if (odd_rows[th / 4] != 0)
#pragma unroll
          for (int i = 0; i < C::TILE_BYTES / C::NTHREADS / 16; ++i) reinterpret_cast<u32x4*>(mine)[i] = u32x4{0u, 0u, 0u, 0u};
        __syncthreads();
#pragma unroll
        for (int gg = 0; gg < 4; ++gg)
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            const unsigned char* const src = smem + 2 * C::TILE_BYTES + (gg * 16 + crow) * C::RB + C::swz_v(crow, 4 * db + 2 * (cga & 1) + ((cjj & 3) >> 1)) * 16 + 8 * (cjj & 1);
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds_tr8(src, src + 8 * C::RB), __builtin_bit_cast(bf16x8, pf[gg]), o[db], 0, 0, 0);
          }
        __syncthreads();
      }
      float times;
      m_rest = rest_of_product(m_run, c, times);
      l_run *= times; l_lo *= times; r_fix *= times;
#pragma unroll
      for (int db = 0; db < NDB; ++db) o[db] *= times;
    }
    // ---- epilogue
    if (!idle) {
      const float l_mine = l_run + l_lo;
      const float l_tot = l_mine + __shfl_xor(l_mine, 32), r_tot = l_tot + (r_fix + __shfl_xor(r_fix, 32));
      const bool none = l_tot == 0.f;
      const float wb = none ? 0.f : 1.f / r_tot, lse2 = none ? -__builtin_inff() : m_run + (m_rest + __builtin_amdgcn_logf(l_tot));
      if (m < rows) {
        if (whole) {
          const int64_t rh = static_cast<int64_t>(run.s.r0 + tok) * p.Hq + head * p.G + mc - tok * p.G;
          if (p.out_fp32) {
            float* const od = static_cast<float*>(p.out) + rh * D + 4 * h;
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
              for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(od + 32 * db + 8 * i) = f32x4{o[db][4 * i] * wb, o[db][4 * i + 1] * wb, o[db][4 * i + 2] * wb, o[db][4 * i + 3] * wb};
          } else {
            __bf16* const od = static_cast<__bf16*>(p.out) + rh * D + 4 * h;
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                *reinterpret_cast<bf16x4*>(od + 32 * db + 8 * i) = bf16x4{static_cast<__bf16>(o[db][4 * i] * wb), static_cast<__bf16>(o[db][4 * i + 1] * wb), static_cast<__bf16>(o[db][4 * i + 2] * wb), static_cast<__bf16>(o[db][4 * i + 3] * wb)};
          }
          if (h == 0) p.lse[rh] = lse2 * kLn2;
        } else {
          float* const part = part_of<BM, D>(p, worker, run.x0 > 0);
          float* const od = part + (m - rt * BM) * D + 4 * h;
#pragma unroll
          for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(od + 32 * db + 8 * i) = f32x4{o[db][4 * i] * wb, o[db][4 * i + 1] * wb, o[db][4 * i + 2] * wb, o[db][4 * i + 3] * wb};
          if (h == 0) { float* const beside = part + BM * D + m - rt * BM; beside[0] = m_run; beside[BM] = l_tot; beside[2 * BM] = m_rest; }
        }
      }
    }
    if (last_piece) break;
    run.step();
    more = run.next(p, lane);
  }
  leave_split(p, worker, split);
}

// Three and two workgroups to a CU.  Beside its keys a row tile costs as much as 512 of them, and less than 512 are not split off one: a partial result
// is as dear (12 ragged chunks of up to 1 500 new tokens: 114 us, 129 with 128 and 256; a window of 2 048 at d = 64: 109 and 112).
bool cut(PagedAttn& p, bool e4m3, int d) { return set_cut(p, 128, d == 64 && !e4m3 ? 768 : 512, 512, 512, 512); }

template <int D, bool F8>
hipError_t launch_variant(const PagedAttn& p, hipStream_t stream) {
  using C = PTileCfg<D, F8>;
  const hipError_t e = TASP_LAUNCH((paged_tile_kernel<D, F8>), dim3(static_cast<unsigned>(p.workers)), dim3(C::NTHREADS), stream, p);
  return e != hipSuccess ? e : launch_paged_combine<D, C::BM>(p, stream);
}

}  // namespace

int64_t paged_tile_workspace(PagedAttn p, bool e4m3, int d) { return cut(p, e4m3, d) ? workspace_of(p, 128, d) : 0; }

hipError_t launch_paged_tile(PagedAttn p, bool e4m3, int d, hipStream_t stream) {
  if (!cut(p, e4m3, d)) return hipErrorInvalidValue;
  place_split(p, 128, d);
  if (d == 64) return e4m3 ? launch_variant<64, true>(p, stream) : launch_variant<64, false>(p, stream);
  return e4m3 ? launch_variant<128, true>(p, stream) : launch_variant<128, false>(p, stream);
}

}  // namespace tasp
