// The walk of a workgroup's queries over 64-key tiles, bf16 on the matrix cores:
// window attention and the attention of chunks over a paged cache. A wavefront
// owns 32 queries; the workgroup copies tiles of keys and values to LDS together.
//
// S^T = K Q^T and O^T = V^T P^T as in the block-sparse attention (a lane holds one
// query's logits, and its probabilities are the value product's operand as they
// stand); keys and values both stay row-major in LDS (row_tile.h), the value
// product's operand is read transposed.
//
// Scale and reference are applied in fp32 (one fused multiply-add a logit) and
// the row sums add the probabilities before they are rounded to bf16: queries
// pre-scaled in bf16 and sums of rounded probabilities would put the
// log-sum-exp off by 10^-4. Probabilities are rounded to bf16 (2^-8 each) for the
// product; the result is rounded once.
//
// A tile that every row of the wavefront sees runs without a maximum, against
// the reference that the rows have: probabilities above 1 cost no accuracy while
// nothing overflows. Tiles at the edges of the window, and the first ones, take the
// maximum and rescale, which loses what is scaled by less than 2^-126 (the
// exponential of that is 0): no weight to speak of next to a sum of at most the number
// of keys, but perhaps most of a sum that grew far above its reference. Where a
// large sum meets such a factor, or one overflows (checked once at the end), the
// workgroup starts over with a maximum in every tile.
#pragma once

#include <math.h>

#include "row_tile.h"
#include "seq.h"

namespace ca {

constexpr int kWalkVmcnt0 = 0x0F70;  // s_waitcnt immediate: vmcnt = 0 only
constexpr int kWalkRows = 128;       // queries of a workgroup
constexpr int KT = 64;               // keys of a tile

// What a wavefront's rows at positions [p0, p1] have to do with the keys
// [k0, k0 + KT): 0 no row sees one, 2 every row sees all, 1 else
__device__ __forceinline__ int tile_class(const KeyRange& a, const KeyRange& z, int k0) {
  if (k0 >= z.s_end && (k0 >= z.hi || k0 + KT <= a.lo)) return 0;
  return k0 + KT <= a.s_end || (k0 >= z.lo && k0 + KT <= a.hi) ? 2 : 1;
}

// What the walk knows of its tiles and rows; a Tiles class adds
//   void first_k()            starts the copy of tile t0's keys into key buffer 0; with kBegun
//                             these, its values and the keys of tile t0 + 1 are on their way
//   void issue_k(t, buf)      ... of tile t's keys into key buffer `buf`
//   void issue_v(t, buf)      ... of tile t's values into value buffer `buf`
//   void issue_both(t)        ... of both into the buffers 0
//   uint64_t holes(buf)       keys of the tile in key buffer `buf` that are not there, bit
//                             by bit, once its copies have landed (kHoles true only)
//   kMostSum                  at least the number of keys
// called by all wavefronts alike, in the order issue_k(t + 1), issue_v(t).
struct WalkRows {
  WinMask mask;
  TileList list;
  int t0, t1;                    // tiles of the list
  int lk;                        // keys
  KeyRange ra, rz;               // what the wavefront's first and last row see
  int pos;                       // this lane's query
  int real;                      // rows of the wavefront
  int block_first, block_last;   // positions of the workgroup's first and last row
  __device__ __forceinline__ int tile(int t) const { return list.tile(t); }
};

// Afterwards oacc holds the sums of probabilities times values (accumulator r of
// oacc[dt]: dim 32 dt + 8 (r / 4) + 4 h + r % 4 of query l % 32) against the reference
// m (log2 units) and l_tot their sum; oacc is NaN where a value that is not finite is seen.
// *redo (in LDS) has to be 0 before the first tile's barrier.
template <int D, class Tiles>
__device__ __forceinline__ void walk_bf16(Tiles& T, char* smem, int* redo,
                                          const bf16x8 (&qreg)[D / 16], float sl2, int w, int lane,
                                          f32x16 (&oacc)[D / 32], float& m, float& l_tot) {
  constexpr int KS = D / 16, DT = D / 32, RB = 2 * D, TILE = KT * RB;
  const int h = lane >> 5;
  int koff[KS], voff[DT][2];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) koff[kk] = row_operand<RB>(lane, kk);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int t = 0; t < 2; ++t) voff[dt][t] = col_operand<RB>(lane, dt, t);

  f32x16 sacc[2];
  bf16x8 pb[2][2];  // probabilities, the value product's operand
  float l;          // this lane's part of the sum
  float alpha;      // what a raised reference scales the results so far by
  bool set;         // every row of the wavefront has a reference

  // Operands are read a step ahead of their products, a fence between (left to itself
  // the compiler reads each right before its product and waits).
  auto logits = [&](const char* ks) __attribute__((always_inline)) {
    constexpr int ST = KS / 2;  // steps of a row tile
    bf16x8 av[2][2];
    auto load = [&](int n) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
        av[n & 1][x] = *(const bf16x8*)(ks + 32 * (n / ST) * RB + koff[2 * (n % ST) + x]);
    };
    f32x16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
    load(0);
#pragma unroll
    for (int n = 0; n < 2 * ST; ++n) {
      const int mt = n / ST;
      if (n + 1 < 2 * ST) load(n + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int kk = 2 * (n % ST) + x;
        sacc[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[n & 1][x], qreg[kk],
                                                           kk == 0 ? z : sacc[mt], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // accumulator r of row tile mt is key k0 + 32 mt + 8 (r / 4) + 4 h + r % 4
  // (the query's ranges are formed here: kept over the loop they cost registers)
  uint64_t hv = 0;  // keys of the tile that are not there
  auto mask = [&](int k0) __attribute__((always_inline)) {
    int p = T.pos;
    asm volatile("" : "+v"(p));
    const KeyRange rr = visible_keys(T.mask, p, T.lk);
    const int a0 = k0 + 4 * h - rr.lo, b0 = rr.s_end - k0 - 4 * h;
    const uint32_t len = (uint32_t)max(0, rr.hi - rr.lo);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int c = 32 * mt + 8 * (r >> 2) + (r & 3);
        if (!((uint32_t)(a0 + c) < len || c < b0)) sacc[mt][r] = -INFINITY;
      }
    if (Tiles::kHoles && hv) {
      const uint64_t x = hv >> (4 * h);
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if ((x >> (32 * mt + 8 * (r >> 2) + (r & 3))) & 1) sacc[mt][r] = -INFINITY;
    }
  };
  auto exp_group = [&](int mt, int s2, float ref) __attribute__((always_inline)) {
    float pv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      pv[j] = __builtin_amdgcn_exp2f(fmaf(sacc[mt][8 * s2 + j], sl2, -ref));
    l += ((pv[0] + pv[1]) + (pv[2] + pv[3])) + ((pv[4] + pv[5]) + (pv[6] + pv[7]));
    pb[mt][s2] = pack8(pv);
  };
  auto pv_group = [&](const char* vs, int mt, int s2) __attribute__((always_inline)) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const char* at = vs + (32 * mt + 16 * s2) * RB;
      const bf16x8 av = read_cols(at + voff[dt][0], at + voff[dt][1]);
      oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av, pb[mt][s2], oacc[dt], 0, 0, 0);
    }
  };
  // The class of the tile in key buffer `buf`, and its holes (before its logits: nothing
  // waits for them there)
  auto class_of = [&](int buf, int k0) __attribute__((always_inline)) {
    int c = tile_class(T.ra, T.rz, k0);
    if constexpr (Tiles::kHoles) {
      hv = T.holes(buf);
      if (hv && c == 2) c = 1;
    }
    return c;
  };
  // The reference of a tile of class c: the rows' own where every row has one and
  // sees all of the tile (`keep`), else raised to the tile's maximum. True if raised.
  auto reference = [&](int c, int k0, bool keep) __attribute__((always_inline)) {
    if (keep && c == 2 && set) return false;
    if (c == 1) mask(k0);
    if (c == 0) {
#pragma unroll
      for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[mt][r] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[mt][r]);
    mx = fmaxf(mx, wave_xor32(mx));
    const float m_new = fmaxf(m, mx * sl2);
    alpha = m_new > m ? __builtin_amdgcn_exp2f(m - m_new) : 1.f;
    // (against maxima no sum is larger than the number of keys)
    l = m_new - m > 126.f && l > Tiles::kMostSum ? INFINITY : l * alpha;
    const bool raised = __builtin_amdgcn_ballot_w64(m_new > m) != 0;
    m = m_new;
    set = __builtin_amdgcn_ballot_w64(m == -INFINITY) == 0;
    return raised;
  };
  auto sync_stage = [&]() __attribute__((always_inline)) {
    wait_vmcnt<0>();
    wait_lgkm();
    raw_barrier();
  };
  // Tile g's keys sit in key buffer g % 2 and its values in value buffer g % 2
  // (g counted from t0). After iteration g's barrier every wavefront is past
  // iteration g - 1 and the copies that it issued have landed: the keys of tile
  // g + 1 and the values of tile g are copied, the logits of tile g formed, and
  // the value product of tile g - 1 runs among the exponentials of tile g. The
  // two edge cases (a tile that none of the wavefront's rows sees, a raised
  // reference) stay around that one piece of code, so that the accumulators stay
  // in place.
  auto copies = [&](auto par_tag, int t) __attribute__((always_inline)) {
    constexpr int PAR = decltype(par_tag)::value;
    sync_stage();
    if (t + 1 < T.t1) T.issue_k(t + 1, PAR ^ 1);
    T.issue_v(t, PAR);
  };
  auto groups = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) f(mt, s2);
  };
  auto rescale = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[dt][r] *= alpha;
  };
  auto step = [&](auto par_tag, int t) __attribute__((always_inline)) {
    constexpr int PAR = decltype(par_tag)::value;
    copies(par_tag, t);
    const int k0 = KT * T.tile(t), c = class_of(PAR, k0);
    logits(smem + PAR * TILE);
    const bool raised = reference(c, k0, true);
    const float ref = m == -INFINITY ? 0.f : m;  // no key yet
    const char* vs = smem + (2 + (PAR ^ 1)) * TILE;
    constexpr int SV = DT / 2;  // steps of a group: two products and some of its exponentials
    bf16x8 av[2][2];
    auto load = [&](int n) __attribute__((always_inline)) {
      const char* at = vs + 16 * (n / SV) * RB;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int dt = 2 * (n % SV) + x;
        av[n & 1][x] = read_cols(at + voff[dt][0], at + voff[dt][1]);
      }
    };
    load(0);
    float p[8];
    // Products go before the other wavefront's exponentials, and every other tile before the
    // other wavefront's: of equal ones the older goes first, whose workgroup then ended 9% before
    // the younger one of its compute unit (8,192 tokens on 24,576: 3.48 -> 3.40 ms)
    if constexpr (Tiles::kBegun) __builtin_amdgcn_s_setprio(1 + PAR);
#pragma unroll
    for (int n = 0; n < 4 * SV; ++n) {
      const int mt = n / SV / 2, s2 = n / SV % 2, st = n % SV;
      if (n + 1 < 4 * SV) load(n + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < 2; ++x)
        oacc[2 * st + x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(av[n & 1][x], pb[mt][s2],
                                                                   oacc[2 * st + x], 0, 0, 0);
#pragma unroll
      for (int j = 8 / SV * st; j < 8 / SV * (st + 1); ++j)
        p[j] = __builtin_amdgcn_exp2f(fmaf(sacc[mt][8 * s2 + j], sl2, -ref));
      if (st == SV - 1) {
        l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
        pb[mt][s2] = pack8(p);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (Tiles::kBegun) __builtin_amdgcn_s_setprio(PAR);
    if (raised) rescale();
  };
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  auto reset = [&]() __attribute__((always_inline)) {
    m = -INFINITY;
    l = 0.f;
    set = false;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[dt][r] = 0.f;
  };
  reset();
  if (T.t0 < T.t1) {
    if constexpr (Tiles::kBegun) {
      sync_stage();
    } else {
      T.first_k();
      copies(even, T.t0);
    }
    if (T.real == 0) {  // no rows: copies only
      for (int t = T.t0 + 1; t < T.t1; t += 2) {
        copies(odd, t);
        if (t + 1 < T.t1) copies(even, t + 1);
      }
      sync_stage();
    } else {
      const int k0 = KT * T.tile(T.t0), c = class_of(0, k0);
      logits(smem);
      reference(c, k0, true);
      const float ref = m == -INFINITY ? 0.f : m;
      groups([&](int mt, int s2) { exp_group(mt, s2, ref); });
      for (int t = T.t0 + 1; t < T.t1; t += 2) {
        step(odd, t);
        if (t + 1 < T.t1) step(even, t + 1);
      }
      sync_stage();
      const char* vs = smem + (2 + ((T.t1 - 1 - T.t0) & 1)) * TILE;
      groups([&](int mt, int s2) { pv_group(vs, mt, s2); });
    }
  }
  l_tot = l + wave_xor32(l);
  bool poison = false;
  {
    bool fine = l_tot <= 0x1p126f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) fine &= fabsf(oacc[dt][r]) <= 0x1p127f;
    if (__builtin_amdgcn_ballot_w64(!fine) && lane == 0) *redo = 1;
  }
  __syncthreads();
  if (*redo) {
    // The workgroup starts over, one tile after the other, each against its own
    // maximum. Where the reason was a value that is infinite or NaN and that some row of
    // the block does not see (zero times it is NaN), `guard` sets the rows of the tile that
    // hold one to zero, and queries that do see one get NaN at the end. Every wavefront
    // looks through all of the tile, so all agree on whether there is anything to do.
    auto guard = [&](char* vs, int k0) __attribute__((always_inline)) {
      if (tile_class(visible_keys(T.mask, T.block_first, T.lk),
                     visible_keys(T.mask, T.block_last, T.lk), k0) == 2)
        return;
      typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      constexpr int NCH = RB / 16;
      u16x2 most = {0, 0};
#pragma unroll 2
      for (int c = 0; c < NCH; ++c) {
        const u32x4 x = *(const u32x4*)(vs + lane * RB + ((c + lane) % NCH) * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x[j] & 0x7fff7fffu));
      }
      uint64_t bad = __builtin_amdgcn_ballot_w64(most.x >= 0x7f80 || most.y >= 0x7f80);
      if (__builtin_expect(bad == 0, 1)) return;
      __syncthreads();
      if (w == 0 && ((bad >> lane) & 1)) {
#pragma unroll 1
        for (int c = 0; c < NCH; ++c) *(f32x4*)(vs + lane * RB + c * 16) = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      __syncthreads();
      if constexpr (Tiles::kHoles) bad &= ~T.holes(0);  // (they hold another key's value)
      const KeyRange rr = visible_keys(T.mask, T.pos, T.lk);
      for (; bad; bad &= bad - 1) poison |= sees(rr, k0 + __builtin_ctzll(bad));
    };

    reset();
    for (int t = T.t0; t < T.t1; ++t) {
      const int k0 = KT * T.tile(t);
      T.issue_both(t);
      sync_stage();
      guard(smem + 2 * TILE, k0);
      if (T.real) {
        const int c = class_of(0, k0);
        logits(smem);
        const bool raised = reference(c, k0, false);
        const float ref = m == -INFINITY ? 0.f : m;
        if (raised) rescale();
        groups([&](int mt, int s2) {
          exp_group(mt, s2, ref);
          pv_group(smem + 2 * TILE, mt, s2);
        });
      }
      __syncthreads();  // every wavefront is past the tile
    }
    l_tot = l + wave_xor32(l);
  }
  if (poison) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[dt][r] = NAN;
  }
}

}  // namespace ca
