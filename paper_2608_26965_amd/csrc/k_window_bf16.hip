// Attention with a sliding window and sinks, bf16, on the matrix cores.
//
// One workgroup per (head, 128 queries), one wavefront per 32 queries, which
// walks the 64-key tiles that one of its rows sees. S^T = K Q^T and O^T =
// V^T P^T as in the block-sparse attention (a lane holds one query's logits, and
// its probabilities are the value product's operand as they stand); keys and
// values both stay row-major in LDS (row_tile.h), the value product's operand
// is read transposed.
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
#include <math.h>

#include "row_tile.h"
#include "seq.h"

namespace ca {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kVmcnt0 = 0x0F70;  // s_waitcnt immediate: vmcnt = 0 only
constexpr int kRows = 128;       // queries of a workgroup
constexpr int KT = 64;           // keys of a tile

// Workgroup w of the grid runs on XCD w % 8. All XCDs work on the same head at
// a time. Where the window is short each takes a contiguous eighth of the
// head's row blocks (neighbours read the same keys, which then stay in that
// XCD's L2), else every eighth block, the ones with most keys first (causal
// attention without a window: a contiguous eighth would leave the last XCD with
// twice the mean work). The start rotates with the key head, so that heads of
// few blocks spread over the XCDs.
struct BlockOrder {
  int nb, splits, G, contiguous;
  int64_t grid(int BH) const { return (int64_t)8 * ((nb + 7) / 8) * BH * splits; }
  __device__ __forceinline__ bool at(int wg, int* bh, int* a, int* sp) const {
    const int chunk = (nb + 7) >> 3, loc = wg >> 3;
    const int hs = loc / chunk, s = loc - hs * chunk;
    *bh = hs / splits;
    *sp = hs - *bh * splits;
    const int x = ((wg & 7) + *bh / G + *sp) & 7;
    if (contiguous) {
      const int first = (int)((int64_t)x * nb >> 3), end = (int)((int64_t)(x + 1) * nb >> 3);
      *a = first + s;
      return *a < end;
    }
    *a = nb - 1 - (8 * s + x);
    return *a >= 0;
  }
};

// What a wavefront's rows at positions [p0, p1] have to do with the keys
// [k0, k0 + KT): 0 no row sees one, 2 every row sees all, 1 else
__device__ __forceinline__ int tile_class(const KeyRange& a, const KeyRange& z, int k0) {
  if (k0 >= z.s_end && (k0 >= z.hi || k0 + KT <= a.lo)) return 0;
  return k0 + KT <= a.s_end || (k0 >= z.lo && k0 + KT <= a.hi) ? 2 : 1;
}

template <int D, bool SPLIT>
__global__ __launch_bounds__(256, (D == 64 ? 3 : 2)) void window_bf16_kernel(
    const WinProb P, const bf16* __restrict__ q, const bf16* __restrict__ k,
    const bf16* __restrict__ v, bf16* __restrict__ out, float* __restrict__ lse,
    float* __restrict__ part, const BlockOrder order, float sl2) {
  constexpr int NW = 4, KS = D / 16, DT = D / 32, RB = 2 * D, TILE = KT * RB;
  __shared__ __attribute__((aligned(1024))) char smem[4 * TILE];  // two tiles of keys, two of values
  __shared__ int redo;
  int bh, a, sp;
  if (!order.at(blockIdx.x, &bh, &a, &sp)) return;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = bh / P.H, bk = b * P.Hk + (bh - b * P.H) / P.G;
  const int lq = P.qlen(b), lk = P.klen(b), off = lk - lq, q0 = a * kRows;
  const int real = max(0, min(kRows, lq - q0));
  TileList list{0, 0, 0};
  if (real > 0) list = visible_tiles<KT>(P.m, q0 + off, q0 + real - 1 + off, lk);
  int t0 = 0, t1 = list.n;
  if constexpr (SPLIT) {
    const int per = (list.n + order.splits - 1) / order.splits;
    t0 = min(list.n, sp * per);
    t1 = min(list.n, t0 + per);
  }
  const int w0 = q0 + 32 * w, wreal = max(0, min(32, lq - w0));
  const KeyRange ra = visible_keys(P.m, w0 + off, lk);
  const KeyRange rz = visible_keys(P.m, w0 + max(wreal, 1) - 1 + off, lk);
  const int i = min(w0 + min(l32, max(wreal, 1) - 1), P.nq - 1);  // this lane's query

  bf16x8 qreg[KS];
  {
    const bf16* row = q + row_off(bh, i, P.lq);
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) qreg[kk] = *(const bf16x8*)(row + 16 * kk + 8 * h);
  }
  // Retire the loads here (a wait the compiler sees), so that no vmcnt wait of
  // theirs lands in the loop, where it would also wait for the copies in flight.
  __builtin_amdgcn_s_waitcnt(kVmcnt0);
  if (tid == 0) redo = 0;  // ordered before any write by the barriers of the tiles

  const bf16* kbase = k + row_off(bk, 0, P.lk);
  const bf16* vbase = v + row_off(bk, 0, P.lv);
  const RowCopy<RB, KT, NW> kcopy(w, lane, (uint32_t)(P.lk.sn * 2));
  const RowCopy<RB, KT, NW> vcopy(w, lane, (uint32_t)(P.lv.sn * 2));
  const uint32_t lds0 = lds_addr(smem);
  auto issue_k = [&](int t, int buf) __attribute__((always_inline)) {
    const int k0 = KT * list.tile(t);
    kcopy.issue(kbase + (int64_t)k0 * P.lk.sn, lds0 + buf * TILE, w, lane, lk - 1 - k0);
  };
  auto issue_v = [&](int t, int buf) __attribute__((always_inline)) {
    const int k0 = KT * list.tile(t);
    vcopy.issue(vbase + (int64_t)k0 * P.lv.sn, lds0 + (2 + buf) * TILE, w, lane,
                lk - 1 - k0);
  };
  int koff[KS], voff[DT][2];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) koff[kk] = row_operand<RB>(lane, kk);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int t = 0; t < 2; ++t) voff[dt][t] = col_operand<RB>(lane, dt, t);

  f32x16 oacc[DT], sacc[2];
  bf16x8 pb[2][2];  // probabilities, the value product's operand
  float m, l;       // reference (log2 units) and this lane's part of the sum
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
  auto mask = [&](int k0) __attribute__((always_inline)) {
    int p = i + off;
    asm volatile("" : "+v"(p));
    const KeyRange rr = visible_keys(P.m, p, lk);
    const int a0 = k0 + 4 * h - rr.lo, b0 = rr.s_end - k0 - 4 * h;
    const uint32_t len = (uint32_t)max(0, rr.hi - rr.lo);
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int c = 32 * mt + 8 * (r >> 2) + (r & 3);
        if (!((uint32_t)(a0 + c) < len || c < b0)) sacc[mt][r] = -INFINITY;
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
    // (2^22 keys at most: against maxima no sum is larger)
    l = m_new - m > 126.f && l > 0x1p22f ? INFINITY : l * alpha;
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
    if (t + 1 < t1) issue_k(t + 1, PAR ^ 1);
    issue_v(t, PAR);
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
    const int k0 = KT * list.tile(t), c = tile_class(ra, rz, k0);
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
  if (t0 < t1) {
    issue_k(t0, 0);
    copies(even, t0);
    if (wreal == 0) {  // no rows: copies only
      for (int t = t0 + 1; t < t1; t += 2) {
        copies(odd, t);
        if (t + 1 < t1) copies(even, t + 1);
      }
      sync_stage();
    } else {
      const int k0 = KT * list.tile(t0);
      logits(smem);
      reference(tile_class(ra, rz, k0), k0, true);
      const float ref = m == -INFINITY ? 0.f : m;
      groups([&](int mt, int s2) { exp_group(mt, s2, ref); });
      for (int t = t0 + 1; t < t1; t += 2) {
        step(odd, t);
        if (t + 1 < t1) step(even, t + 1);
      }
      sync_stage();
      const char* vs = smem + (2 + ((t1 - 1 - t0) & 1)) * TILE;
      groups([&](int mt, int s2) { pv_group(vs, mt, s2); });
    }
  }
  float l_tot = l + wave_xor32(l);
  bool poison = false;
  {
    bool fine = l_tot <= 0x1p126f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) fine &= fabsf(oacc[dt][r]) <= 0x1p127f;
    if (__builtin_amdgcn_ballot_w64(!fine) && lane == 0) redo = 1;
  }
  __syncthreads();
  if (redo) {
    // The workgroup starts over, one tile after the other, each against its own
    // maximum. Where the reason was a value that is infinite or NaN and that some row of
    // the block does not see (zero times it is NaN), `guard` sets the rows of the tile that
    // hold one to zero, and queries that do see one get NaN at the end. Every wavefront
    // looks through all of the tile, so all agree on whether there is anything to do.
    auto guard = [&](char* vs, int k0) __attribute__((always_inline)) {
      if (tile_class(visible_keys(P.m, q0 + off, lk), visible_keys(P.m, q0 + real - 1 + off, lk),
                     k0) == 2)
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
      const KeyRange rr = visible_keys(P.m, i + off, lk);
      for (; bad; bad &= bad - 1) poison |= sees(rr, k0 + __builtin_ctzll(bad));
    };

    reset();
    for (int t = t0; t < t1; ++t) {
      const int k0 = KT * list.tile(t);
      issue_k(t, 0);
      issue_v(t, 0);
      sync_stage();
      guard(smem + 2 * TILE, k0);
      if (wreal) {
        logits(smem);
        const bool raised = reference(tile_class(ra, rz, k0), k0, false);
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
  if constexpr (SPLIT) {
    // A sum far above its reference goes out against a reference at its own size: the
    // joining compares references, and adds up as many sums as there are parts
    const int up = l_tot > 0x1p22f ? __builtin_amdgcn_frexp_expf(l_tot) : 0;
    m += (float)up;
    l_tot = __builtin_amdgcn_ldexpf(l_tot, -up);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[dt][r] = __builtin_amdgcn_ldexpf(oacc[dt][r], -up);
    float* row = part + ((((size_t)bh * order.nb + a) * kRows + 32 * w + l32) * order.splits + sp) *
                            (D + 4);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 x = {oacc[dt][4 * g], oacc[dt][4 * g + 1], oacc[dt][4 * g + 2],
                         oacc[dt][4 * g + 3]};
        *(f32x4*)(row + 32 * dt + 8 * g + 4 * h) = x;
      }
    if (h == 0) {
      row[D] = m;
      row[D + 1] = l_tot;
    }
    return;
  }
  const int row = w0 + l32;
  if (row >= P.nq) return;
  const bool real_row = l32 < wreal && l_tot != 0.f;
  const float inv = real_row ? 1.f / l_tot : 0.f;
  bf16* orow = out + row_off(bh, row, P.lo);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = f2bf(real_row ? oacc[dt][4 * g + j] * inv : 0.f);
      *(bf16x4*)(orow + 32 * dt + 8 * g + 4 * h) = x;
    }
  if (lse && h == 0)
    lse[(size_t)bh * P.nq + row] =
        real_row ? (m + __builtin_amdgcn_logf(l_tot)) * kLn2 : -INFINITY;
}

// Joins the parts of a row: one wavefront a row, four rows a workgroup.
template <int D>
__global__ __launch_bounds__(256) void window_join_kernel(const WinProb P,
                                                          const float* __restrict__ part, int nb,
                                                          int splits, bf16* __restrict__ out,
                                                          float* __restrict__ lse) {
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int bh = (int)(id / P.nq), i = (int)(id - (int64_t)bh * P.nq);
  if (bh >= P.B * P.H) return;
  const bool real = i < P.qlen(bh / P.H);
  const float* p = part + ((size_t)bh * nb * kRows + i) * splits * (D + 4);
  float mx = -INFINITY;
  for (int s = 0; s < splits; ++s)
    if (p[s * (D + 4) + D + 1] != 0.f) mx = fmaxf(mx, p[s * (D + 4) + D]);
  float sum = 0.f, x0 = 0.f, x1 = 0.f;
  for (int s = 0; s < splits; ++s) {
    const float* r = p + s * (D + 4);
    if (r[D + 1] == 0.f) continue;  // no key of the part is visible
    const float f = __builtin_amdgcn_exp2f(r[D] - mx);
    sum += f * r[D + 1];
    x0 += f * r[lane];
    if constexpr (D == 128) x1 += f * r[lane + 64];
  }
  const bool any = real && sum != 0.f;
  const float inv = any ? 1.f / sum : 0.f;
  bf16* o = out + row_off(bh, i, P.lo);
  o[lane] = f2bf(any ? x0 * inv : 0.f);
  if constexpr (D == 128) o[lane + 64] = f2bf(any ? x1 * inv : 0.f);
  if (lse && lane == 0)
    lse[(size_t)bh * P.nq + i] = any ? (mx + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
}

// Parts that the keys of a row block are cut into. A launch of fewer than 384
// workgroups leaves compute units idle (256 of them, two workgroups each or
// three), so short ones take about 512, of at least eight tiles each.
int window_splits(const WinProb& P) {
  const int64_t wgs = (int64_t)((P.nq + kRows - 1) / kRows) * P.B * P.H;
  if (wgs >= 384) return 1;
  int64_t keys = (int64_t)P.m.left + (P.m.causal ? 0 : P.m.right) + kRows + P.m.sinks;
  if (keys > P.nk) keys = P.nk;
  const int64_t want = (512 + wgs - 1) / wgs, room = keys / (8 * KT);
  const int64_t s = want < room ? want : room;
  return (int)(s < 1 ? 1 : s);
}

template <int D>
hipError_t run_window(const WinProb& P, const bf16* q, const bf16* k, const bf16* v, bf16* out,
                      float* lse, float* part, hipStream_t st) {
  BlockOrder order{(P.nq + kRows - 1) / kRows, window_splits(P), P.G, 0};
  // the keys of an eighth of the blocks next to those of all
  order.contiguous = (int64_t)P.m.left + (P.m.causal ? 0 : P.m.right) < P.nk / 2;
  const dim3 grid((unsigned)order.grid(P.B * P.H));
  const float sl2 = P.scale * kLog2e;
  if (order.splits == 1) {
    hipLaunchKernelGGL((window_bf16_kernel<D, false>), grid, dim3(256), 0, st, P, q, k, v, out, lse,
                       part, order, sl2);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((window_bf16_kernel<D, true>), grid, dim3(256), 0, st, P, q, k, v, out, lse,
                     part, order, sl2);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)P.B * P.H * P.nq;
  hipLaunchKernelGGL((window_join_kernel<D>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, P,
                     part, order.nb, order.splits, out, lse);
  return hipGetLastError();
}

}  // namespace

size_t window_bf16_bytes(const WinProb& P) {
  const int s = window_splits(P);
  if (s == 1) return 0;
  const size_t rows = (size_t)P.B * P.H * ((P.nq + kRows - 1) / kRows) * kRows;
  return (rows * s * (P.d + 4) * 4 + 255) & ~(size_t)255;
}

hipError_t launch_window_bf16(const WinProb& P, const void* q, const void* k, const void* v,
                              void* out, float* lse, char* ws, hipStream_t st) {
  if (P.d == 64)
    return run_window<64>(P, (const bf16*)q, (const bf16*)k, (const bf16*)v, (bf16*)out, lse,
                          (float*)ws, st);
  return run_window<128>(P, (const bf16*)q, (const bf16*)k, (const bf16*)v, (bf16*)out, lse,
                         (float*)ws, st);
}

}  // namespace ca
