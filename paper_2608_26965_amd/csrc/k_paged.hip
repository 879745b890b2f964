// Attention of one new token of each sequence over a paged key-value cache.
//
// The tiles of keys that a sequence's token sees (the sinks', then its window's)
// are cut into parts of one size for all sequences, a workgroup each per key head, so
// that a few long sequences fill the chip and sequences of different lengths
// balance; the parts' softmax states are joined by a second launch. All query
// heads of a key head share its keys. What bounds it: the cache, read once.
#include <math.h>

#include "f32_tile.h"
#include "row_tile.h"
#include "seq.h"

namespace ca {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kTile = 32;   // keys of a tile
constexpr int kPartTiles = 8;  // tiles of a part, at least
constexpr int kJoin = 1024;  // threads of the joining kernel

// The keys that the token of a sequence of len keys sees, and their tiles
struct SeenKeys {
  KeyRange r;
  TileList list;
};
__device__ __forceinline__ SeenKeys seen_keys(const PagedProb& P, int len) {
  SeenKeys s;
  s.r.s_end = min(P.sinks, len);
  s.r.lo = max(0, len - 1 - P.left);
  s.r.hi = len;
  s.list.ns = (s.r.s_end + kTile - 1) / kTile;
  s.list.b0 = max(s.list.ns, s.r.lo / kTile);
  s.list.n = s.list.ns + max(0, (len + kTile - 1) / kTile - s.list.b0);
  return s;
}
// key j0 + i of a tile that holds a visible key, or for a hidden one a visible key of
// the tile (hidden rows are not read: their pages may be gone, what they hold
// may be anything)
__device__ __forceinline__ int nearest_seen(const KeyRange& r, int j0, int i) {
  int j = min(j0 + i, r.hi - 1);
  if (j >= r.s_end && j < r.lo) j = r.lo < j0 + kTile ? r.lo : r.s_end - 1;
  return j;
}

// ---- fp32 (f32_tile.h) ----------------------------------------------------------------

template <int DP>
struct PagedKeys {
  const float *k, *v;  // of this key head
  const int32_t* table;
  const PagedProb& P;
  SeenKeys seen;
  int first, ntile, lane;  // tiles of 16 keys, from the one numbered `first`

  // page and place of key i of tile t; -1 where there is none
  __device__ __forceinline__ int place(int t, int i, int& in) const {
    if (t >= ntile) return -1;
    const int x = first + t;
    const int j = kTile * seen.list.tile(x / 2) + 16 * (x % 2) + i;
    if (!sees(seen.r, j)) return -1;
    const int e = j / P.page;
    in = j - e * P.page;
    const int pg = table[e];
    return pg < P.pages ? pg : -1;
  }
  __device__ __forceinline__ void rows(int t, f32x4 (&f)[DP / 16]) const {
    int in = 0;
    const int pg = place(t, lane & 15, in);
#pragma unroll
    for (int j = 0; j < DP / 16; ++j) {
      const int x = 16 * j + 4 * (lane >> 4);
      f[j] = pg >= 0 && x < P.d ? load4f(k + pg * P.k_sp + in * P.k_st + x)
                                : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  __device__ __forceinline__ void vals(int t, f32x4 (&f)[DP / 16]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      int in = 0;
      const int pg = place(t, 4 * (lane >> 4) + r, in);
#pragma unroll
      for (int x = 0; x < DP / 16; ++x) {
        const int dim = 16 * x + (lane & 15);
        f[x][r] = pg >= 0 && dim < P.d ? v[pg * P.v_sp + in * P.v_st + dim] : 0.f;
      }
    }
  }
  __device__ __forceinline__ void mask_vals(int, f32x4 (&)[DP / 16]) const {}
  __device__ __forceinline__ void logits(int t, f32x4& s) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      int in = 0;
      s[r] = place(t, 4 * (lane >> 4) + r, in) >= 0 ? s[r] * P.scale : -INFINITY;
    }
  }
};

// A workgroup: part `sp` (tiles per part: `tiles`) of key head bk, query heads g0 ..
// g0 + 15 of its group. Parts that a sequence does not have end at once.
struct PartOf {
  int b, hk, g0, rows, sp;
  // Parts go slowest and the heads rotate with them: workgroup i runs on XCD
  // i % 8, and with a sequence's parts on neighbouring workgroups the XCDs that
  // hold the late parts had only the longest sequences (32 sequences of 512 to
  // 32,768, eight parts: 451 us, now 240).
  __device__ __forceinline__ PartOf(const PagedProb& P, int splits) {
    const int qt = (P.G + 15) / 16, heads = P.B * P.Hk;
    const int s = blockIdx.x / heads, x = blockIdx.x - s * heads;
    sp = s / qt;
    g0 = 16 * (s - sp * qt);
    const int bk = (x + sp) % heads;
    b = bk / P.Hk;
    hk = bk - b * P.Hk;
    rows = min(16, P.G - g0);
  }
  __device__ __forceinline__ int head(const PagedProb& P, int r) const { return hk * P.G + g0 + r; }
};

// Part results: [B H][splits] of (d sums, reference in log2 units, sum of exponentials)
__device__ __forceinline__ float* part_of(const PagedProb& P, float* part, int splits, int b, int h,
                                          int sp) {
  return part + ((size_t)(b * P.H + h) * splits + sp) * (P.d + 4);
}

template <int DP, int NW>
__global__ __launch_bounds__(64 * NW, kF32Waves) void paged_f32_kernel(
    const PagedProb P, const float* __restrict__ q, const float* __restrict__ kp,
    const float* __restrict__ vp, float* __restrict__ out, float* __restrict__ lse,
    float* __restrict__ part, int splits, int tiles) {
  __shared__ F32Merge<DP, NW> M;
  const PartOf me(P, splits);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, b = me.b;
  const SeenKeys seen = seen_keys(P, P.klen(b));
  const int t0 = me.sp * tiles, t1 = min(seen.list.n, t0 + tiles);
  if (t0 >= t1 && me.sp > 0) return;
  const int h = me.head(P, min(lane & 15, me.rows - 1));
  f32x4 qf[DP / 16];
#pragma unroll
  for (int j = 0; j < DP / 16; ++j) {
    const int x = 16 * j + 4 * (lane >> 4);
    qf[j] = x < P.d ? load4f(q + b * P.q_sb + h * P.q_sh + x) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const PagedKeys<DP> src{kp + me.hk * P.k_sh, vp + me.hk * P.v_sh, P.table + b * P.table_sb,
                          P, seen, 2 * t0, 2 * (t1 - t0), lane};
  f32_parts<DP, NW, NW>(src, qf, M, w, lane);
  f32_merge(M, w, lane);
  for (int e = threadIdx.x; e < me.rows * P.d; e += 64 * NW) {
    const int r = e / P.d, t = e - r * P.d, hh = me.head(P, r);
    const float x = f32_merged(M, r, t);
    if (splits == 1)
      out[b * P.o_sb + hh * P.o_sh + t] = M.sum[r] != 0.f ? x / M.sum[r] : 0.f;
    else
      part_of(P, part, splits, b, hh, me.sp)[t] = x;
  }
  if (threadIdx.x < me.rows) {
    const int r = threadIdx.x, hh = me.head(P, r);
    if (splits == 1) {
      if (lse) lse[(size_t)b * P.H + hh] = M.sum[r] != 0.f ? M.mx[r] + logf(M.sum[r]) : -INFINITY;
    } else {
      float* p = part_of(P, part, splits, b, hh, me.sp) + P.d;
      p[0] = M.mx[r] * kLog2e;
      p[1] = M.sum[r];
    }
  }
}

// ---- bf16 -------------------------------------------------------------------------------
//
// A wavefront walks its own tiles (every NW-th of the part): keys and values go
// straight to LDS, one tile ahead of the one that is computed, and need no barrier. A
// key's page is looked up two tiles ahead, also through LDS (a load to registers would
// wait for the copies behind it). 16 query heads fill a 16x16x32 product: with
// one head most of it is wasted, but a tile's 16 KB at d = 128 take 3 us of a wavefront's
// share of the memory, its 24 products 0.2.

__device__ __forceinline__ void lds_dma16_at(const void* p, uint32_t lds) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "v"(p), "s"(lds)
      : "memory");
}
__device__ __forceinline__ void lds_dma4_at(const void* p, uint32_t lds) {
  uint32_t saved;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %2\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dword %1, off\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "v"(p), "s"(lds)
      : "memory");
}

template <int D>
constexpr int paged_waves() {
  return D == 64 ? 4 : 2;  // 64 KB of tiles, two workgroups a compute unit
}

template <int D>
__global__ __launch_bounds__(64 * paged_waves<D>(), 1) void paged_bf16_kernel(
    const PagedProb P, const bf16* __restrict__ q, const bf16* __restrict__ kp,
    const bf16* __restrict__ vp, bf16* __restrict__ out, float* __restrict__ lse,
    float* __restrict__ part, int splits, int tiles, float sl2) {
  constexpr int NW = paged_waves<D>(), KK = D / 32, DT = D / 16, RB = 2 * D, TILE = kTile * RB;
  constexpr int NI = TILE / 1024, RPI = 1024 / RB;  // copies of a tile, rows of a copy
  constexpr int OP = D + 4;                         // floats of a row when the wavefronts join
  static_assert(NW * 16 * OP * 4 <= NW * 4 * TILE, "joining fits the tiles");
  __shared__ __attribute__((aligned(1024))) char smem[NW * 4 * TILE];
  __shared__ __attribute__((aligned(256))) int32_t ents[NW][2][64];
  __shared__ __attribute__((aligned(16))) int64_t offs[NW][kTile][2];
  __shared__ float ms[NW][16], ls[NW][16];
  const PartOf me(P, splits);
  const int b = me.b, lane = threadIdx.x & 63, l16 = lane & 15, gr = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const SeenKeys seen = seen_keys(P, P.klen(b));
  const int t0 = me.sp * tiles, t1 = min(seen.list.n, t0 + tiles);
  if (t0 >= t1 && me.sp > 0) return;
  const int nt = t1 > t0 + w ? (t1 - t0 - w + NW - 1) / NW : 0;  // this wavefront's tiles

  bf16x8 qf[KK];
  {
    const bf16* row = q + b * P.q_sb + me.head(P, min(l16, me.rows - 1)) * P.q_sh;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) qf[kk] = *(const bf16x8*)(row + 32 * kk + 8 * gr);
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt = 0: none of these waits lands in the loop
  const int32_t* table = P.table + b * P.table_sb;
  const bf16 *kh = kp + me.hk * P.k_sh, *vh = vp + me.hk * P.v_sh;
  char* mine = smem + w * 4 * TILE;  // K, K, V, V
  const uint32_t lds0 = lds_addr(mine), lds_ents = lds_addr(&ents[w][0][0]);
  auto first_key = [&](int i) __attribute__((always_inline)) {
    return kTile * seen.list.tile(t0 + w + i * NW);
  };
  // the table's entries for the keys of tile i
  auto issue_entries = [&](int i) __attribute__((always_inline)) {
    const int j = nearest_seen(seen.r, first_key(i), lane & 31);
    const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_ents + 256 * (i & 1));
    lds_dma4_at(table + (uint32_t)j / (uint32_t)P.page, dst);
  };
  // copies tile i's rows; returns the mask of its keys that are there
  auto issue_rows = [&](int i) __attribute__((always_inline)) {
    const int j0 = first_key(i), j = nearest_seen(seen.r, j0, lane & 31);
    const int e = ents[w][i & 1][lane];
    const bool there = e >= 0 && e < P.pages;
    const uint32_t any = (uint32_t)__builtin_amdgcn_ballot_w64(there);
    const int in = (int)((uint32_t)j % (uint32_t)P.page);
    int64_t ko = there ? e * P.k_sp + in * P.k_st : 0, vo = there ? e * P.v_sp + in * P.v_st : 0;
    if (any != 0xffffffffu && any != 0) {  // rows that are not there: copies of one that is
      const int src = __builtin_ctz(any);
      const int64_t k1 = __shfl(ko, src, 64), v1 = __shfl(vo, src, 64);
      ko = there ? ko : k1;
      vo = there ? vo : v1;
    }
    if (lane < kTile) {
      offs[w][lane][0] = ko;
      offs[w][lane][1] = vo;
    }
    __builtin_amdgcn_wave_barrier();
    const uint32_t kd = lds0 + (i & 1) * TILE, vd = lds0 + (2 + (i & 1)) * TILE;
#pragma unroll
    for (int c = 0; c < NI; ++c) {
      const int r = c * RPI + lane / (RB / 16);
      const int ch = ((lane % (RB / 16)) ^ row_key<RB>(r)) * 8;
      typedef __attribute__((__vector_size__(2 * sizeof(int64_t)))) int64_t i64x2;
      const i64x2 o = *(const i64x2*)&offs[w][r][0];
      lds_dma16_at(kh + o[0] + ch, __builtin_amdgcn_readfirstlane(kd + 1024 * c));
      lds_dma16_at(vh + o[1] + ch, __builtin_amdgcn_readfirstlane(vd + 1024 * c));
    }
    __builtin_amdgcn_wave_barrier();
    return (uint32_t)__builtin_amdgcn_ballot_w64(there && lane < kTile &&
                                                 sees(seen.r, j0 + (lane & 31)));
  };

  int xoff[KK], coff[DT];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk)
    xoff[kk] = l16 * RB + (((4 * kk + gr) ^ row_key<RB>(l16)) << 4);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    const int r = 4 * gr + (l16 >> 2), lc = 2 * dt + ((l16 & 3) >> 1);
    coff[dt] = r * RB + ((lc ^ row_key<RB>(r)) << 4) + 8 * (l16 & 1);
  }
  f32x4 acc[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) acc[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  auto compute = [&](int i, uint32_t there) __attribute__((always_inline)) {
    if (there == 0) return;
    const char* ks = mine + (i & 1) * TILE;
    const char* vs = mine + (2 + (i & 1)) * TILE;
    f32x4 s[2];
#pragma unroll
    for (int T = 0; T < 2; ++T) {
      s[T] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
        s[T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8*)(ks + 16 * T * RB + xoff[kk]),
                                                       qf[kk], s[T], 0, 0, 0);
    }
    // element r of s[T] is key 16 T + 4 gr + r of the tile
    if (there != 0xffffffffu) {
      const uint32_t x = there >> (4 * gr);
#pragma unroll
      for (int T = 0; T < 2; ++T)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (!((x >> (16 * T + r)) & 1u)) s[T][r] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int T = 0; T < 2; ++T)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[T][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * sl2;
    if (__builtin_amdgcn_ballot_w64(mx > m)) {
      const float m_new = fmaxf(m, mx);
      const float alpha = m_new > m ? __builtin_amdgcn_exp2f(m - m_new) : 1.f;
      l *= alpha;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[dt][r] *= alpha;
      m = m_new;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      p[j] = __builtin_amdgcn_exp2f(fmaf(s[j >> 2][j & 3], sl2, -ref));
      l += p[j];
    }
    const bf16x8 pp = pack8(p);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
      acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          read_cols(vs + coff[dt], vs + 16 * RB + coff[dt]), pp, acc[dt], 0, 0, 0);
  };

  if (nt > 0) {
    issue_entries(0);
    if (nt > 1) issue_entries(1);
    wait_vmcnt<0>();
    uint32_t now = issue_rows(0), next = 0;
    for (int i = 0; i < nt; ++i) {
      wait_lgkm();  // the reads of tile i - 1, whose buffers tile i + 1 takes
      if (i + 2 < nt) issue_entries(i + 2);
      if (i + 1 < nt) {
        next = issue_rows(i + 1);
        wait_vmcnt<2 * NI>();  // all but tile i + 1
      } else {
        wait_vmcnt<0>();
      }
      compute(i, now);
      now = next;
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);

  // join the wavefronts: row r of head r, in the space of the tiles
  float* sums = (float*)smem;
  __syncthreads();
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
    *(f32x4*)&sums[(w * 16 + l16) * OP + 16 * dt + 4 * gr] = acc[dt];
  if (gr == 0) {
    ms[w][l16] = m;
    ls[w][l16] = l;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < me.rows * (D / 4); e += 64 * NW) {
    const int r = e / (D / 4), t = 4 * (e % (D / 4)), hh = me.head(P, r);
    float mx = -INFINITY;
#pragma unroll
    for (int x = 0; x < NW; ++x) mx = fmaxf(mx, ms[x][r]);
    const float ref = mx == -INFINITY ? 0.f : mx;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const float f = __builtin_amdgcn_exp2f(ms[x][r] - ref);
      sum += f * ls[x][r];
      const f32x4 y = *(const f32x4*)&sums[(x * 16 + r) * OP + t];
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] += f * y[c];
    }
    if (splits == 1) {
      const float inv = sum != 0.f ? 1.f / sum : 0.f;
      bf16x4 y;
#pragma unroll
      for (int c = 0; c < 4; ++c) y[c] = f2bf(sum != 0.f ? o[c] * inv : 0.f);
      *(bf16x4*)(out + b * P.o_sb + hh * P.o_sh + t) = y;
      if (lse && t == 0)
        lse[(size_t)b * P.H + hh] =
            sum != 0.f ? (mx + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
    } else {
      float* x = part_of(P, part, splits, b, hh, me.sp);
      *(f32x4*)(x + t) = o;
      if (t == 0) {
        x[D] = ref;
        x[D + 1] = sum;
      }
    }
  }
}

// ---- joining the parts -----------------------------------------------------------------

// One workgroup a head: its wavefronts take every sixteenth part, lanes the dims (a
// few heads of many parts: with four wavefronts joining 128 parts of 16 heads took
// 10 us longer).
template <typename T>
__global__ __launch_bounds__(kJoin) void paged_join_kernel(const PagedProb P,
                                                           const float* __restrict__ part,
                                                           int splits, int tiles,
                                                           T* __restrict__ out,
                                                           float* __restrict__ lse) {
  constexpr int NW = kJoin / 64;
  __shared__ float acc[NW][kMaxD], wsum[NW];
  const int bh = blockIdx.x, b = bh / P.H, h = bh - b * P.H;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int n = (seen_keys(P, P.klen(b)).list.n + tiles - 1) / tiles;  // the sequence's parts
  const float* p = part + (size_t)bh * splits * (P.d + 4);
  const int stride = P.d + 4;
  float mx = -INFINITY;
  for (int i = lane; i < n; i += 64)
    if (p[(size_t)i * stride + P.d + 1] != 0.f) mx = fmaxf(mx, p[(size_t)i * stride + P.d]);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
  const float ref = mx == -INFINITY ? 0.f : mx;
  const int d0 = min(lane, P.d - 1), d1 = min(lane + 64, P.d - 1);
  float sum = 0.f, a0 = 0.f, a1 = 0.f;
#pragma unroll 4
  for (int i = w; i < n; i += NW) {
    const float* r = p + (size_t)i * stride;
    const float s = r[P.d + 1], x0 = r[d0], x1 = r[d1];
    // no key of the part is there: its reference is not one
    const float f = s == 0.f ? 0.f : __builtin_amdgcn_exp2f(r[P.d] - ref);
    sum += f * s;
    a0 += f * x0;
    a1 += f * x1;
  }
  acc[w][lane] = a0;
  acc[w][lane + 64] = a1;
  if (lane == 0) wsum[w] = sum;
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) sum += wsum[i];
  const int t = threadIdx.x;
  if (t < P.d) {
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) x += acc[i][t];
    store_f(out + b * P.o_sb + h * P.o_sh + t, sum != 0.f ? x / sum : 0.f);
  }
  if (lse && t == 0)
    lse[bh] = sum != 0.f ? (ref + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
}

// Parts of the launch's longest possible sequence, and tiles of a part
struct PagedPlan {
  int splits, tiles;
};
PagedPlan paged_plan(const PagedProb& P) {
  const int64_t most = (int64_t)P.max_pages * P.page;
  int64_t seen = most;
  if (P.left < kNoWindow && (int64_t)P.left + 1 + P.sinks < most) seen = (int64_t)P.left + 1 + P.sinks;
  const int64_t all = (seen + kTile - 1) / kTile + 2;  // a window may begin and end inside a tile
  const int64_t wgs = (int64_t)P.B * P.Hk * ((P.G + 15) / 16);
  // Workgroups of the launch if all sequences are as long as can be. Many sequences often
  // have different lengths and balance in smaller parts, fewer pay more for their joining
  // (lengths of 512 to 32,768 at 8 key heads of 128, us with 2,048 and 4,096: 4 sequences 73
  // and 83, 6 71 and 81, 8 114 and 125, 12 152 and 144, 16 194 and 180, 32 175 and 173; equal
  // lengths 2 to 5% more with 4,096; one of 262,144 with 16 heads 203 and 210; at 16 heads of
  // 64 and one of 128 the two are within 3% from 8 sequences on).
  const int parts = P.B >= 12 ? 4096 : 2048;
  int64_t tiles = (all * wgs + parts - 1) / parts;
  // A table can hold far more than the sequences have: 64 tiles at most keep short
  // sequences in wide tables parallel (20 parts of 40,000 keys in a table for a million),
  // up to 65,536 workgroups. (Parts sized on the device by the sum of the lengths, for
  // which every workgroup reads them, were slower: 32 ragged sequences 256 to 299 us.)
  if (tiles > 64) tiles = 64;
  if (tiles < (all * wgs) >> 16) tiles = (all * wgs) >> 16;
  if (tiles < kPartTiles) tiles = kPartTiles;
  if (all <= tiles + 2) return PagedPlan{1, (int)all};
  return PagedPlan{(int)((all + tiles - 1) / tiles), (int)tiles};
}

template <int DP>
hipError_t run_f32(const PagedProb& P, const float* q, const float* kp, const float* vp, float* out,
                   float* lse, float* part, const PagedPlan& pl, hipStream_t st) {
  constexpr int NW = 4;
  hipLaunchKernelGGL((paged_f32_kernel<DP, NW>),
                     dim3((unsigned)((int64_t)pl.splits * ((P.G + 15) / 16) * P.B * P.Hk)),
                     dim3(64 * NW), 0, st, P, q, kp, vp, out, lse, part, pl.splits, pl.tiles);
  return hipGetLastError();
}

template <int D>
hipError_t run_bf16(const PagedProb& P, const bf16* q, const bf16* kp, const bf16* vp, bf16* out,
                    float* lse, float* part, const PagedPlan& pl, hipStream_t st) {
  hipLaunchKernelGGL((paged_bf16_kernel<D>),
                     dim3((unsigned)((int64_t)pl.splits * ((P.G + 15) / 16) * P.B * P.Hk)),
                     dim3(64 * paged_waves<D>()), 0, st, P, q, kp, vp, out, lse, part, pl.splits,
                     pl.tiles, P.scale * kLog2e);
  return hipGetLastError();
}

}  // namespace

size_t paged_bytes(const PagedProb& P) {
  const int s = paged_plan(P).splits;
  return s == 1 ? 0 : ((size_t)P.B * P.H * s * (P.d + 4) * 4 + 255) & ~(size_t)255;
}

hipError_t launch_paged(const PagedProb& P, const void* q, const void* kp, const void* vp, void* out,
                        float* lse, char* ws, hipStream_t st) {
  const PagedPlan pl = paged_plan(P);
  float* part = (float*)ws;
  const dim3 heads(P.B * P.H), threads(kJoin);
  hipError_t e;
  if (P.dtype == CA_BF16) {
    const bf16 *a = (const bf16*)q, *b = (const bf16*)kp, *c = (const bf16*)vp;
    e = P.d == 64 ? run_bf16<64>(P, a, b, c, (bf16*)out, lse, part, pl, st)
                  : run_bf16<128>(P, a, b, c, (bf16*)out, lse, part, pl, st);
    if (e != hipSuccess || pl.splits == 1) return e;
    hipLaunchKernelGGL((paged_join_kernel<bf16>), heads, threads, 0, st, P, part, pl.splits,
                       pl.tiles, (bf16*)out, lse);
  } else {
    const float *a = (const float*)q, *b = (const float*)kp, *c = (const float*)vp;
    e = P.d <= 32   ? run_f32<32>(P, a, b, c, (float*)out, lse, part, pl, st)
        : P.d <= 64 ? run_f32<64>(P, a, b, c, (float*)out, lse, part, pl, st)
                    : run_f32<128>(P, a, b, c, (float*)out, lse, part, pl, st);
    if (e != hipSuccess || pl.splits == 1) return e;
    hipLaunchKernelGGL((paged_join_kernel<float>), heads, threads, 0, st, P, part, pl.splits,
                       pl.tiles, (float*)out, lse);
  }
  return hipGetLastError();
}

}  // namespace ca
