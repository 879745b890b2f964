// Attention with a sliding window and sinks, bf16, on the matrix cores.
//
// One workgroup per (head, 128 queries), which walks the 64-key tiles that one of its
// rows sees (walk_bf16.h).
#include <math.h>

#include "seq.h"
#include "walk_bf16.h"

namespace ca {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kRows = kWalkRows;

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

// Tiles of keys and values whose rows lie `stride` apart
template <int D>
struct DenseTiles : WalkRows {
  static constexpr bool kHoles = false, kBegun = false;
  static constexpr float kMostSum = 0x1p22f;
  static constexpr int NW = 4, RB = 2 * D, TILE = KT * RB;
  const bf16 *kbase, *vbase;
  int64_t ksn, vsn;
  RowCopy<RB, KT, NW> kcopy, vcopy;
  uint32_t lds0;
  int w, lane;
  __device__ __forceinline__ void issue_k(int t, int buf) const {
    const int k0 = KT * tile(t);
    kcopy.issue(kbase + (int64_t)k0 * ksn, lds0 + buf * TILE, w, lane, lk - 1 - k0);
  }
  __device__ __forceinline__ void issue_v(int t, int buf) const {
    const int k0 = KT * tile(t);
    vcopy.issue(vbase + (int64_t)k0 * vsn, lds0 + (2 + buf) * TILE, w, lane, lk - 1 - k0);
  }
  __device__ __forceinline__ void first_k() const { issue_k(t0, 0); }
  __device__ __forceinline__ void issue_both(int t) const {
    issue_k(t, 0);
    issue_v(t, 0);
  }
};

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
  __builtin_amdgcn_s_waitcnt(kWalkVmcnt0);
  if (tid == 0) redo = 0;  // ordered before any write by the barriers of the tiles

  const DenseTiles<D> T{
      {P.m, list, t0, t1, lk, ra, rz, i + off, wreal, q0 + off, q0 + real - 1 + off},
      k + row_off(bk, 0, P.lk),
      v + row_off(bk, 0, P.lv),
      P.lk.sn,
      P.lv.sn,
      RowCopy<RB, KT, NW>(w, lane, (uint32_t)(P.lk.sn * 2)),
      RowCopy<RB, KT, NW>(w, lane, (uint32_t)(P.lv.sn * 2)),
      lds_addr(smem),
      w,
      lane};
  f32x16 oacc[DT];
  float m, l_tot;
  walk_bf16<D>(T, smem, &redo, qreg, sl2, w, lane, oacc, m, l_tot);
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
