// Attention with a sliding window and sinks: forward and backward.
//
// Every kernel walks only the tiles that some row of its block sees
// (visible_tiles), so the work goes with the window, not with the length.
#include <math.h>

#include "f32_tile.h"
#include "seq.h"

namespace ca {

namespace {

// ---- on the fp32 matrix instructions -------------------------------------------------
// 16 rows a workgroup, tiles of 16, operands straight from memory (f32_tile.h).

// transposed operand of 16 rows: dim 16 t + l % 16 of the rows r0 + 4 (l / 16) + r,
// those at or past n as zeros (the rows themselves: f32_load_rows)
template <int DP>
__device__ __forceinline__ void load_cols(const float* base, int64_t sn, int r0, int n, int d,
                                          int lane, f32x4 (&f)[DP / 16]) {
#pragma unroll
  for (int t = 0; t < DP / 16; ++t) {
    const int dim = 16 * t + (lane & 15);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = r0 + 4 * (lane >> 4) + r;
      f[t][r] = dim < d && row < n ? base[row * sn + dim] : 0.f;
    }
  }
}

// Workgroups of a launch: blocks of 16 rows, the first nsink of them cut into psink
// parts of their tiles and the others into p
struct Cut {
  int nb, nsink, psink, p;
  __host__ __device__ int items() const { return nsink * psink + (nb - nsink) * p; }
  __device__ __forceinline__ void at(int v, int* blk, int* part, int* parts) const {
    const int s = nsink * psink;
    const bool sink = v < s;
    *parts = sink ? psink : p;
    *part = (sink ? v : v - s) % *parts;
    *blk = (sink ? 0 : nsink) + (sink ? v : v - s) / *parts;
  }
  // places of partial sums: blocks of one part need none
  __host__ __device__ int sink_places() const { return psink > 1 ? nsink * psink : 0; }
  __host__ __device__ int places() const { return sink_places() + (p > 1 ? (nb - nsink) * p : 0); }
  __device__ __forceinline__ int place(int v) const {  // of a workgroup of a block that is cut
    return v < nsink * psink ? v : sink_places() + v - nsink * psink;
  }
  __device__ __forceinline__ int first_place(int blk) const {  // of its first part
    return blk < nsink ? blk * psink : sink_places() + (blk - nsink) * p;
  }
};

template <int DP>
struct WindowKeys {
  const float *k, *v;
  int64_t k_sn, v_sn;
  TileList list;
  int t0, ntile, lk, d, lane;
  KeyRange r;  // of this lane's query
  float scale;

  __device__ __forceinline__ int key(int t) const { return 16 * list.tile(t0 + t); }
  __device__ __forceinline__ void rows(int t, f32x4 (&f)[DP / 16]) const {
    const int j = min(key(t) + (lane & 15), lk - 1);
    f32_load_rows<DP>(k + j * k_sn, d, lane >> 4, f);
  }
  __device__ __forceinline__ void vals(int t, f32x4 (&f)[DP / 16]) const {
    load_cols<DP>(v, v_sn, key(t), lk, d, lane, f);
  }
  // Values that are infinite or NaN and that one of the tile's queries does not see are
  // set to zero (zero times them is NaN); a query that does see one is marked.
  mutable bool poison;
  __device__ __forceinline__ void mask_vals(int t, f32x4 (&f)[DP / 16]) const {
    const int g = lane >> 4, j0 = key(t) + 4 * g;
    bool all = true, fine = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) all &= sees(r, j0 + i);
    if (__builtin_amdgcn_ballot_w64(!all) == 0) return;
#pragma unroll
    for (int x = 0; x < DP / 16; ++x)
#pragma unroll
      for (int i = 0; i < 4; ++i) fine &= fabsf(f[x][i]) <= 3.402823466e38f;
    if (__builtin_amdgcn_ballot_w64(!fine) == 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bool bad = false;
#pragma unroll
      for (int x = 0; x < DP / 16; ++x) {
        const bool b = !(fabsf(f[x][i]) <= 3.402823466e38f);
        f[x][i] = b ? 0.f : f[x][i];
        bad |= b;
      }
      // any dim of key j0 + i: held by the 16 lanes of group g
      const uint64_t m = __builtin_amdgcn_ballot_w64(bad) >> (16 * g);
      poison |= (m & 0xffffu) != 0 && t < ntile && sees(r, j0 + i);
    }
  }
  __device__ __forceinline__ void logits(int t, f32x4& s) const {
    const int j0 = key(t) + 4 * (lane >> 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = t < ntile && sees(r, j0 + i) ? s[i] * scale : -INFINITY;
  }
};

// Partial results of a row: [B H][nq][parts] of (d sums, reference, sum of exponentials)
template <int DP, int NW>
__global__ __launch_bounds__(64 * NW, kF32Waves) void window_f32_kernel(
    const WinProb P, const float* __restrict__ q, const float* __restrict__ k,
    const float* __restrict__ v, float* __restrict__ out, float* __restrict__ lse,
    float* __restrict__ partial, int parts) {
  __shared__ F32Merge<DP, NW> M;
  const int bh = blockIdx.y, b = bh / P.H, h = bh - b * P.H;
  const int part = blockIdx.x % parts, q0 = 16 * (blockIdx.x / parts);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int lq = P.qlen(b), lk = P.klen(b), off = lk - lq;
  const int rows = min(16, P.nq - q0), real = max(0, min(rows, lq - q0));
  const int bk = b * P.Hk + h / P.G;
  TileList list{0, 0, 0};
  if (real > 0) list = visible_tiles<16>(P.m, q0 + off, q0 + real - 1 + off, lk);
  const int per = (list.n + parts - 1) / parts, t0 = min(list.n, part * per);
  const int i = q0 + min(lane & 15, rows - 1);
  f32x4 qf[DP / 16];
  f32_load_rows<DP>(q + row_off(bh, i, P.lq), P.d, lane >> 4, qf);
  const WindowKeys<DP> src{k + row_off(bk, 0, P.lk), v + row_off(bk, 0, P.lv), P.lk.sn, P.lv.sn,
                           list, t0, min(per, list.n - t0), lk, P.d, lane,
                           visible_keys(P.m, i + off, lk), P.scale, false};
  f32_parts<DP, NW, NW>(src, qf, M, w, lane);
  int poison = src.poison;  // of this wavefront's keys, in the four lanes of a query
  poison |= __shfl_xor(poison, 16, 64);
  poison |= __shfl_xor(poison, 32, 64);
  if (poison)
    for (int t = lane >> 4; t < DP; t += 4) M.o[w][t][lane & 15] = NAN;
  f32_merge(M, w, lane);
  if (parts > 1) {
    for (int e = threadIdx.x; e < rows * P.d; e += 64 * NW) {
      const int r = e / P.d, t = e - r * P.d;
      partial[(((size_t)bh * P.nq + q0 + r) * parts + part) * (P.d + 2) + t] = f32_merged(M, r, t);
    }
    if (threadIdx.x < rows) {
      const int r = threadIdx.x;
      float* x = partial + (((size_t)bh * P.nq + q0 + r) * parts + part) * (P.d + 2) + P.d;
      x[0] = M.mx[r];
      x[1] = M.sum[r];
    }
    return;
  }
  for (int e = threadIdx.x; e < rows * P.d; e += 64 * NW) {
    const int r = e / P.d, t = e - r * P.d;
    const float sum = r < real ? M.sum[r] : 0.f;
    out[row_off(bh, q0 + r, P.lo) + t] = sum != 0.f ? f32_merged(M, r, t) / sum : 0.f;
  }
  if (lse && threadIdx.x < rows) {
    const int r = threadIdx.x;
    lse[(size_t)bh * P.nq + q0 + r] = r < real && M.sum[r] != 0.f ? M.mx[r] + logf(M.sum[r]) : -INFINITY;
  }
}

// Joins a row's parts: one wavefront a row.
__global__ __launch_bounds__(256) void window_join_f32_kernel(const WinProb P,
                                                              const float* __restrict__ partial,
                                                              int parts, float* __restrict__ out,
                                                              float* __restrict__ lse) {
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int bh = (int)(id / P.nq), i = (int)(id - (int64_t)bh * P.nq);
  if (bh >= P.B * P.H) return;
  const float* p = partial + (size_t)id * parts * (P.d + 2);
  float mx = -INFINITY;
  for (int s = 0; s < parts; ++s)
    if (p[s * (P.d + 2) + P.d + 1] != 0.f) mx = fmaxf(mx, p[s * (P.d + 2) + P.d]);
  const int d0 = min(lane, P.d - 1), d1 = min(lane + 64, P.d - 1);
  float sum = 0.f, x0 = 0.f, x1 = 0.f;
  for (int s = 0; s < parts; ++s) {
    const float* r = p + s * (P.d + 2);
    if (r[P.d + 1] == 0.f) continue;  // no key of the part is visible
    const float f = expf(r[P.d] - mx);
    sum += f * r[P.d + 1];
    x0 += f * r[d0];
    x1 += f * r[d1];
  }
  const bool any = i < P.qlen(bh / P.H) && sum != 0.f;
  float* o = out + row_off(bh, i, P.lo);
  if (lane < P.d) o[lane] = any ? x0 / sum : 0.f;
  if (lane + 64 < P.d) o[lane + 64] = any ? x1 / sum : 0.f;
  if (lse && lane == 0) lse[id] = any ? mx + logf(sum) : -INFINITY;
}

// sums the wavefronts' accumulators a (16 rows of d) in LDS and writes row r
template <int DP, int NW, typename Row>
__device__ __forceinline__ void sum_rows(float (*S)[DP][17], const f32x4 (&a)[DP / 16], int w,
                                         int lane, int rows, int d, const Row& row) {
  __syncthreads();
#pragma unroll
  for (int j = 0; j < DP / 16; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) S[w][16 * j + 4 * (lane >> 4) + r][lane & 15] = a[j][r];
  __syncthreads();
  for (int e = threadIdx.x; e < rows * d; e += 64 * NW) {
    const int r = e / d, t = e - r * d;
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) x += S[i][t][r];
    row(r)[t] = x;
  }
}

// dq of 16 queries, and delta = row sums of dout * out. Blocks of one part write dq
// itself, others their place of the partial sums, [heads][places][16][d].
template <int DP, int NW>
__global__ __launch_bounds__(64 * NW, kF32Waves) void window_dq_f32_kernel(
    const WinProb P, const float* __restrict__ q, const float* __restrict__ k,
    const float* __restrict__ v, const float* __restrict__ out, const float* __restrict__ lse,
    const float* __restrict__ dout, float* __restrict__ dq, float* __restrict__ delta,
    float* __restrict__ partial, const Cut cut) {
  constexpr int NJ = DP / 16;
  __shared__ float S[NW][DP][17];
  int blk, part, parts;
  cut.at(blockIdx.x, &blk, &part, &parts);
  const int bh = blockIdx.y, b = bh / P.H, h = bh - b * P.H, q0 = 16 * blk;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, g = lane >> 4;
  const int lq = P.qlen(b), lk = P.klen(b), off = lk - lq;
  const int rows = min(16, P.nq - q0), real = max(0, min(rows, lq - q0));
  const int bk = b * P.Hk + h / P.G;
  TileList list{0, 0, 0};
  if (real > 0) list = visible_tiles<16>(P.m, q0 + off, q0 + real - 1 + off, lk);
  const int per = (list.n + parts - 1) / parts;
  const int i = q0 + min(lane & 15, rows - 1);
  f32x4 qf[NJ], df[NJ], of[NJ], acc[NJ];
  f32_load_rows<DP>(q + row_off(bh, i, P.lq), P.d, g, qf);
  f32_load_rows<DP>(dout + row_off(bh, i, P.ldo), P.d, g, df);
  f32_load_rows<DP>(out + row_off(bh, i, P.lo), P.d, g, of);
  float del = 0.f;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e) del += of[j][e] * df[j][e];
  }
  del += __shfl_xor(del, 16, 64);
  del += __shfl_xor(del, 32, 64);
  if (part == 0 && w == 0 && g == 0 && lane < rows)
    delta[(size_t)bh * P.nq + i] = lane < real ? del : 0.f;
  const KeyRange r = visible_keys(P.m, i + off, lk);
  const float ls = lse[(size_t)bh * P.nq + i];
  const float *kb = k + row_off(bk, 0, P.lk), *vb = v + row_off(bk, 0, P.lv);
  const int t1 = min(list.n, (part + 1) * per);
  for (int t = part * per + w; t < t1; t += NW) {
    const int j0 = 16 * list.tile(t), j = min(j0 + (lane & 15), lk - 1);
    f32x4 kf[NJ], vf[NJ], kt[NJ];
    f32_load_rows<DP>(kb + j * P.lk.sn, P.d, g, kf);
    f32_load_rows<DP>(vb + j * P.lv.sn, P.d, g, vf);
    load_cols<DP>(kb, P.lk.sn, j0, lk, P.d, lane, kt);
    f32x4 s[4], dp[4], ds;
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = dp[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < NJ; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[x][e], qf[x][e], s[e], 0, 0, 0);
        dp[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[x][e], df[x][e], dp[e], 0, 0, 0);
      }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float l = ((s[0][e] + s[1][e]) + (s[2][e] + s[3][e])) * P.scale;
      const float p = (dp[0][e] + dp[1][e]) + (dp[2][e] + dp[3][e]);
      ds[e] = sees(r, j0 + 4 * g + e) ? expf(l - ls) * (p - del) * P.scale : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int x = 0; x < NJ; ++x)
        acc[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(kt[x][e], ds[e], acc[x], 0, 0, 0);
  }
  // rows past the sequence: written as zeros
#pragma unroll
  for (int x = 0; x < NJ; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[x][e] = (lane & 15) < real ? acc[x][e] : 0.f;
  float* place = partial + ((size_t)bh * cut.places() + cut.place(blockIdx.x)) * 16 * P.d;
  sum_rows<DP, NW>(S, acc, w, lane, rows, P.d, [&](int x) {
    return parts > 1 ? place + x * P.d : dq + row_off(bh, q0 + x, P.ldq);
  });
}

// dk and dv of 16 keys of a key head: all queries of its group that see them
template <int DP, int NW>
__global__ __launch_bounds__(64 * NW, (DP == 128 ? 1 : kF32Waves)) void window_dkv_f32_kernel(
    const WinProb P, const float* __restrict__ q, const float* __restrict__ k,
    const float* __restrict__ v, const float* __restrict__ lse, const float* __restrict__ dout,
    const float* __restrict__ delta, float* __restrict__ dk, float* __restrict__ dv,
    float* __restrict__ partial, const Cut cut) {
  constexpr int NJ = DP / 16;
  __shared__ float S[NW][DP][17];
  int blk, part, parts;
  cut.at(blockIdx.x, &blk, &part, &parts);
  const int bk = blockIdx.y, b = bk / P.Hk, hk = bk - b * P.Hk, k0 = 16 * blk;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, g = lane >> 4;
  const int lq = P.qlen(b), lk = P.klen(b), off = lk - lq;
  const int rows = min(16, P.nk - k0), real = max(0, min(rows, lk - k0));
  int i0 = 0, i1 = 0;  // queries that see one of the keys
  if (real > 0) {
    i0 = max(0, seeing_positions(P.m, k0).lo - off);
    const int last = k0 < P.m.sinks ? kUnlimited : seeing_positions(P.m, k0 + real - 1).hi;
    i1 = min(lq, last - off + 1);
  }
  const int j = k0 + min(lane & 15, rows - 1);
  const PosRange see = seeing_positions(P.m, j);
  f32x4 kf[NJ], vf[NJ], ak[NJ], av[NJ];
  f32_load_rows<DP>(k + row_off(bk, j, P.lk), P.d, g, kf);
  f32_load_rows<DP>(v + row_off(bk, j, P.lv), P.d, g, vf);
#pragma unroll
  for (int x = 0; x < NJ; ++x) ak[x] = av[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int first = i0 / 16, nt = i1 > i0 ? (i1 + 15) / 16 - first : 0, all = nt * P.G;
  const int per = (all + parts - 1) / parts, t1 = min(all, (part + 1) * per);
  for (int it = part * per + w; it < t1; it += NW) {
    const int gh = it / nt, q0 = 16 * (first + it - gh * nt), bh = b * P.H + hk * P.G + gh;
    const int i = min(q0 + (lane & 15), lq - 1);
    const float *qb = q + row_off(bh, 0, P.lq), *db = dout + row_off(bh, 0, P.ldo);
    f32x4 qf[NJ], df[NJ], qt[NJ], dt[NJ];
    f32_load_rows<DP>(qb + i * P.lq.sn, P.d, g, qf);
    f32_load_rows<DP>(db + i * P.ldo.sn, P.d, g, df);
    load_cols<DP>(qb, P.lq.sn, q0, lq, P.d, lane, qt);
    load_cols<DP>(db, P.ldo.sn, q0, lq, P.d, lane, dt);
    float ls[4], de[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const size_t at = (size_t)bh * P.nq + min(q0 + 4 * g + e, lq - 1);
      ls[e] = lse[at];
      de[e] = delta[at];
    }
    f32x4 s[4], dp[4], ds, pr;
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = dp[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < NJ; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(qf[x][e], kf[x][e], s[e], 0, 0, 0);
        dp[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(df[x][e], vf[x][e], dp[e], 0, 0, 0);
      }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int ie = q0 + 4 * g + e;
      const float l = ((s[0][e] + s[1][e]) + (s[2][e] + s[3][e])) * P.scale;
      const float p = (dp[0][e] + dp[1][e]) + (dp[2][e] + dp[3][e]);
      const bool on = ie < lq && ie + off >= see.lo && ie + off <= see.hi;
      pr[e] = on ? expf(l - ls[e]) : 0.f;
      ds[e] = on ? pr[e] * (p - de[e]) * P.scale : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int x = 0; x < NJ; ++x) {
        av[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(dt[x][e], pr[e], av[x], 0, 0, 0);
        ak[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(qt[x][e], ds[e], ak[x], 0, 0, 0);
      }
  }
#pragma unroll
  for (int x = 0; x < NJ; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      ak[x][e] = (lane & 15) < real ? ak[x][e] : 0.f;
      av[x][e] = (lane & 15) < real ? av[x][e] : 0.f;
    }
  float* place = partial + ((size_t)bk * cut.places() + cut.place(blockIdx.x)) * 32 * P.d;
  sum_rows<DP, NW>(S, ak, w, lane, rows, P.d, [&](int x) {
    return parts > 1 ? place + x * P.d : dk + row_off(bk, k0 + x, P.ldk);
  });
  sum_rows<DP, NW>(S, av, w, lane, rows, P.d, [&](int x) {
    return parts > 1 ? place + (16 + x) * P.d : dv + row_off(bk, k0 + x, P.ldv);
  });
}

// Adds up the parts of the blocks that were cut, in order: a thread an element. `sets`
// is 1 (dq) or 2 (dk, dv).
__global__ __launch_bounds__(256) void window_sum_f32_kernel(const float* __restrict__ partial,
                                                             const Cut cut, int n, int d, int sets,
                                                             float* __restrict__ a, Lay la,
                                                             float* __restrict__ b, Lay lb) {
  const int blk = blockIdx.x + (cut.psink > 1 ? 0 : cut.nsink), hx = blockIdx.y;
  const int rows = min(16, n - 16 * blk), parts = blk < cut.nsink ? cut.psink : cut.p;
  const float* p = partial + ((size_t)hx * cut.places() + cut.first_place(blk)) * 16 * sets * d;
  const int e = blockIdx.z * 256 + threadIdx.x, set = e / (16 * d), x = e - set * 16 * d;
  const int r = x / d, t = x - r * d;
  if (set >= sets || r >= rows) return;
  float sum = 0.f;
#pragma unroll 4
  for (int i = 0; i < parts; ++i) sum += p[((size_t)i * sets + set) * 16 * d + x];
  (set ? b : a)[row_off(hx, 16 * blk + r, set ? lb : la) + t] = sum;
}

// Wavefronts of a workgroup: eight, four where eight leave too little LDS or registers
template <int DP>
constexpr int f32_waves() {
  return DP == 128 ? 4 : 8;
}
int waves_of(const WinProb& P) { return P.d > 64 ? 4 : 8; }

int clamp(int64_t x, int64_t most) { return (int)(x < 1 ? 1 : x < most ? x : most < 1 ? 1 : most); }

// Parts of the forward pass and of dq: about 1024 workgroups where there are fewer than
// 512, of at least two steps for every wavefront (of one tile in the gradients, TPS in the
// forward pass)
int parts_of(const WinProb& P, int tiles_per_step) {
  const int64_t wgs = (int64_t)((P.nq + 15) / 16) * P.B * P.H;
  if (wgs >= 512) return 1;
  int64_t keys = (int64_t)P.m.left + (P.m.causal ? 0 : P.m.right) + 16 + P.m.sinks;
  if (keys > P.nk) keys = P.nk;
  const int64_t steps = keys / 16 / (tiles_per_step * waves_of(P));
  const int64_t want = (1024 + wgs - 1) / wgs;
  return clamp(want < steps / 2 ? want : steps / 2, 64);
}
int forward_parts(const WinProb& P) { return parts_of(P, P.d > 64 ? 2 : 4); }
Cut query_cut(const WinProb& P) {
  return Cut{(P.nq + 15) / 16, 0, 1, parts_of(P, 1)};
}
// dk and dv: blocks that hold sinks are seen by all queries of the group and cut into
// parts of about the other blocks' tiles, two steps at least
Cut key_cut(const WinProb& P) {
  const int nw = waves_of(P);
  const int64_t all = (int64_t)(P.nq + 15) / 16 * P.G;
  int64_t seen = (((int64_t)P.m.left + (P.m.causal ? 0 : P.m.right) + 16) / 16 + 1) * P.G;
  if (seen > all) seen = all;
  Cut c{(P.nk + 15) / 16, 0, 1, 1};
  const int64_t wgs = (int64_t)c.nb * P.B * P.Hk;
  if (wgs < 512) c.p = clamp((1024 + wgs - 1) / wgs, seen / nw / 2 < 64 ? seen / nw / 2 : 64);
  if (seen < all && P.m.sinks > 0) {
    c.nsink = P.m.sinks < P.nk ? (P.m.sinks + 15) / 16 : c.nb;
    const int64_t each = seen / c.p > 2 * nw ? seen / c.p : 2 * nw;
    const int64_t sinks = (int64_t)c.nsink * P.B * P.Hk;  // 4096 workgroups are enough
    c.psink = clamp((all + each - 1) / each, (4096 + sinks - 1) / sinks < 64 ? (4096 + sinks - 1) / sinks : 64);
  }
  return c;
}

template <int DP>
hipError_t run_f32(const WinProb& P, const float* q, const float* k, const float* v, float* out,
                   float* lse, float* partial, hipStream_t st) {
  constexpr int NW = f32_waves<DP>();
  const int parts = forward_parts(P);
  hipLaunchKernelGGL((window_f32_kernel<DP, NW>), dim3((P.nq + 15) / 16 * parts, P.B * P.H),
                     dim3(64 * NW), 0, st, P, q, k, v, out, lse, partial, parts);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  const int64_t rows = (int64_t)P.B * P.H * P.nq;
  hipLaunchKernelGGL(window_join_f32_kernel, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, P,
                     partial, parts, out, lse);
  return hipGetLastError();
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t delta_bytes(const WinProb& P) { return align256((size_t)P.B * P.H * P.nq * 4); }

template <int DP>
hipError_t run_backward_f32(const WinProb& P, const float* q, const float* k, const float* v,
                            const float* out, const float* lse, const float* dout, float* dq,
                            float* dk, float* dv, char* ws, hipStream_t st) {
  constexpr int NW = f32_waves<DP>();
  float *delta = (float*)ws, *partial = (float*)(ws + delta_bytes(P));
  auto sum = [&](const Cut& c, int heads, int n, int sets, float* a, const Lay& la, float* b,
                 const Lay& lb) {
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || c.places() == 0) return e;
    const int blocks = (c.p > 1 ? c.nb : c.nsink) - (c.psink > 1 ? 0 : c.nsink);
    hipLaunchKernelGGL(window_sum_f32_kernel, dim3(blocks, heads, (16 * sets * P.d + 255) / 256),
                       dim3(256), 0, st, partial, c, n, P.d, sets, a, la, b, lb);
    return hipGetLastError();
  };
  const Cut cq = query_cut(P), ck = key_cut(P);
  hipLaunchKernelGGL((window_dq_f32_kernel<DP, NW>), dim3(cq.items(), P.B * P.H), dim3(64 * NW), 0,
                     st, P, q, k, v, out, lse, dout, dq, delta, partial, cq);
  const hipError_t e = sum(cq, P.B * P.H, P.nq, 1, dq, P.ldq, dq, P.ldq);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((window_dkv_f32_kernel<DP, NW>), dim3(ck.items(), P.B * P.Hk), dim3(64 * NW),
                     0, st, P, q, k, v, lse, dout, delta, dk, dv, partial, ck);
  return sum(ck, P.B * P.Hk, P.nk, 2, dk, P.ldk, dv, P.ldv);
}

}  // namespace

size_t window_bytes(const WinProb& P) {
  if (P.dtype == CA_BF16) return window_bf16_bytes(P);
  const int parts = forward_parts(P);
  return parts == 1 ? 0 : align256((size_t)P.B * P.H * P.nq * parts * (P.d + 2) * 4);
}

hipError_t launch_window(const WinProb& P, const void* q, const void* k, const void* v, void* out,
                         float* lse, char* ws, hipStream_t st) {
  if (P.dtype == CA_BF16) return launch_window_bf16(P, q, k, v, out, lse, ws, st);
#define CA_WINDOW(DP)                                                                            \
  return run_f32<DP>(P, (const float*)q, (const float*)k, (const float*)v, (float*)out, lse,     \
                     (float*)ws, st)
  if (P.d <= 32) CA_WINDOW(32);
  if (P.d <= 64) CA_WINDOW(64);
  CA_WINDOW(128);
#undef CA_WINDOW
}

size_t window_backward_bytes(const WinProb& P) {
  if (P.dtype == CA_BF16) return window_grad_bf16_bytes(P);
  // the partial sums of dq, and after them those of dk and dv, in the same place
  const Cut cq = query_cut(P), ck = key_cut(P);
  const size_t a = (size_t)P.B * P.H * cq.places() * 16 * P.d * 4;
  const size_t b = (size_t)P.B * P.Hk * ck.places() * 32 * P.d * 4;
  return delta_bytes(P) + align256(a > b ? a : b);
}

hipError_t launch_window_backward(const WinProb& P, const void* q, const void* k, const void* v,
                                  const void* out, const float* lse, const void* dout, void* dq,
                                  void* dk, void* dv, char* ws, hipStream_t st) {
  if (P.dtype == CA_BF16)
    return launch_window_grad_bf16(P, q, k, v, out, lse, dout, dq, dk, dv, ws, st);
#define CA_WINDOW(DP)                                                                              \
  return run_backward_f32<DP>(P, (const float*)q, (const float*)k, (const float*)v,                \
                              (const float*)out, lse, (const float*)dout, (float*)dq, (float*)dk,  \
                              (float*)dv, ws, st)
  if (P.d <= 32) CA_WINDOW(32);
  if (P.d <= 64) CA_WINDOW(64);
  CA_WINDOW(128);
#undef CA_WINDOW
}

}  // namespace ca
