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

// this lane's operand of 16 rows: row l % 16, dims 16 j + 4 (l / 16) + e
template <int DP, typename T>
__device__ __forceinline__ void load_rows(const T* row, int d, int g, f32x4 (&f)[DP / 16]) {
#pragma unroll
  for (int j = 0; j < DP / 16; ++j) {
    const int t = 16 * j + 4 * g;
    f[j] = t < d ? load4f(row + t) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
}
// ... and transposed: dim 16 t + l % 16 of the rows r0 + 4 (l / 16) + r, those
// at or past n as zeros
template <int DP, typename T>
__device__ __forceinline__ void load_cols(const T* base, int64_t sn, int r0, int n, int d, int lane,
                                          f32x4 (&f)[DP / 16]) {
#pragma unroll
  for (int t = 0; t < DP / 16; ++t) {
    const int dim = 16 * t + (lane & 15);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = r0 + 4 * (lane >> 4) + r;
      f[t][r] = dim < d && row < n ? to_f(base[row * sn + dim]) : 0.f;
    }
  }
}

template <int DP, typename T>
struct WindowKeys {
  const T *k, *v;
  int64_t k_sn, v_sn;
  TileList list;
  int ntile, lk, d, lane;
  KeyRange r;  // of this lane's query
  float scale;

  __device__ __forceinline__ void rows(int t, f32x4 (&f)[DP / 16]) const {
    const int j = min(16 * list.tile(t) + (lane & 15), lk - 1);
    load_rows<DP>(k + j * k_sn, d, lane >> 4, f);
  }
  __device__ __forceinline__ void vals(int t, f32x4 (&f)[DP / 16]) const {
    load_cols<DP>(v, v_sn, 16 * list.tile(t), lk, d, lane, f);
  }
  __device__ __forceinline__ void mask_vals(int, f32x4 (&)[DP / 16]) const {}
  __device__ __forceinline__ void logits(int t, f32x4& s) const {
    const int j0 = 16 * list.tile(t) + 4 * (lane >> 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = t < ntile && sees(r, j0 + i) ? s[i] * scale : -INFINITY;
  }
};

template <int DP, int NW, typename T>
__global__ __launch_bounds__(64 * NW, kF32Waves) void window_f32_kernel(const WinProb P,
                                                                        const T* __restrict__ q,
                                                                        const T* __restrict__ k,
                                                                        const T* __restrict__ v,
                                                                        T* __restrict__ out,
                                                                        float* __restrict__ lse) {
  __shared__ F32Merge<DP, NW> M;
  const int bh = blockIdx.y, b = bh / P.H, h = bh - b * P.H, q0 = 16 * blockIdx.x;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int lq = P.qlen(b), lk = P.klen(b), off = lk - lq;
  const int rows = min(16, P.nq - q0), real = max(0, min(rows, lq - q0));
  const int bk = b * P.Hk + h / P.G;
  TileList list{0, 0, 0};
  if (real > 0) list = visible_tiles<16>(P.m, q0 + off, q0 + real - 1 + off, lk);
  const int i = q0 + min(lane & 15, rows - 1);
  f32x4 qf[DP / 16];
  load_rows<DP>(q + row_off(bh, i, P.lq), P.d, lane >> 4, qf);
  const WindowKeys<DP, T> src{k + row_off(bk, 0, P.lk), v + row_off(bk, 0, P.lv), P.lk.sn, P.lv.sn,
                              list, list.n, lk, P.d, lane, visible_keys(P.m, i + off, lk), P.scale};
  f32_parts<DP, NW, NW>(src, qf, M, w, lane);
  f32_merge(M, w, lane);
  for (int e = threadIdx.x; e < rows * P.d; e += 64 * NW) {
    const int r = e / P.d, t = e - r * P.d;
    const float sum = r < real ? M.sum[r] : 0.f;
    store_f(out + row_off(bh, q0 + r, P.lo) + t, sum != 0.f ? f32_merged(M, r, t) / sum : 0.f);
  }
  if (lse && threadIdx.x < rows) {
    const int r = threadIdx.x;
    lse[(size_t)bh * P.nq + q0 + r] = r < real && M.sum[r] != 0.f ? M.mx[r] + logf(M.sum[r]) : -INFINITY;
  }
}

// sums the wavefronts' accumulators a (16 rows of d) in LDS and writes row r
template <int DP, int NW, typename T, typename Row>
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
    store_f(row(r) + t, x);
  }
}

// dq of 16 queries, and delta = row sums of dout * out
template <int DP, int NW, typename T>
__global__ __launch_bounds__(64 * NW, kF32Waves) void window_dq_f32_kernel(
    const WinProb P, const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
    const T* __restrict__ out, const float* __restrict__ lse, const T* __restrict__ dout,
    T* __restrict__ dq, float* __restrict__ delta) {
  constexpr int NJ = DP / 16;
  __shared__ float S[NW][DP][17];
  const int bh = blockIdx.y, b = bh / P.H, h = bh - b * P.H, q0 = 16 * blockIdx.x;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, g = lane >> 4;
  const int lq = P.qlen(b), lk = P.klen(b), off = lk - lq;
  const int rows = min(16, P.nq - q0), real = max(0, min(rows, lq - q0));
  const int bk = b * P.Hk + h / P.G;
  TileList list{0, 0, 0};
  if (real > 0) list = visible_tiles<16>(P.m, q0 + off, q0 + real - 1 + off, lk);
  const int i = q0 + min(lane & 15, rows - 1);
  f32x4 qf[NJ], df[NJ], of[NJ], acc[NJ];
  load_rows<DP>(q + row_off(bh, i, P.lq), P.d, g, qf);
  load_rows<DP>(dout + row_off(bh, i, P.ldo), P.d, g, df);
  load_rows<DP>(out + row_off(bh, i, P.lo), P.d, g, of);
  float del = 0.f;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e) del += of[j][e] * df[j][e];
  }
  del += __shfl_xor(del, 16, 64);
  del += __shfl_xor(del, 32, 64);
  if (w == 0 && g == 0 && lane < rows) delta[(size_t)bh * P.nq + i] = lane < real ? del : 0.f;
  const KeyRange r = visible_keys(P.m, i + off, lk);
  const float ls = lse[(size_t)bh * P.nq + i];
  const T *kb = k + row_off(bk, 0, P.lk), *vb = v + row_off(bk, 0, P.lv);
  for (int t = w; t < list.n; t += NW) {
    const int j0 = 16 * list.tile(t), j = min(j0 + (lane & 15), lk - 1);
    f32x4 kf[NJ], vf[NJ], kt[NJ];
    load_rows<DP>(kb + j * P.lk.sn, P.d, g, kf);
    load_rows<DP>(vb + j * P.lv.sn, P.d, g, vf);
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
  sum_rows<DP, NW, T>(S, acc, w, lane, rows, P.d,
                      [&](int x) { return dq + row_off(bh, q0 + x, P.ldq); });
}

// dk and dv of 16 keys of a key head: all queries of its group that see them
template <int DP, int NW, typename T>
__global__ __launch_bounds__(64 * NW, kF32Waves) void window_dkv_f32_kernel(
    const WinProb P, const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
    const float* __restrict__ lse, const T* __restrict__ dout, const float* __restrict__ delta,
    T* __restrict__ dk, T* __restrict__ dv) {
  constexpr int NJ = DP / 16;
  __shared__ float S[NW][DP][17];
  const int bk = blockIdx.y, b = bk / P.Hk, hk = bk - b * P.Hk, k0 = 16 * blockIdx.x;
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
  load_rows<DP>(k + row_off(bk, j, P.lk), P.d, g, kf);
  load_rows<DP>(v + row_off(bk, j, P.lv), P.d, g, vf);
#pragma unroll
  for (int x = 0; x < NJ; ++x) ak[x] = av[x] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int t0 = i0 / 16, nt = max(0, (i1 + 15) / 16 - t0);
  for (int it = w; it < nt * P.G; it += NW) {
    const int gh = it / nt, q0 = 16 * (t0 + it - gh * nt), bh = b * P.H + hk * P.G + gh;
    const int i = min(q0 + (lane & 15), lq - 1);
    const T *qb = q + row_off(bh, 0, P.lq), *db = dout + row_off(bh, 0, P.ldo);
    f32x4 qf[NJ], df[NJ], qt[NJ], dt[NJ];
    load_rows<DP>(qb + i * P.lq.sn, P.d, g, qf);
    load_rows<DP>(db + i * P.ldo.sn, P.d, g, df);
    load_cols<DP>(qb, P.lq.sn, q0, lq, P.d, lane, qt);
    load_cols<DP>(db, P.ldo.sn, q0, lq, P.d, lane, dt);
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
      const int ie = q0 + 4 * g + e, ic = min(ie, lq - 1);
      const float ls = lse[(size_t)bh * P.nq + ic], de = delta[(size_t)bh * P.nq + ic];
      const float l = ((s[0][e] + s[1][e]) + (s[2][e] + s[3][e])) * P.scale;
      const float p = (dp[0][e] + dp[1][e]) + (dp[2][e] + dp[3][e]);
      const bool on = ie < lq && ie + off >= see.lo && ie + off <= see.hi;
      pr[e] = on ? expf(l - ls) : 0.f;
      ds[e] = on ? pr[e] * (p - de) * P.scale : 0.f;
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
  sum_rows<DP, NW, T>(S, ak, w, lane, rows, P.d,
                      [&](int x) { return dk + row_off(bk, k0 + x, P.ldk); });
  sum_rows<DP, NW, T>(S, av, w, lane, rows, P.d,
                      [&](int x) { return dv + row_off(bk, k0 + x, P.ldv); });
}

template <int DP, typename T>
hipError_t run_f32(const WinProb& P, const T* q, const T* k, const T* v, T* out, float* lse,
                   hipStream_t st) {
  constexpr int NW = DP == 128 ? 4 : 8;
  hipLaunchKernelGGL((window_f32_kernel<DP, NW, T>), dim3((P.nq + 15) / 16, P.B * P.H),
                     dim3(64 * NW), 0, st, P, q, k, v, out, lse);
  return hipGetLastError();
}

template <int DP, typename T>
hipError_t run_backward_f32(const WinProb& P, const T* q, const T* k, const T* v, const T* out,
                            const float* lse, const T* dout, T* dq, T* dk, T* dv, float* delta,
                            hipStream_t st) {
  constexpr int NW = 4;
  hipLaunchKernelGGL((window_dq_f32_kernel<DP, NW, T>), dim3((P.nq + 15) / 16, P.B * P.H),
                     dim3(64 * NW), 0, st, P, q, k, v, out, lse, dout, dq, delta);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((window_dkv_f32_kernel<DP, NW, T>), dim3((P.nk + 15) / 16, P.B * P.Hk),
                     dim3(64 * NW), 0, st, P, q, k, v, lse, dout, delta, dk, dv);
  return hipGetLastError();
}

}  // namespace

size_t window_bytes(const WinProb& P) { return P.dtype == CA_BF16 ? window_bf16_bytes(P) : 0; }

hipError_t launch_window(const WinProb& P, const void* q, const void* k, const void* v, void* out,
                         float* lse, char* ws, hipStream_t st) {
  if (P.dtype == CA_BF16) return launch_window_bf16(P, q, k, v, out, lse, ws, st);
#define CA_WINDOW(DP) \
  return run_f32<DP, float>(P, (const float*)q, (const float*)k, (const float*)v, (float*)out, lse, st)
  if (P.d <= 32) CA_WINDOW(32);
  if (P.d <= 64) CA_WINDOW(64);
  CA_WINDOW(128);
#undef CA_WINDOW
}

size_t window_backward_bytes(const WinProb& P) {
  if (P.dtype == CA_BF16) return window_grad_bf16_bytes(P);
  return ((size_t)P.B * P.H * P.nq * 4 + 255) & ~(size_t)255;
}

hipError_t launch_window_backward(const WinProb& P, const void* q, const void* k, const void* v,
                                  const void* out, const float* lse, const void* dout, void* dq,
                                  void* dk, void* dv, char* ws, hipStream_t st) {
  if (P.dtype == CA_BF16)
    return launch_window_grad_bf16(P, q, k, v, out, lse, dout, dq, dk, dv, ws, st);
#define CA_WINDOW(DP)                                                                             \
  return run_backward_f32<DP, float>(P, (const float*)q, (const float*)k, (const float*)v,        \
                                     (const float*)out, lse, (const float*)dout, (float*)dq,      \
                                     (float*)dk, (float*)dv, (float*)ws, st)
  if (P.d <= 32) CA_WINDOW(32);
  if (P.d <= 64) CA_WINDOW(64);
  CA_WINDOW(128);
#undef CA_WINDOW
}

}  // namespace ca
