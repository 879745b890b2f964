// Attention of one new token of each sequence over a paged key-value cache.
//
// The keys that a sequence's token sees (the sinks, then its window) are cut
// into parts of equal size, one workgroup each per key head, so that a few
// long sequences fill the chip too; the parts' softmax states are joined by a
// second launch. All query heads of a key head share its keys. What bounds it:
// the cache, read once.
#include <math.h>

#include "f32_tile.h"
#include "seq.h"

namespace ca {

namespace {

// the keys that the token of sequence b sees, numbered 0 .. n - 1: the sinks
// [0, ns), then the window from key lo
struct SeenKeys {
  int ns, lo, n;
  __device__ __forceinline__ int key(int s) const { return s < ns ? s : lo + s - ns; }
};
__device__ __forceinline__ SeenKeys seen_keys(const PagedProb& P, int b) {
  const int len = P.klen(b);
  const int lo = max(0, len - 1 - P.left);
  SeenKeys s;
  s.ns = min(P.sinks, lo);
  s.lo = lo;
  s.n = s.ns + len - lo;
  return s;
}

template <int DP, typename T>
struct PagedKeys {
  const T *k, *v;  // of this key head
  const int32_t* table;
  const PagedProb* P;
  SeenKeys seen;
  int s0, n, ntile, lane;  // keys s0 .. n - 1 of the seen ones

  // page and place of seen key s; -1 where there is none
  __device__ __forceinline__ int place(int s, int& in) const {
    if (s >= n) return -1;
    const int j = seen.key(s);
    const int e = j / P->page;
    in = j - e * P->page;
    const int pg = table[e];
    return pg < P->pages ? pg : -1;
  }
  __device__ __forceinline__ void rows(int t, f32x4 (&f)[DP / 16]) const {
    int in = 0;
    const int pg = place(s0 + 16 * t + (lane & 15), in);
#pragma unroll
    for (int j = 0; j < DP / 16; ++j) {
      const int x = 16 * j + 4 * (lane >> 4);
      f[j] = pg >= 0 && x < P->d ? load4f(k + pg * P->k_sp + in * P->k_st + x)
                                 : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  __device__ __forceinline__ void vals(int t, f32x4 (&f)[DP / 16]) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      int in = 0;
      const int pg = place(s0 + 16 * t + 4 * (lane >> 4) + r, in);
#pragma unroll
      for (int x = 0; x < DP / 16; ++x) {
        const int dim = 16 * x + (lane & 15);
        f[x][r] = pg >= 0 && dim < P->d ? to_f(v[pg * P->v_sp + in * P->v_st + dim]) : 0.f;
      }
    }
  }
  __device__ __forceinline__ void mask_vals(int, f32x4 (&)[DP / 16]) const {}
  __device__ __forceinline__ void logits(int t, f32x4& s) const {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      int in = 0;
      s[r] = place(s0 + 16 * t + 4 * (lane >> 4) + r, in) >= 0 ? s[r] * P->scale : -INFINITY;
    }
  }
};

// keys of a part: an equal share in whole tiles of 64, so that parts and tiles
// do not depend on the launch's other sequences
__device__ __forceinline__ int part_keys(int n, int splits) {
  return ((n + splits - 1) / splits + 63) / 64 * 64;
}

// Part results: [B Hk][splits][G] of (d sums, reference, sum of exponentials)
template <int DP, int NW, typename T>
__global__ __launch_bounds__(64 * NW, kF32Waves) void paged_f32_kernel(
    const PagedProb P, const T* __restrict__ q, const T* __restrict__ kp, const T* __restrict__ vp,
    T* __restrict__ out, float* __restrict__ lse, float* __restrict__ part, int splits) {
  __shared__ F32Merge<DP, NW> M;
  const int qt = (P.G + 15) / 16;
  const int sp = blockIdx.x / qt, g0 = 16 * (blockIdx.x % qt), bk = blockIdx.y;
  const int b = bk / P.Hk, hk = bk - b * P.Hk;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int rows = min(16, P.G - g0);
  const int h = hk * P.G + g0 + min(lane & 15, rows - 1);
  f32x4 qf[DP / 16];
#pragma unroll
  for (int j = 0; j < DP / 16; ++j) {
    const int x = 16 * j + 4 * (lane >> 4);
    qf[j] = x < P.d ? load4f(q + b * P.q_sb + h * P.q_sh + x) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const SeenKeys seen = seen_keys(P, b);
  const int per = part_keys(seen.n, splits), s0 = min(seen.n, sp * per), n = min(seen.n, s0 + per);
  const PagedKeys<DP, T> src{kp + hk * P.k_sh, vp + hk * P.v_sh, P.table + b * P.table_sb,
                             &P, seen, s0, n, (n - s0 + 15) / 16, lane};
  f32_parts<DP, NW, NW>(src, qf, M, w, lane);
  f32_merge(M, w, lane);
  for (int e = threadIdx.x; e < rows * P.d; e += 64 * NW) {
    const int r = e / P.d, t = e - r * P.d, hh = hk * P.G + g0 + r;
    const float x = f32_merged(M, r, t);
    if (splits == 1)
      store_f(out + b * P.o_sb + hh * P.o_sh + t, M.sum[r] != 0.f ? x / M.sum[r] : 0.f);
    else
      part[((size_t)(b * P.H + hh) * splits + sp) * (P.d + 2) + t] = x;
  }
  if (threadIdx.x < rows) {
    const int r = threadIdx.x, hh = hk * P.G + g0 + r;
    if (splits == 1) {
      if (lse) lse[(size_t)b * P.H + hh] = M.sum[r] != 0.f ? M.mx[r] + logf(M.sum[r]) : -INFINITY;
    } else {
      float* p = part + ((size_t)(b * P.H + hh) * splits + sp) * (P.d + 2) + P.d;
      p[0] = M.mx[r];
      p[1] = M.sum[r];
    }
  }
}

// Joins the parts of a head: one wavefront each.
template <typename T>
__global__ __launch_bounds__(64) void paged_join_kernel(const PagedProb P,
                                                        const float* __restrict__ part, int splits,
                                                        T* __restrict__ out,
                                                        float* __restrict__ lse) {
  const int bh = blockIdx.x, b = bh / P.H, h = bh - b * P.H, lane = threadIdx.x;
  const float* p = part + (size_t)bh * splits * (P.d + 2);
  float mx = -INFINITY;
  for (int i = lane; i < splits; i += 64)
    if (p[(size_t)i * (P.d + 2) + P.d + 1] != 0.f) mx = fmaxf(mx, p[(size_t)i * (P.d + 2) + P.d]);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
  float sum = 0.f, a0 = 0.f, a1 = 0.f;
  for (int i = 0; i < splits; ++i) {
    const float* r = p + (size_t)i * (P.d + 2);
    if (r[P.d + 1] == 0.f) continue;  // no key
    const float f = expf(r[P.d] - mx);
    sum += f * r[P.d + 1];
    if (lane < P.d) a0 += f * r[lane];
    if (lane + 64 < P.d) a1 += f * r[lane + 64];
  }
  T* o = out + b * P.o_sb + h * P.o_sh;
  const float inv = sum != 0.f ? 1.f / sum : 0.f;
  if (lane < P.d) store_f(o + lane, a0 * inv);
  if (lane + 64 < P.d) store_f(o + lane + 64, a1 * inv);
  if (lse && lane == 0) lse[bh] = sum != 0.f ? mx + logf(sum) : -INFINITY;
}

template <int DP, typename T>
hipError_t run_paged(const PagedProb& P, const T* q, const T* kp, const T* vp, T* out, float* lse,
                     float* part, hipStream_t st) {
  constexpr int NW = 4;
  const int splits = paged_splits(P);
  hipLaunchKernelGGL((paged_f32_kernel<DP, NW, T>), dim3(splits * ((P.G + 15) / 16), P.B * P.Hk),
                     dim3(64 * NW), 0, st, P, q, kp, vp, out, lse, part, splits);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  hipLaunchKernelGGL((paged_join_kernel<T>), dim3(P.B * P.H), dim3(64), 0, st, P, part, splits, out,
                     lse);
  return hipGetLastError();
}

}  // namespace

int paged_splits(const PagedProb& P) {
  const int64_t most = (int64_t)P.max_pages * P.page;
  const int64_t seen = P.left < kNoWindow ? min(most, (int64_t)P.left + 1 + P.sinks) : most;
  const int64_t wgs = (int64_t)P.B * P.Hk * ((P.G + 15) / 16);
  const int64_t want = (1024 + wgs - 1) / wgs, room = (seen + 255) / 256;
  const int64_t s = want < room ? want : room;
  return (int)(s < 1 ? 1 : s);
}

size_t paged_bytes(const PagedProb& P) {
  const int s = paged_splits(P);
  return s == 1 ? 0 : ((size_t)P.B * P.H * s * (P.d + 2) * 4 + 255) & ~(size_t)255;
}

hipError_t launch_paged(const PagedProb& P, const void* q, const void* kp, const void* vp, void* out,
                        float* lse, char* ws, hipStream_t st) {
#define CA_PAGED(DP, T)                                                                          \
  return run_paged<DP, T>(P, (const T*)q, (const T*)kp, (const T*)vp, (T*)out, lse, (float*)ws, st)
  if (P.dtype == CA_BF16) {
    if (P.d == 64) CA_PAGED(64, bf16);
    CA_PAGED(128, bf16);
  }
  if (P.d <= 32) CA_PAGED(32, float);
  if (P.d <= 64) CA_PAGED(64, float);
  CA_PAGED(128, float);
#undef CA_PAGED
}

}  // namespace ca
