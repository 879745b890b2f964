// Rotary positions of several axes.
//
// Pair p of a head turns by the angle t = position on the pair's axis *
// freq[p]: (x, y) -> (x cos t - y sin t, x sin t + y cos t). The product is
// formed and reduced to [-pi/4, pi/4] in fp64 (at position 10^6 an fp32 angle
// is off by 0.03), sine and cosine of the rest are fp32 Taylor sums.
//
// What bounds it: memory traffic, every query and key read and written once.
// A thread keeps the sines and cosines of its 16 bytes of a token's head and
// takes the same 16 bytes of many heads, so the fp64 work is done once for all
// of them.
#include "seq.h"

namespace ca {

namespace {

constexpr int kRopeThreads = 256;

// sin and cos of |y| <= pi/4 by their series: the first terms left out are
// y^11/11! < 2e-9 and y^12/12! < 2e-10.
__device__ __forceinline__ void sincos_small(float y, float* s, float* c) {
  const float z = y * y;
  float a = fmaf(z, 1.f / 362880.f, -1.f / 5040.f);
  a = fmaf(z, a, 1.f / 120.f);
  a = fmaf(z, a, -1.f / 6.f);
  *s = fmaf(y * z, a, y);
  float b = fmaf(z, -1.f / 3628800.f, 1.f / 40320.f);
  b = fmaf(z, b, -1.f / 720.f);
  b = fmaf(z, b, 1.f / 24.f);
  b = fmaf(z, b, -0.5f);
  *c = fmaf(z, b, 1.f);
}

// sin and cos of pos * freq
__device__ __forceinline__ void sincos_of(int pos, double freq, float* s, float* c) {
  constexpr double kTwoOverPi = 0.63661977236758134308;
  constexpr double kHalfPiHi = 1.57079632679489655800, kHalfPiLo = 6.12323399573676603587e-17;
  const double t = (double)pos * freq;
  const double k = rint(t * kTwoOverPi);
  const double r = fma(-k, kHalfPiLo, fma(-k, kHalfPiHi, t));
  float u, v;
  sincos_small((float)r, &u, &v);
  const int quad = (int)(int64_t)k & 3;
  const float sn = quad & 1 ? v : u, cs = quad & 1 ? u : v;
  *s = quad & 2 ? -sn : sn;
  *c = (quad + 1) & 2 ? -cs : cs;
}

__device__ __forceinline__ int axis_position(const RopeProb& P, int b, int a, int i) {
  if (P.pos) return P.pos[b * P.pos_sb + a * P.pos_sa + i * P.pos_sn];
  return (i / P.inner[a]) % P.grid[a] + P.start[a];
}

template <typename T>
struct Piece {  // 16 bytes
  static constexpr int N = 16 / sizeof(T);
  T x[N];
};

// One thread: piece c of token i of batch b, heads [h0, h1) of the H + Hk.
// Interleaved pairs: piece c is dims N c .. + N - 1, pairs of neighbours.
// Halves: piece c is dims N c .. with their partners npairs later, for the
// npairs / N pieces of the first half; pieces after those are the dims that do
// not turn. In place (out = in) is sound: a thread reads what it writes.
template <typename T, bool HALVES>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(const RopeProb P, const T* q,
                                                            const T* k, T* qo, T* ko, int pieces,
                                                            int per_block) {
  constexpr int N = 16 / sizeof(T);
  constexpr int NP = HALVES ? N : N / 2;  // pairs of a thread
  const int64_t id = (int64_t)blockIdx.x * kRopeThreads + threadIdx.x;
  const int c = (int)(id % pieces);
  const int64_t tok = id / pieces;
  if (tok >= (int64_t)P.B * P.n) return;
  const int b = (int)(tok / P.n), i = (int)(tok - (int64_t)b * P.n);
  const bool turns = !HALVES || c < P.npairs / N;
  // first dim of the piece; its partner's with halves
  const int t0 = HALVES && !turns ? 2 * P.npairs + (c - P.npairs / N) * N : N * c;
  float sn[NP], cs[NP];
#pragma unroll
  for (int j = 0; j < NP; ++j) {
    const int p = HALVES ? t0 + j : t0 / 2 + j;
    sn[j] = 0.f;
    cs[j] = 1.f;
    if (turns && p < P.npairs) {
      int a = 0;
#pragma unroll
      for (int x = 0; x < kMaxAxes - 1; ++x) a += x + 1 < P.axes && p >= P.end[x];
      sincos_of(axis_position(P, b, a, i), P.freq[p], &sn[j], &cs[j]);
      sn[j] *= P.sign;
    }
  }
  const int h0 = blockIdx.y * per_block, h1 = min(h0 + per_block, P.H + P.Hk);
#pragma unroll 4
  for (int h = h0; h < h1; ++h) {
    const bool isq = h < P.H;
    const Lay &Li = isq ? P.lq : P.lk, &Lo = isq ? P.lqo : P.lko;
    const int hh = isq ? h : h - P.H;
    const T* src = (isq ? q : k) + b * Li.sb + hh * Li.sh + i * Li.sn + t0;
    T* dst = (isq ? qo : ko) + b * Lo.sb + hh * Lo.sh + i * Lo.sn + t0;
    Piece<T> u = *(const Piece<T>*)src;
    if constexpr (HALVES) {
      if (turns) {
        Piece<T> w = *(const Piece<T>*)(src + P.npairs);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const float x = to_f(u.x[j]), y = to_f(w.x[j]);
          store_f(&u.x[j], x * cs[j] - y * sn[j]);
          store_f(&w.x[j], x * sn[j] + y * cs[j]);
        }
        *(Piece<T>*)(dst + P.npairs) = w;
      }
    } else {
#pragma unroll
      for (int j = 0; j < NP; ++j) {
        if (t0 / 2 + j >= P.npairs) break;  // dims that do not turn stay as they are
        const float x = to_f(u.x[2 * j]), y = to_f(u.x[2 * j + 1]);
        store_f(&u.x[2 * j], x * cs[j] - y * sn[j]);
        store_f(&u.x[2 * j + 1], x * sn[j] + y * cs[j]);
      }
    }
    *(Piece<T>*)dst = u;
  }
}

// Token t of n new ones of sequence b goes to place lens[b] - n + t of its
// pages. Places before 0 or past the table, and pages outside the pool, are
// left out. One thread per 16 bytes of a head, keys and values.
template <typename T>
__global__ __launch_bounds__(256) void append_kernel(const PagedProb P, const AppendProb A,
                                                     const T* k, const T* v, T* kp, T* vp,
                                                     int pieces) {
  constexpr int N = 16 / sizeof(T);
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int c = (int)(id % pieces);
  const int64_t row = id / pieces;
  const int h = (int)(row % P.Hk);
  const int64_t tok = row / P.Hk;
  if (tok >= (int64_t)P.B * A.n) return;
  const int b = (int)(tok / A.n), t = (int)(tok - (int64_t)b * A.n);
  const int at = P.lens[b] - A.n + t;
  if (at < 0 || at >= (int64_t)P.max_pages * P.page) return;
  const int pg = P.table[b * P.table_sb + at / P.page];
  if (pg < 0 || pg >= P.pages) return;
  const int in = at % P.page;
  *(Piece<T>*)(kp + pg * P.k_sp + in * P.k_st + h * P.k_sh + N * c) =
      *(const Piece<T>*)(k + b * A.k_sb + t * A.k_st + h * A.k_sh + N * c);
  *(Piece<T>*)(vp + pg * P.v_sp + in * P.v_st + h * P.v_sh + N * c) =
      *(const Piece<T>*)(v + b * A.v_sb + t * A.v_st + h * A.v_sh + N * c);
}

}  // namespace

hipError_t launch_rope(const RopeProb& P, const void* q, const void* k, void* qo, void* ko,
                       hipStream_t st) {
  const int N = P.dtype == CA_BF16 ? 8 : 4;
  const int pieces = P.halves ? P.npairs / N + (P.d - 2 * P.npairs) / N : P.d / N;
  const int64_t threads = (int64_t)P.B * P.n * pieces;
  const int64_t blocks = (threads + kRopeThreads - 1) / kRopeThreads;
  const int heads = P.H + P.Hk;
  const int parts = (int)(blocks >= 2048 ? 1 : (2048 + blocks - 1) / blocks);
  const int per_block = (heads + parts - 1) / parts;
  const dim3 grid((unsigned)blocks, (heads + per_block - 1) / per_block);
#define CA_ROPE(T, HALVES)                                                                      \
  hipLaunchKernelGGL((rope_kernel<T, HALVES>), grid, dim3(kRopeThreads), 0, st, P, (const T*)q, \
                     (const T*)k, (T*)qo, (T*)ko, pieces, per_block)
  if (P.dtype == CA_BF16) {
    if (P.halves)
      CA_ROPE(bf16, true);
    else
      CA_ROPE(bf16, false);
  } else {
    if (P.halves)
      CA_ROPE(float, true);
    else
      CA_ROPE(float, false);
  }
#undef CA_ROPE
  return hipGetLastError();
}

hipError_t launch_append(const PagedProb& P, const AppendProb& A, const void* k, const void* v,
                         void* kp, void* vp, hipStream_t st) {
  const int pieces = P.d / (P.dtype == CA_BF16 ? 8 : 4);
  const int64_t threads = (int64_t)P.B * A.n * P.Hk * pieces;
  const dim3 grid((unsigned)((threads + 255) / 256));
  if (P.dtype == CA_BF16)
    hipLaunchKernelGGL((append_kernel<bf16>), grid, dim3(256), 0, st, P, A, (const bf16*)k,
                       (const bf16*)v, (bf16*)kp, (bf16*)vp, pieces);
  else
    hipLaunchKernelGGL((append_kernel<float>), grid, dim3(256), 0, st, P, A, (const float*)k,
                       (const float*)v, (float*)kp, (float*)vp, pieces);
  return hipGetLastError();
}

}  // namespace ca
