// Attention of packed chunks of new tokens over a paged key-value cache.
//
// One workgroup per (token, head). Its wavefronts take every fourth group of 64
// keys, a lane a key: the logits of a group, an online softmax, and the value
// product with a lane for one or two dims. The wavefronts' states are joined
// through LDS.
#include <math.h>

#include "seq.h"

namespace ca {

namespace {

// The sequence whose new tokens hold packed row t; -1 if none does
__device__ __forceinline__ int seq_of(const ChunkProb& P, int t) {
  if (t < P.start(0) || t >= P.start(P.B)) return -1;
  int lo = 0, hi = P.B;  // start(lo) <= t < start(hi)
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (P.start(mid) <= t)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

template <typename T>
__global__ __launch_bounds__(256) void chunk_kernel(const ChunkProb P, const T* __restrict__ q,
                                                    const T* __restrict__ kp,
                                                    const T* __restrict__ vp, T* __restrict__ out,
                                                    float* __restrict__ lse) {
  __shared__ float qs[kMaxD], prob[4][64], o[4][kMaxD], ms[4], ls[4];
  __shared__ int64_t at[4][64];
  const int t = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int b = seq_of(P, t);
  if (b < 0) return;
  const int s0 = P.start(b), lq = P.start(b + 1) - s0, lk = P.klen(b), hk = h / P.G;
  const KeyRange r = visible_keys(P.m, t - s0 + lk - lq, lk);
  for (int i = tid; i < P.d; i += 256) qs[i] = to_f(q[t * P.q_st + h * P.q_sh + i]);
  __syncthreads();
  float m = -INFINITY, l = 0.f, acc[2] = {0.f, 0.f};
  for (int j0 = 64 * w; j0 < lk; j0 += 256) {
    const int j = j0 + lane;
    float s = -INFINITY;
    int64_t va = -1;
    if (j < lk && sees(r, j)) {
      const int e = P.table[b * P.table_sb + j / P.page], in = j % P.page;
      if (e >= 0 && e < P.pages) {
        const T* row = kp + e * P.k_sp + in * P.k_st + hk * P.k_sh;
        s = 0.f;
        for (int x = 0; x < P.d; x += 4) {
          const f32x4 y = load4f(row + x);
#pragma unroll
          for (int c = 0; c < 4; ++c) s = fmaf(y[c], qs[x + c], s);
        }
        s *= P.scale;
        va = e * P.v_sp + in * P.v_st + hk * P.v_sh;
      }
    }
    float mx = s;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) mx = fmaxf(mx, __shfl_xor(mx, x, 64));
    const float m_new = fmaxf(m, mx);
    if (m_new == -INFINITY) continue;
    const float al = expf(m - m_new), p = expf(s - m_new);
    float sum = p;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x, 64);
    l = l * al + sum;
    m = m_new;
    acc[0] *= al;
    acc[1] *= al;
    prob[w][lane] = p;
    at[w][lane] = va;
    __builtin_amdgcn_wave_barrier();
    for (int i = 0; i < 64; ++i) {
      const int64_t a = at[w][i];
      if (a < 0) continue;
      const float x = prob[w][i];
      if (lane < P.d) acc[0] = fmaf(x, to_f(vp[a + lane]), acc[0]);
      if (lane + 64 < P.d) acc[1] = fmaf(x, to_f(vp[a + lane + 64]), acc[1]);
    }
    __builtin_amdgcn_wave_barrier();
  }
  o[w][lane] = acc[0];
  o[w][lane + 64] = acc[1];
  if (lane == 0) {
    ms[w] = m;
    ls[w] = l;
  }
  __syncthreads();
  float mx = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
  if (mx == -INFINITY) mx = 0.f;
  float sum = 0.f, f[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    f[x] = expf(ms[x] - mx);
    sum += f[x] * ls[x];
  }
  for (int i = tid; i < P.d; i += 256) {
    const float x = f[0] * o[0][i] + f[1] * o[1][i] + f[2] * o[2][i] + f[3] * o[3][i];
    store_f(out + t * P.o_st + h * P.o_sh + i, sum != 0.f ? x / sum : 0.f);
  }
  if (lse && tid == 0) lse[(size_t)t * P.H + h] = sum != 0.f ? mx + logf(sum) : -INFINITY;
}

}  // namespace

size_t chunk_bytes(const ChunkProb& P) { return 0; }

hipError_t launch_chunk(const ChunkProb& P, const void* q, const void* kp, const void* vp, void* out,
                        float* lse, char* ws, hipStream_t st) {
  const dim3 grid(P.tokens, P.H);
  if (P.dtype == CA_BF16)
    hipLaunchKernelGGL((chunk_kernel<bf16>), grid, dim3(256), 0, st, P, (const bf16*)q,
                       (const bf16*)kp, (const bf16*)vp, (bf16*)out, lse);
  else
    hipLaunchKernelGGL((chunk_kernel<float>), grid, dim3(256), 0, st, P, (const float*)q,
                       (const float*)kp, (const float*)vp, (float*)out, lse);
  return hipGetLastError();
}

}  // namespace ca
