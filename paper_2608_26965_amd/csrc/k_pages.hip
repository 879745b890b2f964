// Page tables and slot maps from the sequences' lengths, pages given back, and
// new keys and values written by the slot map.
//
// What bounds them: latency. A step's tables are a few kilobytes; the launches and
// the chains of dependent loads (length, entry, free page) are what takes time.
// 256 sequences of up to 32,768 tokens grow by a token and give pages back in 12 us
// on the device, 64 that grow by up to 4,096 each in 18. The writes of keys and values are
// bound by memory traffic, each read and written once (32,760 rows of 40 heads of 128: 246 us,
// 5.45 TB/s; a plain copy of 2 GiB reaches 6.3).
#include "seq.h"

namespace ca {

namespace {

// Steps of so few tokens and sequences: the growing workgroup, of four wavefronts, writes the
// slots too. Growing and giving back on the device, against the larger workgroup and a launch
// for the slots: 16 sequences, 64 tokens 9.2 and 13.9 us; 256 sequences, 2,048 tokens 13.0 and
// 15.9, 4,096 tokens 19.4 and 17.4; 2,048 tokens of 700 sequences 16.7 and 17.6, of 2,000 30.9
// and 27.3.
constexpr int kFewTokens = 2048, kFewSequences = 256;

// Sum of x over the threads before this one, and over all of them (NW wavefronts)
template <int NW, typename T>
__device__ __forceinline__ T scan_before(T x, T (&sums)[NW], T* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  T in = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const T y = __shfl_up(in, o, 64);
    if (lane >= o) in += y;
  }
  __syncthreads();  // the sums of a scan before are read
  if (lane == 63) sums[w] = in;
  __syncthreads();
  T before = 0, all = 0;
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    if (i < w) before += sums[i];
    all += sums[i];
  }
  *total = all;
  return before + in - x;
}

// New tokens of sequence b, its last n of len
struct NewTokens {
  int len, n;
  __device__ __forceinline__ NewTokens(int l, int m) : len(l), n(m) {}
  __device__ __forceinline__ NewTokens(const PagesProb& P, const int32_t* n_new, int b) {
    len = P.len(b);
    n = min(max(n_new[b], 0), len);
  }
};

// Slot and position of the i-th new token of a sequence
__device__ __forceinline__ void place_token(const PagesProb& P, const NewTokens& s, int b, int i,
                                            int t, int64_t* slots, int32_t* positions) {
  const int pos = s.len - s.n + i, entry = pos / P.page, e = P.table[b * P.table_sb + entry];
  slots[t] = e >= 0 && e < P.pages ? (int64_t)e * P.page + (pos - entry * P.page) : -1;
  positions[t] = pos;
}

// The last place of ascending list[0 .. N - 1] that holds at most i
template <int N, typename T>
__device__ __forceinline__ int find_in(const T* list, T i) {
  int lo = 0;
#pragma unroll
  for (int step = N / 2; step > 0; step >>= 1)
    if (list[lo + step] <= i) lo += step;
  return lo;
}

// One workgroup: starts, and pages for the entries that lack one. N sequences are taken
// at a time, the entries that their new tokens lie on one after the other, thread by
// thread; ballots say how many of the entries before lack a page. With SLOTS also the
// slots of those sequences' tokens (few tokens: one launch less).
template <int N, bool SLOTS>
__global__ __launch_bounds__(N) void grow_kernel(const PagesProb P, const int32_t* n_new,
                                                 int32_t* starts, int64_t* slots,
                                                 int32_t* positions, int32_t* seen) {
  constexpr int NW = N / 64, kItems = N > 256 ? 8 : 4;  // entries that a thread looks at in one go
  __shared__ int64_t first_item[N];  // entries of the sequences before
  __shared__ int64_t first_token[N];
  __shared__ int32_t s_len[N], s_new[N];
  __shared__ int64_t sums[NW];
  __shared__ int32_t counts[kItems][NW];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int n_free = min(max(P.state[0], 0), P.pages);
  int64_t tokens = 0, taken = 0;
  for (int b0 = 0; b0 < P.B; b0 += N) {
    const int b = b0 + tid;
    int n = 0, entries = 0;
    s_len[tid] = s_new[tid] = 0;
    if (b < P.B) {
      const NewTokens s(P, n_new, b);
      s_len[tid] = s.len;
      s_new[tid] = n = s.n;
      entries = n > 0 ? (s.len - 1) / P.page - (s.len - n) / P.page + 1 : 0;
    }
    int64_t total, items;
    const int64_t before = tokens + scan_before<NW, int64_t>(n, sums, &total);
    const int64_t item0 = scan_before<NW, int64_t>(entries, sums, &items);
    if (b < P.B) {
      starts[b] = (int32_t)min(before, (int64_t)P.tokens);
      // (the first of its new tokens have the rows that there are)
      if (seen) seen[b] = s_len[tid] - n + (int)min(max(P.tokens - before, (int64_t)0), (int64_t)n);
    }
    first_item[tid] = item0;
    first_token[tid] = before;
    __syncthreads();
    for (int64_t i0 = 0; i0 < items; i0 += N * kItems) {
      int64_t at[kItems];
      int lack = 0;
#pragma unroll
      for (int r = 0; r < kItems; ++r) {
        const int64_t i = i0 + r * N + tid;
        at[r] = 0;
        if (i < items) {
          const int x = find_in<N, int64_t>(first_item, i);
          at[r] = (b0 + x) * P.table_sb + (s_len[x] - s_new[x]) / P.page + (i - first_item[x]);
        }
      }
      int e[kItems];
#pragma unroll
      for (int r = 0; r < kItems; ++r) e[r] = i0 + r * N + tid < items ? P.table[at[r]] : 0;
#pragma unroll
      for (int r = 0; r < kItems; ++r) {
        const bool l = e[r] < 0 || e[r] >= P.pages;
        const uint64_t who = __ballot(l);
        if (lane == 0) counts[r][w] = __popcll(who);
        if (l) lack |= 1 << r;
      }
      __syncthreads();
      int64_t rank = taken;
#pragma unroll
      for (int r = 0; r < kItems; ++r) {
        const bool l = (lack >> r) & 1;
        const uint64_t who = __ballot(l);
        int before_me = 0, all = 0;
#pragma unroll
        for (int x = 0; x < NW; ++x) {
          if (x < w) before_me += counts[r][x];
          all += counts[r][x];
        }
        if (l) {
          const int64_t k = rank + before_me + __popcll(who & ((1ull << lane) - 1));
          if (k < n_free) P.table[at[r]] = P.free[n_free - 1 - k];
        }
        rank += all;
      }
      taken = rank;
      __syncthreads();  // the counts are read
    }
    if constexpr (SLOTS) {
      const int end = (int)min(tokens + total, (int64_t)P.tokens);
      for (int t = (int)min(tokens, (int64_t)P.tokens) + tid; t < end; t += N) {
        const int x = find_in<N, int64_t>(first_token, (int64_t)t);
        place_token(P, NewTokens{s_len[x], s_new[x]}, b0 + x, (int)(t - first_token[x]), t, slots,
                    positions);
      }
    }
    tokens += total;
    __syncthreads();  // the lists are read
  }
  if (tid == 0) {
    starts[P.B] = (int32_t)min(tokens, (int64_t)P.tokens);
    P.state[0] = (int32_t)max(n_free - taken, (int64_t)0);
    P.state[1] = (int32_t)min(max(taken - n_free, (int64_t)0), (int64_t)INT32_MAX);
    P.state[2] = (int32_t)min(max(tokens - P.tokens, (int64_t)0), (int64_t)INT32_MAX);
  }
  if constexpr (SLOTS)
    for (int t = (int)min(tokens, (int64_t)P.tokens) + tid; t < P.tokens; t += N) {
      slots[t] = -1;
      positions[t] = 0;
    }
}

__global__ __launch_bounds__(256) void slots_kernel(const PagesProb P,
                                                    const int32_t* __restrict__ n_new,
                                                    const int32_t* __restrict__ starts,
                                                    int64_t* __restrict__ slots,
                                                    int32_t* __restrict__ positions) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= P.tokens) return;
  if (t >= starts[P.B]) {
    slots[t] = -1;
    positions[t] = 0;
    return;
  }
  int lo = 0, hi = P.B;  // starts[lo] <= t < starts[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (starts[mid] <= t)
      lo = mid;
    else
      hi = mid;
  }
  place_token(P, NewTokens(P, n_new, lo), lo, t - starts[lo], t, slots, positions);
}

// Whether entry i of a sequence of n tokens holds a page that goes back
__device__ __forceinline__ bool goes_back(const PagesProb& P, int n, int i, int e) {
  const int first = i * P.page, last = min(first + P.page, n) - 1;
  const bool keep = first < n && (P.left == kNoWindow || first < P.sinks || last >= n - P.left);
  return !keep && e >= 0 && e < P.pages;
}

// What a row's first launch leaves for the second one
struct RowBack {
  int count, first, end;  // pages that go back, and the entries that hold them
};

// rows[b]: of row b; rows[B].count: the free pages before
__global__ __launch_bounds__(256) void release_count_kernel(const PagesProb P, RowBack* rows) {
  __shared__ int32_t part[4][3];
  const int b = blockIdx.x, n = P.len(b), lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int count = 0, first = INT32_MAX, end = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < P.max_pages; i += 256)
    if (goes_back(P, n, i, P.table[b * P.table_sb + i])) {
      ++count;
      first = min(first, i);
      end = i + 1;
    }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    count += __shfl_xor(count, o, 64);
    first = min(first, __shfl_xor(first, o, 64));
    end = max(end, __shfl_xor(end, o, 64));
  }
  if (lane == 0) {
    part[w][0] = count;
    part[w][1] = first;
    part[w][2] = end;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int x = 1; x < 4; ++x) {
      count += part[x][0];
      first = min(first, part[x][1]);
      end = max(end, part[x][2]);
    }
    rows[b] = RowBack{count, first, end};
    if (b == 0) rows[P.B].count = min(max(P.state[0], 0), P.pages);
  }
}

__global__ __launch_bounds__(256) void release_kernel(const PagesProb P,
                                                      const RowBack* __restrict__ rows) {
  __shared__ int64_t sums[4];
  __shared__ int32_t each[2][4];
  const int b = blockIdx.x, n = P.len(b), tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const RowBack mine = rows[b];
  if (mine.count == 0 && b != 0) return;
  const int n_free = rows[P.B].count;
  // pages of the rows from this one on; the stack ends with row 0's first
  int64_t after = 0, total;
  for (int x = b + tid; x < P.B; x += 256) after += rows[x].count;
  scan_before<4, int64_t>(after, sums, &total);
  if (b == 0 && tid == 0) P.state[0] = (int32_t)min((int64_t)n_free + total, (int64_t)P.pages);
  int64_t top = n_free + total - 1;  // place of the row's next page
  int turn = 0;
  for (int i0 = mine.first; i0 < mine.end; i0 += 256, turn ^= 1) {
    const int i = i0 + tid;
    int e = -1;
    if (i < mine.end) e = P.table[b * P.table_sb + i];
    const bool back = i < mine.end && goes_back(P, n, i, e);
    const uint64_t who = __ballot(back);
    if (lane == 0) each[turn][w] = __popcll(who);
    __syncthreads();  // (those of two turns before are read)
    int before = 0, all = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (x < w) before += each[turn][x];
      all += each[turn][x];
    }
    if (back) {
      const int64_t at = top - before - __popcll(who & ((1ull << lane) - 1));
      if (at >= 0 && at < P.pages) P.free[at] = e;
      P.table[b * P.table_sb + i] = -1;
    }
    top -= all;
  }
}

template <typename T>
struct Piece {  // 16 bytes
  T x[16 / sizeof(T)];
};

// One thread per 16 bytes of a head, keys and values
template <typename T>
__global__ __launch_bounds__(256) void write_kernel(const WriteProb P, const T* __restrict__ k,
                                                    const T* __restrict__ v, T* __restrict__ kp,
                                                    T* __restrict__ vp, int pieces) {
  constexpr int N = 16 / sizeof(T);
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int c = (int)(id % pieces);
  const int64_t row = id / pieces;
  const int h = (int)(row % P.Hk);
  const int64_t t = row / P.Hk;
  if (t >= P.tokens) return;
  const int64_t slot = P.slots[t];
  if (slot < 0 || slot >= (int64_t)P.pages * P.page) return;
  const int64_t pg = slot / P.page, in = slot - pg * P.page;
  *(Piece<T>*)(kp + pg * P.k_sp + in * P.k_st + h * P.k_sh + N * c) =
      *(const Piece<T>*)(k + t * P.kn_st + h * P.kn_sh + N * c);
  *(Piece<T>*)(vp + pg * P.v_sp + in * P.v_st + h * P.v_sh + N * c) =
      *(const Piece<T>*)(v + t * P.vn_st + h * P.vn_sh + N * c);
}

}  // namespace

hipError_t launch_grow(const PagesProb& P, const int32_t* n_new, int32_t* starts, int64_t* slots,
                       int32_t* positions, int32_t* seen, hipStream_t st) {
  const bool few = P.B <= kFewSequences && P.tokens <= kFewTokens;
  if (few)
    hipLaunchKernelGGL((grow_kernel<256, true>), dim3(1), dim3(256), 0, st, P, n_new, starts, slots,
                       positions, seen);
  else
    hipLaunchKernelGGL((grow_kernel<1024, false>), dim3(1), dim3(1024), 0, st, P, n_new, starts,
                       slots, positions, seen);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || few) return e;
  hipLaunchKernelGGL(slots_kernel, dim3((P.tokens + 255) / 256), dim3(256), 0, st, P, n_new, starts,
                     slots, positions);
  return hipGetLastError();
}

size_t release_bytes(const PagesProb& P) {
  return ((size_t)(P.B + 1) * sizeof(RowBack) + 255) & ~(size_t)255;
}

hipError_t launch_release(const PagesProb& P, char* ws, hipStream_t st) {
  RowBack* rows = (RowBack*)ws;
  hipLaunchKernelGGL(release_count_kernel, dim3(P.B), dim3(256), 0, st, P, rows);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(release_kernel, dim3(P.B), dim3(256), 0, st, P, rows);
  return hipGetLastError();
}

hipError_t launch_write(const WriteProb& P, const void* k, const void* v, void* kp, void* vp,
                        hipStream_t st) {
  const int pieces = P.d / (P.dtype == CA_BF16 ? 8 : 4);
  const int64_t threads = (int64_t)P.tokens * P.Hk * pieces;
  const dim3 grid((unsigned)((threads + 255) / 256));
  if (P.dtype == CA_BF16)
    hipLaunchKernelGGL((write_kernel<bf16>), grid, dim3(256), 0, st, P, (const bf16*)k,
                       (const bf16*)v, (bf16*)kp, (bf16*)vp, pieces);
  else
    hipLaunchKernelGGL((write_kernel<float>), grid, dim3(256), 0, st, P, (const float*)k,
                       (const float*)v, (float*)kp, (float*)vp, pieces);
  return hipGetLastError();
}

}  // namespace ca
