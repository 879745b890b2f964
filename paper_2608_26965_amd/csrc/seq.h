// Internal declarations of the sequence operators: rotary positions, attention
// with a sliding window and sinks (forward and backward), the paged key-value
// cache and the attention that reads it. Not part of the public ABI.
#pragma once

#include "common.h"

namespace ca {

// ---- visibility -----------------------------------------------------------------
// Query i of a sequence with lq queries and lk keys sits at p = i + lk - lq and
// sees key j < lk where (j < sinks or p - left <= j <= p + right) and, in causal
// attention, j <= p: two ranges of keys, [0, s_end) and [lo, hi), each monotone
// in p. An unlimited side is kUnlimited (sequences have at most 2^22 tokens, so
// no sum leaves 32 bits).
constexpr int kUnlimited = 1 << 23;

struct WinMask {
  int left, right, sinks, causal;
};

struct KeyRange {
  int s_end, lo, hi;  // sees keys [0, s_end) and [lo, hi)
};

__device__ __forceinline__ KeyRange visible_keys(const WinMask& m, int p, int lk) {
  const int top = m.causal ? min(lk, p + 1) : lk;
  KeyRange r;
  r.s_end = max(0, min(m.sinks, top));
  r.lo = max(0, p - m.left);
  r.hi = min(top, p + m.right + 1);  // at or below lo: no window
  return r;
}
__device__ __forceinline__ bool sees(const KeyRange& r, int j) {
  return j < r.s_end || (j >= r.lo && j < r.hi);
}

// The positions p that see key j: [lo, hi] (lo is monotone in j)
struct PosRange {
  int lo, hi;
};
__device__ __forceinline__ PosRange seeing_positions(const WinMask& m, int j) {
  const int after = m.causal ? j : -kUnlimited;
  PosRange r;
  r.lo = j < m.sinks ? after : max(after, j - m.right);
  r.hi = j < m.sinks ? kUnlimited : j + m.left;
  return r;
}

// Tiles of KT keys that hold every key seen from positions [p0, p1]: the sinks'
// tiles first, then the window's, none twice.
struct TileList {
  int ns, b0, n;  // sink tiles 0 .. ns - 1, then b0 .. b0 + n - ns - 1
  __device__ __forceinline__ int tile(int t) const { return t < ns ? t : b0 + t - ns; }
};
template <int KT>
__device__ __forceinline__ TileList visible_tiles(const WinMask& m, int p0, int p1, int lk) {
  const KeyRange a = visible_keys(m, p0, lk), b = visible_keys(m, p1, lk);
  TileList t;
  t.ns = (b.s_end + KT - 1) / KT;
  t.b0 = max(t.ns, a.lo / KT);
  t.n = t.ns + max(0, (max(b.hi, 0) + KT - 1) / KT - t.b0);
  return t;
}

// ---- window attention ---------------------------------------------------------------

struct WinProb {
  int B, H, Hk, G, nq, nk, d, dtype;  // G query heads share a key head
  WinMask m;
  float scale;
  const int32_t *len_q, *len_k;       // [B] or NULL
  Lay lq, lk, lv, lo, ldo, ldq, ldk, ldv;

  __device__ __forceinline__ int qlen(int b) const { return len_q ? min(max(len_q[b], 0), nq) : nq; }
  __device__ __forceinline__ int klen(int b) const { return len_k ? min(max(len_k[b], 0), nk) : nk; }
};

// workspace of the forward pass: partial results where the keys are cut into parts
size_t window_bytes(const WinProb& P);
hipError_t launch_window(const WinProb& P, const void* q, const void* k, const void* v, void* out,
                         float* lse, char* ws, hipStream_t st);
size_t window_bf16_bytes(const WinProb& P);
hipError_t launch_window_bf16(const WinProb& P, const void* q, const void* k, const void* v,
                              void* out, float* lse, char* ws, hipStream_t st);
size_t window_grad_bf16_bytes(const WinProb& P);
hipError_t launch_window_grad_bf16(const WinProb& P, const void* q, const void* k, const void* v,
                                   const void* out, const float* lse, const void* dout, void* dq,
                                   void* dk, void* dv, char* ws, hipStream_t st);
// Workspace of the backward pass (fp32): delta (the row sums of dout * out), fp32 [B H][nq],
// then the partial sums of the blocks that are cut, those of dq and afterwards of dk and dv
size_t window_backward_bytes(const WinProb& P);
hipError_t launch_window_backward(const WinProb& P, const void* q, const void* k, const void* v,
                                  const void* out, const float* lse, const void* dout, void* dq,
                                  void* dk, void* dv, char* ws, hipStream_t st);

// ---- rotary positions ------------------------------------------------------------------

constexpr int kMaxAxes = 4;

struct RopeProb {
  int B, H, Hk, n, d, dtype;
  int axes, npairs, halves;
  int end[kMaxAxes];   // pairs [end[a - 1], end[a]) turn with axis a
  int grid[kMaxAxes], start[kMaxAxes];
  int inner[kMaxAxes]; // tokens between neighbours on the axis, INT32_MAX at most
  float sign;          // of the angle: -1 for the transposed rotation
  const int32_t* pos;  // NULL: from the grid
  int64_t pos_sb, pos_sa, pos_sn;
  Lay lq, lk, lqo, lko;
  double freq[kMaxD / 2];
};

hipError_t launch_rope(const RopeProb& P, const void* q, const void* k, void* qo, void* ko,
                       hipStream_t st);

// ---- paged cache -------------------------------------------------------------------------

constexpr int kNoWindow = 1 << 30;  // left of a cache read whole (caches hold fewer tokens)

struct PagedProb {
  int B, H, Hk, G, d, dtype, page, pages, max_pages;
  int left, sinks;
  float scale;
  const int32_t *table, *lens;
  int64_t table_sb;
  int64_t q_sb, q_sh, o_sb, o_sh;
  int64_t k_sp, k_st, k_sh, v_sp, v_st, v_sh;  // page, token, head

  // keys of sequence b, at most what its row of the table holds
  __device__ __forceinline__ int klen(int b) const {
    const int64_t most = (int64_t)max_pages * page;
    return (int)min((int64_t)max(lens[b], 0), most);
  }
};

struct AppendProb {
  int n;
  int64_t k_sb, k_st, k_sh, v_sb, v_st, v_sh;  // new keys and values: batch, token, head
};

hipError_t launch_append(const PagedProb& P, const AppendProb& A, const void* k, const void* v,
                         void* kp, void* vp, hipStream_t st);
// workspace of the partial results of the parts that a sequence's keys are cut into
size_t paged_bytes(const PagedProb& P);
hipError_t launch_paged(const PagedProb& P, const void* q, const void* kp, const void* vp, void* out,
                        float* lse, char* ws, hipStream_t st);

// ---- chunks of new tokens over the paged cache --------------------------------------------

struct PagesProb {
  int B, page, pages, max_pages, tokens;
  int left, sinks;  // left: kNoWindow without a window
  int64_t table_sb;
  const int32_t* lens;
  int32_t *table, *free, *state;

  __device__ __forceinline__ int len(int b) const {
    return (int)min((int64_t)max(lens[b], 0), (int64_t)max_pages * page);
  }
};

hipError_t launch_grow(const PagesProb& P, const int32_t* n_new, int32_t* starts, int64_t* slots,
                       int32_t* positions, int32_t* seen, hipStream_t st);  // seen: may be NULL
size_t release_bytes(const PagesProb& P);
hipError_t launch_release(const PagesProb& P, char* ws, hipStream_t st);

struct ChunkProb {
  int B, H, Hk, G, d, dtype, page, pages, max_pages, tokens;
  WinMask m;  // unlimited sides: kNoWindow - 1 (caches hold fewer tokens; position + side fits)
  float scale;
  const int32_t *table, *lens, *starts;
  int64_t table_sb;
  int64_t q_st, q_sh, o_st, o_sh;              // token, head
  int64_t k_sp, k_st, k_sh, v_sp, v_st, v_sh;  // page, token, head

  __device__ __forceinline__ int klen(int b) const {
    return (int)min((int64_t)max(lens[b], 0), (int64_t)max_pages * page);
  }
  __device__ __forceinline__ int start(int b) const { return min(max(starts[b], 0), tokens); }
};

struct WriteProb {
  int Hk, d, dtype, page, pages, tokens;
  const int64_t* slots;
  int64_t kn_st, kn_sh, vn_st, vn_sh;          // new rows: token, head
  int64_t k_sp, k_st, k_sh, v_sp, v_st, v_sh;  // pools: page, token, head
};

hipError_t launch_write(const WriteProb& P, const void* k, const void* v, void* kp, void* vp,
                        hipStream_t st);
bool chunk_fits(const ChunkProb& P);  // sizes that one launch can have
size_t chunk_bytes(const ChunkProb& P);
hipError_t launch_chunk(const ChunkProb& P, const void* q, const void* kp, const void* vp, void* out,
                        float* lse, char* ws, hipStream_t st);

// ---- elements ------------------------------------------------------------------------------

// four consecutive elements in fp32
__device__ __forceinline__ f32x4 load4f(const float* p) { return *(const f32x4*)p; }
__device__ __forceinline__ f32x4 load4f(const bf16* p) {
  const bf16x4 x = *(const bf16x4*)p;
  return f32x4{bf2f(x[0]), bf2f(x[1]), bf2f(x[2]), bf2f(x[3])};
}
__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(bf16 x) { return bf2f(x); }
__device__ __forceinline__ void store_f(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_f(bf16* p, float x) { *p = f2bf(x); }

}  // namespace ca
