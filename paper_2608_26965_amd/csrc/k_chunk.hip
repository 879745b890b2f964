// Attention of packed chunks of new tokens over a paged key-value cache.
//
// All query heads of a key head share its keys, so a sequence's rows are its new
// tokens times the G heads of the group (row r: token r / G, head r % G), taken
// in blocks; a block walks the 64-key tiles that one of its rows sees. Blocks
// have very different lengths (a prompt's beside a single token's on a long cache),
// so a first launch plans them: it counts all tiles and cuts long blocks into parts of
// about what a workgroup's share is. The parts' softmax states are joined by a
// last launch. The plan is the same for all key heads.
//
// What bounds it: the matrix cores for prompts, the cache (read once by each block)
// for few new tokens.
#include <math.h>

#include "seq.h"
#include "walk_bf16.h"

namespace ca {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kPlan = 256;     // threads of the planning workgroup
constexpr int kPartTiles = 8;  // tiles of a part, at least
constexpr int kF32Rows = 64;   // rows of a block, fp32

// A workgroup's work, for every key head: tiles [t0, t1) of block a of sequence b (with
// its lengths and first row). slot: where a part's state goes, -1 for a whole block.
struct Item {
  int b, a, t0, t1, slot, lq, lk, start;
};
// A block that is cut: its parts' states lie in slots slot .. slot + n - 1
struct Cut {
  int a, slot, n, lq, lk, start;
};
struct PlanHead {
  int items, cuts;
};

// Bounds that the host knows, and where things lie in the workspace
struct Plan {
  int rows;                           // of a block
  int blocks, share, items, slots;    // at most, for one key head; share: parts that blocks
                                      // are cut for
  int cuts;
  size_t item_at, cut_at, part_at, bytes;
};

// Positions of a block's first and last row (a sequence has fewer than 2^30 rows)
struct BlockSpan {
  int p0, p1;
  __device__ __forceinline__ BlockSpan(int a, int rows, int G, int lq, int lk) {
    const int r0 = a * rows;
    p0 = r0 / G + lk - lq;
    p1 = min((r0 + rows - 1) / G, lq - 1) + lk - lq;
  }
};

// Sums of x and y over the threads before this one, and over all of them
struct Pair {
  int x, y;
};
__device__ __forceinline__ Pair plan_scan(int x, int y, Pair (&sums)[kPlan / 64], Pair* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int a = x, b = y;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int c = __shfl_up(a, o, 64), d = __shfl_up(b, o, 64);
    if (lane >= o) {
      a += c;
      b += d;
    }
  }
  __syncthreads();  // the sums of a scan before are read
  if (lane == 63) sums[w] = Pair{a, b};
  __syncthreads();
  Pair before{a - x, b - y}, all{0, 0};
#pragma unroll
  for (int i = 0; i < kPlan / 64; ++i) {
    if (i < w) {
      before.x += sums[i].x;
      before.y += sums[i].y;
    }
    all.x += sums[i].x;
    all.y += sums[i].y;
  }
  *total = all;
  return before;
}

// The last place of ascending list[0 .. kPlan - 1] that holds at most i
__device__ __forceinline__ int plan_find(const int* list, int i) {
  int lo = 0;
#pragma unroll
  for (int step = kPlan / 2; step > 0; step >>= 1)
    if (list[lo + step] <= i) lo += step;
  return lo;
}

// One workgroup: blocks by sequence, the last one (with most keys, if causal) first. A pass
// counts the tiles, another one cuts and writes the items, thread by item.
__global__ __launch_bounds__(kPlan) void chunk_plan_kernel(const ChunkProb P, const Plan L,
                                                           char* ws) {
  __shared__ Pair sums[kPlan / 64];
  __shared__ int64_t tiles_of[kPlan / 64];
  // of a sequence: its first block; of a block: its first item
  __shared__ int first[kPlan], s_n[kPlan], s_lq[kPlan], s_lk[kPlan], s_start[kPlan];
  __shared__ int b_item[kPlan], b_seq[kPlan], b_a[kPlan], b_tiles[kPlan], b_slot[kPlan];
  PlanHead* head = (PlanHead*)ws;
  Item* items = (Item*)(ws + L.item_at);
  Cut* cuts = (Cut*)(ws + L.cut_at);
  const int tid = threadIdx.x;
  int64_t tiles_seen = 0;
  int n_items = 0, n_slots = 0, n_cuts = 0, part = 1;
  for (int pass = 0; pass < 2; ++pass) {
    int seen = 0;  // blocks so far: no more than the host counted
    for (int b0 = 0; b0 < P.B && seen < L.blocks; b0 += kPlan) {
      const int b = b0 + tid;
      int n = 0;
      if (b < P.B) {
        const int start = P.start(b), lq = max(0, P.start(b + 1) - start);
        s_start[tid] = start;
        s_lq[tid] = lq;
        s_lk[tid] = P.klen(b);
        s_n[tid] = n = (int)(((uint32_t)lq * (uint32_t)P.G + L.rows - 1) / (uint32_t)L.rows);
      }
      Pair total;
      const Pair before = plan_scan(min(n, L.blocks), 0, sums, &total);
      // (unsigned: the sum of starts that do not ascend may pass 2^31)
      const int blocks = (int)min((uint32_t)total.x, (uint32_t)(L.blocks - seen));
      first[tid] = (int)min((uint32_t)before.x, (uint32_t)INT32_MAX);
      __syncthreads();
      for (int i0 = 0; i0 < blocks; i0 += kPlan) {
        const int i = i0 + tid;
        int tiles = 0, parts = 0, lo = 0, a = 0;
        if (i < blocks) {
          lo = plan_find(first, i);
          a = s_n[lo] - 1 - (i - first[lo]);
          const BlockSpan s(a, L.rows, P.G, s_lq[lo], s_lk[lo]);
          tiles = visible_tiles<KT>(P.m, s.p0, s.p1, s_lk[lo]).n;
          parts = max(1, (tiles + part - 1) / part);
        }
        if (pass == 0) {
          tiles_seen += tiles;
          continue;
        }
        const Pair at = plan_scan(parts, parts > 1 ? 1 : 0, sums, &total);
        // slots count the parts of cut blocks: all items but those of whole ones
        const int slot = n_slots + at.x - (tid - at.y), cut = n_cuts + at.y;
        b_item[tid] = at.x;
        b_seq[tid] = lo;
        b_a[tid] = a;
        b_tiles[tid] = tiles;
        b_slot[tid] = parts > 1 ? slot : -1;
        // (the host's bounds hold for ascending starts; nothing is written outside them)
        if (parts > 1 && cut < L.cuts && slot + parts <= L.slots)
          cuts[cut] = Cut{a, slot, parts, s_lq[lo], s_lk[lo], s_start[lo]};
        __syncthreads();
        const int some = min(kPlan, blocks - i0);
        for (int j = tid; j < total.x; j += kPlan) {
          const int x = min(plan_find(b_item, j), some - 1), y = j - b_item[x], q = b_seq[x];
          const int all = (x + 1 < some ? b_item[x + 1] : total.x) - b_item[x];
          const int per = (b_tiles[x] + all - 1) / all, t0 = min(b_tiles[x], y * per);
          const int z = b_slot[x] < 0 ? -1 : b_slot[x] + y;
          if (n_items + j < L.items && z < L.slots)
            items[n_items + j] = Item{b0 + q, b_a[x], t0, min(b_tiles[x], t0 + per), z,
                                      s_lq[q], s_lk[q], s_start[q]};
        }
        n_items += total.x;
        n_cuts += total.y;
        n_slots += total.x - (some - total.y);
      }
      seen += blocks;
      __syncthreads();  // the segment's lists are read
    }
    if (pass == 0) {
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) tiles_seen += __shfl_xor(tiles_seen, o, 64);
      if ((tid & 63) == 0) tiles_of[tid >> 6] = tiles_seen;
      __syncthreads();
      int64_t all = 0;
#pragma unroll
      for (int x = 0; x < kPlan / 64; ++x) all += tiles_of[x];
      part = (int)min(max((int64_t)kPartTiles, (all + L.share - 1) / L.share), (int64_t)1 << 25);
    }
  }
  if (tid == 0) {
    head->items = min(n_items, L.items);
    head->cuts = min(n_cuts, L.cuts);
  }
}

// Workgroup w of the grid runs on XCD w % 8. The key heads are spread over the XCDs,
// each of which then works on one head at a time, whose keys stay in its L2; where
// the heads' number and 8 have g as their greatest common divisor, 8 / g XCDs share a
// head, neighbouring items on different ones.
struct ItemOrder {
  int g, slots;  // slots: heads of an XCD
  static ItemOrder of(int Hk) {
    int g = 8;
    while (Hk % g) g /= 2;
    return ItemOrder{g, Hk / g};
  }
  int64_t grid(int items) const { return (int64_t)8 * slots * ((items + 8 / g - 1) / (8 / g)); }
  __device__ __forceinline__ bool at(int wg, int items, int* item, int* hk) const {
    const int r = 8 / g, x = wg & 7, s = wg >> 3, per = (items + r - 1) / r;
    if (per == 0) return false;
    const int hs = s / per;
    *item = (s - hs * per) * r + x / g;
    *hk = hs * g + x % g;
    return hs < slots && *item < items;
  }
};

// ---- bf16 ---------------------------------------------------------------------------------

// n / d for 0 <= n < 2^30, d < 2^30
struct FastDiv {
  uint32_t m;
  int s;
  static FastDiv of(int d) {
    int k = 0;
    while ((1 << k) < d) ++k;
    return FastDiv{(uint32_t)(((uint64_t)1 << (30 + k)) / (uint32_t)d + 1), 30 + k};
  }
  __host__ __device__ __forceinline__ int div(int n) const {
    return (int)(((uint64_t)(uint32_t)n * m) >> s);
  }
};

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

// Tiles whose rows lie on pages. Wavefront w copies rows 16 w .. 16 w + 15 of a
// tile. GROUPS: pages of a multiple of 16 tokens, so that the sixteen lie on one page,
// whose entry is one scalar load (from the constant address space: no kernel writes the
// table while this one runs); else a lane looks up its row's entry. Entries are
// loaded a tile before the copies that need them.
template <int D, bool GROUPS>
struct PagedTiles : WalkRows {
  static constexpr bool kHoles = true;
  static constexpr float kMostSum = 0x1p30f;
  static constexpr int RB = 2 * D, TILE = KT * RB, NI = RB / 64, RPI = 1024 / RB;
  typedef const __attribute__((address_space(4))) int32_t* Entries;
  const bf16 *kh, *vh;  // of this key head
  const int32_t* table;
  int64_t k_sp, k_st, v_sp, v_st;
  int page, pages, most;  // most: last entry of the row
  FastDiv by_page;
  char* smem;
  uint16_t (*hole)[4];
  uint32_t lds0;
  int w, lane;
  int ev, ek;  // entries of the tile whose values, and of the one whose keys are next

  __device__ __forceinline__ int key(int t) const {
    return KT * tile(t) + 16 * w + (GROUPS ? 0 : lane & 15);
  }
  __device__ __forceinline__ int entry(int t) const {
    const int e = min(by_page.div(min(key(t), lk - 1)), most);
    if constexpr (GROUPS)
      return ((Entries)table)[__builtin_amdgcn_readfirstlane(e)];
    else
      return table[e];
  }
  // keys (V false) or values of tile t, entry e, into LDS tile `at`
  template <bool V>
  __device__ __forceinline__ void copy(int t, int e, int at, int buf) const {
    const bf16* base = V ? vh : kh;
    const int64_t sp = V ? v_sp : k_sp, st = V ? v_st : k_st;
    const uint32_t dst = lds0 + at * TILE + 1024 * NI * w;
    const int row = lane / (RB / 16), j = key(t);
    auto chunk = [&](int c) __attribute__((always_inline)) {
      return ((lane % (RB / 16)) ^ row_key<RB>(RPI * c + row)) << 4;
    };
    auto nothing = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < NI; ++c)
        *(f32x4*)(smem + at * TILE + 1024 * (NI * w + c) + 16 * lane) = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    if constexpr (GROUPS) {
      const bool there = e >= 0 && e < pages;
      const int last = lk - 1 - j;  // of the group's rows
      if (!V && lane == 0) hole[buf][w] = there || last < 0 ? 0 : 0xffff;
      if (!there || last < 0) {
        nothing();
        return;
      }
      const int in = j - by_page.div(j) * page;
      const char* src = (const char*)(base + e * sp + in * st);
      const uint32_t rb = (uint32_t)st * 2;
      if (last >= 15) {
#pragma unroll
        for (int c = 0; c < NI; ++c)
          lds_dma16(src + (int64_t)(RPI * c) * rb, (uint32_t)row * rb + chunk(c),
                    __builtin_amdgcn_readfirstlane(dst + 1024 * c));
      } else {  // rows past the last are copies of it
#pragma unroll
        for (int c = 0; c < NI; ++c)
          lds_dma16(src, (uint32_t)min(RPI * c + row, last) * rb + chunk(c),
                    __builtin_amdgcn_readfirstlane(dst + 1024 * c));
      }
    } else {
      const bool there = e >= 0 && e < pages;
      const uint32_t any = (uint32_t)__builtin_amdgcn_ballot_w64(there) & 0xffff;
      const uint32_t gone = (uint32_t)__builtin_amdgcn_ballot_w64(!there && j < lk) & 0xffff;
      if (!V && lane == 0) hole[buf][w] = (uint16_t)gone;
      if (any == 0) {
        nothing();
        return;
      }
      const int n = min(j, lk - 1), in = n - by_page.div(n) * page;
      int64_t o = there ? e * sp + in * st : 0;
      // rows that are not there: copies of one that is
      const int64_t o1 = __shfl(o, __builtin_ctz(any), 64);
      o = there ? o : o1;
#pragma unroll
      for (int c = 0; c < NI; ++c)
        lds_dma16_at((const char*)(base + __shfl(o, RPI * c + row, 64)) + chunk(c),
                     __builtin_amdgcn_readfirstlane(dst + 1024 * c));
    }
  }
  __device__ __forceinline__ void issue_k(int t, int buf) { copy<false>(t, ek, buf, buf); }
  __device__ __forceinline__ void issue_v(int t, int buf) {
    copy<true>(t, ev, 2 + buf, buf);
    ev = ek;
    ek = entry(min(t + 2, t1 - 1));
  }
  __device__ __forceinline__ void first_k() {
    ev = entry(t0);
    copy<false>(t0, ev, 0, 0);
    ek = entry(min(t0 + 1, t1 - 1));
  }
  __device__ __forceinline__ void issue_both(int t) const {
    const int e = entry(t);
    copy<false>(t, e, 0, 0);
    copy<true>(t, e, 2, 0);
  }
  __device__ __forceinline__ uint64_t holes(int buf) const {
    uint2 x;
    __builtin_memcpy(&x, hole[buf], 8);
    return (uint64_t)__builtin_amdgcn_readfirstlane(x.y) << 32 |
           (uint32_t)__builtin_amdgcn_readfirstlane(x.x);
  }
};

template <int D, bool GROUPS>
__global__ __launch_bounds__(256, (D == 64 ? 3 : 2)) void chunk_bf16_kernel(
    const ChunkProb P, const Plan L, const ItemOrder order, const FastDiv by_page,
    const bf16* __restrict__ q, const bf16* __restrict__ kp, const bf16* __restrict__ vp,
    bf16* __restrict__ out, float* __restrict__ lse, char* __restrict__ ws, float sl2) {
  constexpr int KS = D / 16, DT = D / 32, RB = 2 * D, TILE = KT * RB;
  __shared__ __attribute__((aligned(1024))) char smem[4 * TILE];  // two tiles of keys, two of values
  __shared__ __attribute__((aligned(8))) uint16_t hole[2][4];
  __shared__ int redo;
  int item, hk;
  if (!order.at(blockIdx.x, ((const PlanHead*)ws)->items, &item, &hk)) return;
  const Item it = ((const Item*)(ws + L.item_at))[item];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int off = it.lk - it.lq, r0 = it.a * kWalkRows, rows = it.lq * P.G;
  const BlockSpan span(it.a, kWalkRows, P.G, it.lq, it.lk);
  const int w0 = r0 + 32 * w, wreal = max(0, min(32, rows - w0));
  const int row = min(w0 + min(l32, max(wreal, 1) - 1), rows - 1);  // this lane's row
  const int tok = row / P.G, head = hk * P.G + row - tok * P.G;
  const int wl = min(w0 + max(wreal, 1) - 1, rows - 1);
  PagedTiles<D, GROUPS> T;
  T.mask = P.m;
  T.list = visible_tiles<KT>(P.m, span.p0, span.p1, it.lk);
  T.t0 = it.t0;
  T.t1 = it.t1;
  T.lk = it.lk;
  T.ra = visible_keys(P.m, min(w0, rows - 1) / P.G + off, it.lk);
  T.rz = visible_keys(P.m, wl / P.G + off, it.lk);
  T.pos = tok + off;
  T.real = wreal;
  T.block_first = span.p0;
  T.block_last = span.p1;
  T.kh = kp + hk * P.k_sh;
  T.vh = vp + hk * P.v_sh;
  T.table = P.table + it.b * P.table_sb;
  T.k_sp = P.k_sp;
  T.k_st = P.k_st;
  T.v_sp = P.v_sp;
  T.v_st = P.v_st;
  T.page = P.page;
  T.pages = P.pages;
  T.most = P.max_pages - 1;
  T.by_page = by_page;
  T.smem = smem;
  T.hole = hole;
  T.lds0 = lds_addr(smem);
  T.w = w;
  T.lane = lane;
  T.ev = T.ek = 0;

  bf16x8 qreg[KS];
  {
    const bf16* src = q + (it.start + tok) * P.q_st + head * P.q_sh;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) qreg[kk] = *(const bf16x8*)(src + 16 * kk + 8 * h);
  }
  // Retire the loads here (a wait the compiler sees), so that no vmcnt wait of
  // theirs lands in the loop, where it would also wait for the copies in flight.
  __builtin_amdgcn_s_waitcnt(kWalkVmcnt0);
  if (tid == 0) redo = 0;  // ordered before any write by the barriers of the tiles
  f32x16 oacc[DT];
  float m, l_tot;
  walk_bf16<D>(T, smem, &redo, qreg, sl2, w, lane, oacc, m, l_tot);
  if (it.slot >= 0) {
    // A sum far above its reference goes out against a reference at its own size: the
    // joining compares references, and adds up as many sums as there are parts
    const int up = l_tot > 0x1p22f ? __builtin_amdgcn_frexp_expf(l_tot) : 0;
    m += (float)up;
    l_tot = __builtin_amdgcn_ldexpf(l_tot, -up);
    if (l32 >= wreal) return;
    float* x = (float*)(ws + L.part_at) +
               (((size_t)hk * L.slots + it.slot) * L.rows + 32 * w + l32) * (D + 4);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = __builtin_amdgcn_ldexpf(oacc[dt][4 * g + j], -up);
        *(f32x4*)(x + 32 * dt + 8 * g + 4 * h) = y;
      }
    if (h == 0) {
      x[D] = m;
      x[D + 1] = l_tot;
    }
    return;
  }
  if (l32 >= wreal) return;
  const bool any = l_tot != 0.f;
  const float inv = any ? 1.f / l_tot : 0.f;
  bf16* orow = out + (it.start + tok) * P.o_st + head * P.o_sh;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = f2bf(any ? oacc[dt][4 * g + j] * inv : 0.f);
      *(bf16x4*)(orow + 32 * dt + 8 * g + 4 * h) = x;
    }
  if (lse && h == 0)
    lse[(size_t)(it.start + tok) * P.H + head] =
        any ? (m + __builtin_amdgcn_logf(l_tot)) * kLn2 : -INFINITY;
}

// ---- joining the parts --------------------------------------------------------------------

// A row's parts are read 16 bytes a lane, D / 4 lanes a part, by one wavefront where there
// are few of them, by the four of the workgroup where there are many. The workgroups take
// groups of four rows (few parts) or a row (many) one after the other.
constexpr int kJoinGrid = 2048, kFewParts = 16;

template <typename T, int DP>
__global__ __launch_bounds__(256) void chunk_join_kernel(const ChunkProb P, const Plan L,
                                                         const char* __restrict__ ws,
                                                         T* __restrict__ out,
                                                         float* __restrict__ lse) {
  constexpr int LP = DP / 4, NP = 64 / LP;  // lanes of a part, parts of a wavefront's read
  __shared__ float acc[4][DP], wmax[4], wsum[4];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int t = 4 * (lane % LP), stride = P.d + 4, n_cuts = ((const PlanHead*)ws)->cuts;
  const size_t next = (size_t)L.rows * stride;
  for (int c = blockIdx.x; c < n_cuts * P.Hk * (L.rows / 4); c += gridDim.x) {
    const int rq = c % (L.rows / 4), x = c / (L.rows / 4), hk = x / n_cuts;
    const Cut cut = ((const Cut*)(ws + L.cut_at))[x - hk * n_cuts];
    const int r0 = cut.a * L.rows, real = min(L.rows, cut.lq * P.G - r0);
    const bool few = cut.n <= kFewParts;
    for (int r = 4 * rq + (few ? w : 0); r < min(real, 4 * rq + 4); r += few ? 4 : 1) {
      const float* p = (const float*)(ws + L.part_at) +
                       (((size_t)hk * L.slots + cut.slot) * L.rows + r) * stride;
      // each lane's own parts against their own maximum, then all against the largest
      float mx = -INFINITY, sum = 0.f;
      f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
      for (int i = (few ? 0 : w * NP) + lane / LP; i < cut.n; i += few ? NP : 4 * NP) {
        const float* y = p + i * next;
        const f32x4 v = t < P.d ? *(const f32x4*)(y + t) : f32x4{0.f, 0.f, 0.f, 0.f};
        const float m = y[P.d], s = y[P.d + 1];
        // no key of the part is there: its reference is not one
        const float m1 = s == 0.f ? mx : fmaxf(mx, m);
        const float ref = m1 == -INFINITY ? 0.f : m1;
        const float f = s == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - ref);
        const float g = __builtin_amdgcn_exp2f(mx - ref);
        sum = sum * g + s * f;
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = a[e] * g + v[e] * f;
        mx = m1;
      }
      auto merge = [&](float m2, float s2, f32x4 a2) __attribute__((always_inline)) {
        const float m1 = fmaxf(mx, m2), ref = m1 == -INFINITY ? 0.f : m1;
        const float f = __builtin_amdgcn_exp2f(mx - ref), g = __builtin_amdgcn_exp2f(m2 - ref);
        sum = sum * f + s2 * g;
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = a[e] * f + a2[e] * g;
        mx = m1;
      };
#pragma unroll
      for (int o = LP; o < 64; o <<= 1) {
        const f32x4 b = {__shfl_xor(a[0], o, 64), __shfl_xor(a[1], o, 64), __shfl_xor(a[2], o, 64),
                         __shfl_xor(a[3], o, 64)};
        merge(__shfl_xor(mx, o, 64), __shfl_xor(sum, o, 64), b);
      }
      if (!few) {
        __syncthreads();  // the row before is read
        if (lane < LP) *(f32x4*)&acc[w][t] = a;
        if (lane == 0) {
          wmax[w] = mx;
          wsum[w] = sum;
        }
        __syncthreads();
        if (w > 0) continue;
#pragma unroll
        for (int i = 1; i < 4; ++i) merge(wmax[i], wsum[i], *(const f32x4*)&acc[i][t]);
      }
      if (lane >= LP) continue;
      const int row = r0 + r, tok = row / P.G, h = hk * P.G + row - tok * P.G;
      T* o = out + (cut.start + tok) * P.o_st + h * P.o_sh + t;
      if (t < P.d)
#pragma unroll
        for (int e = 0; e < 4; ++e) store_f(o + e, sum != 0.f ? a[e] / sum : 0.f);
      if (lse && lane == 0)
        lse[(size_t)(cut.start + tok) * P.H + h] =
            sum != 0.f ? (mx + __builtin_amdgcn_logf(sum)) * kLn2 : -INFINITY;
    }
  }
}

// ---- fp32 ---------------------------------------------------------------------------------
//
// One wavefront per 16 rows, on the fp32 matrix instructions (v_mfma_f32_16x16x4_f32): S^T =
// K Q^T leaves lane l with row l % 16 and the logits of keys 4 (l / 16) + r, which is
// the P^T operand of O^T = V^T P^T as it stands. Half tiles of 32 keys go through registers
// to LDS, one ahead of the one that is computed; rows of DP + 4 floats there, so that
// neither the keys' 16-byte reads nor the values' 4-byte reads meet on a bank. What bounds
// it: the matrix instructions, 32 cycles each.

template <int DP, int WAVES>
__global__ __launch_bounds__(256, WAVES) void chunk_f32_kernel(
    const ChunkProb P, const Plan L, const ItemOrder order, const FastDiv by_page,
    const float* __restrict__ q, const float* __restrict__ kp, const float* __restrict__ vp,
    float* __restrict__ out, float* __restrict__ lse, char* __restrict__ ws, float sl2) {
  constexpr int HK = 32, NJ = DP / 16, LD = DP + 4, NC = DP / 4;
  constexpr int RP = 256 / NC, NP = HK / RP;  // rows of a pass of the copy, passes
  __shared__ __attribute__((aligned(16))) float ks[2][HK][LD], vs[2][HK][LD];
  __shared__ uint32_t gone[4], bad[4];  // keys not there, values that are not finite
  int item, hk;
  if (!order.at(blockIdx.x, ((const PlanHead*)ws)->items, &item, &hk)) return;
  const Item it = ((const Item*)(ws + L.item_at))[item];
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, l16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int off = it.lk - it.lq, r0 = it.a * kF32Rows, rows = it.lq * P.G;
  const BlockSpan span(it.a, kF32Rows, P.G, it.lq, it.lk);
  const TileList list = visible_tiles<KT>(P.m, span.p0, span.p1, it.lk);
  const int w0 = r0 + 16 * w, wreal = max(0, min(16, rows - w0));
  const int wl = min(w0 + max(wreal, 1) - 1, rows - 1);
  const int row = min(w0 + l16, wl);  // this lane's row
  const int tok = row / P.G, head = hk * P.G + row - tok * P.G;
  const KeyRange ra = visible_keys(P.m, min(w0, rows - 1) / P.G + off, it.lk);
  const KeyRange rz = visible_keys(P.m, wl / P.G + off, it.lk);
  const KeyRange mine = visible_keys(P.m, tok + off, it.lk);

  f32x4 qf[NJ];
  {
    const float* src = q + (it.start + tok) * P.q_st + head * P.q_sh;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int x = 16 * j + 4 * g;
      qf[j] = x < P.d ? *(const f32x4*)(src + x) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  const int cc = 4 * (tid % NC), cr = tid / NC;  // this thread's piece of a row, and row
  const int32_t* table = P.table + it.b * P.table_sb;
  const float *kh = kp + hk * P.k_sh + cc, *vh = vp + hk * P.v_sh + cc;
  const int n = 2 * (it.t1 - it.t0);  // half tiles
  auto first_key = [&](int i) __attribute__((always_inline)) {
    return KT * list.tile(it.t0 + (i >> 1)) + HK * (i & 1);
  };
  int ent[NP];
  auto entries = [&](int i) __attribute__((always_inline)) {
    const int j0 = first_key(min(i, n - 1)) + cr;
#pragma unroll
    for (int x = 0; x < NP; ++x) ent[x] = table[by_page.div(min(j0 + x * RP, it.lk - 1))];
  };
  f32x4 kr[NP], vr[NP];
  uint32_t missing;
  auto load = [&](int i) __attribute__((always_inline)) {
    const int j0 = first_key(i) + cr;
    missing = 0;
#pragma unroll
    for (int x = 0; x < NP; ++x) {
      const int j = j0 + x * RP, e = ent[x], c = min(j, it.lk - 1), in = c - by_page.div(c) * P.page;
      const bool there = e >= 0 && e < P.pages;
      kr[x] = vr[x] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (there && j < it.lk && cc < P.d) {
        kr[x] = *(const f32x4*)(kh + e * P.k_sp + in * P.k_st);
        vr[x] = *(const f32x4*)(vh + e * P.v_sp + in * P.v_st);
      }
      if (!there && j < it.lk) missing |= 1u << (cr + x * RP);
    }
  };
  auto store = [&](int i) __attribute__((always_inline)) {
    if (missing) atomicOr(&gone[i & 3], missing);
#pragma unroll
    for (int x = 0; x < NP; ++x) {
      const int r = cr + x * RP;
      bool fine = true;
#pragma unroll
      for (int e = 0; e < 4; ++e) fine &= fabsf(vr[x][e]) < INFINITY;
      if (__builtin_expect(!fine, 0)) {
        // zero times it would reach rows that do not see it: those that do get NaN at the end
        atomicOr(&bad[i & 3], 1u << r);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!(fabsf(vr[x][e]) < INFINITY)) vr[x][e] = 0.f;
      }
      *(f32x4*)&ks[i & 1][r][cc] = kr[x];
      *(f32x4*)&vs[i & 1][r][cc] = vr[x];
    }
  };
  f32x4 o[NJ];
  float m = -INFINITY, l = 0.f;  // reference (log2 units), this lane's part of the sum
  bool poison = false;
#pragma unroll
  for (int j = 0; j < NJ; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto compute = [&](int i) __attribute__((always_inline)) {
    const int k0 = first_key(i);
    // no row sees a key; every row sees all
    if (k0 >= rz.s_end && (k0 >= rz.hi || k0 + HK <= ra.lo)) return;
    const uint32_t hv = gone[i & 3], bv = bad[i & 3];
    const bool all = (k0 + HK <= ra.s_end || (k0 >= rz.lo && k0 + HK <= ra.hi)) && hv == 0;
    const float(*kt)[LD] = ks[i & 1];
    const float(*vt)[LD] = vs[i & 1];
    // four partial sums a logit: shorter chains of rounded sums
    f32x4 p[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) p[u][e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const f32x4 kf = *(const f32x4*)&kt[16 * u + l16][16 * j + 4 * g];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          p[u][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[e], qf[j][e], p[u][e], 0, 0, 0);
      }
    float s[2][4], mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[u][r] = (p[u][0][r] + p[u][1][r]) + (p[u][2][r] + p[u][3][r]);
        const int j = 16 * u + 4 * g + r;
        if (!all && (!sees(mine, k0 + j) || ((hv >> j) & 1))) s[u][r] = -INFINITY;
        mx = fmaxf(mx, s[u][r]);
      }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * sl2;
    if (__builtin_amdgcn_ballot_w64(mx > m)) {
      const float m1 = fmaxf(m, mx), al = m1 > m ? __builtin_amdgcn_exp2f(m - m1) : 1.f;
      l *= al;
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[j][r] *= al;
      m = m1;
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        s[u][r] = __builtin_amdgcn_exp2f(fmaf(s[u][r], sl2, -ref));
        l += s[u][r];
      }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
          o[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vt[16 * u + 4 * g + r][16 * j + l16], s[u][r],
                                                      o[j], 0, 0, 0);
    if (__builtin_expect(bv != 0, 0))
      for (uint32_t x = bv; x; x &= x - 1) poison |= sees(mine, k0 + __builtin_ctz(x));
  };
  if (tid < 4) gone[tid] = bad[tid] = 0;
  __syncthreads();
  if (n > 0) {
    entries(0);
    load(0);
    entries(1);
    store(0);
    __syncthreads();
    for (int i = 0; i < n; ++i) {
      if (i + 1 < n) load(i + 1);
      entries(i + 2);
      // the flags of half tile i + 2 (those of i - 2 were read before the last barrier)
      if (tid == 0) gone[(i + 2) & 3] = bad[(i + 2) & 3] = 0;
      if (wreal) compute(i);
      if (i + 1 < n) store(i + 1);
      __syncthreads();
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (l16 >= wreal) return;
  if (poison) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) o[j] = f32x4{NAN, NAN, NAN, NAN};
  }
  if (it.slot >= 0) {
    float* x = (float*)(ws + L.part_at) +
               (((size_t)hk * L.slots + it.slot) * L.rows + 16 * w + l16) * (P.d + 4);
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      if (16 * j + 4 * g < P.d) *(f32x4*)(x + 16 * j + 4 * g) = o[j];
    if (g == 0) {
      x[P.d] = m;
      x[P.d + 1] = l;
    }
    return;
  }
  const bool any = l != 0.f;
  float* orow = out + (it.start + tok) * P.o_st + head * P.o_sh;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
    if (16 * j + 4 * g < P.d) {
      f32x4 x;
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = any ? o[j][r] / l : 0.f;
      *(f32x4*)(orow + 16 * j + 4 * g) = x;
    }
  if (lse && g == 0)
    lse[(size_t)(it.start + tok) * P.H + head] =
        any ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
}

// ---- launches -----------------------------------------------------------------------------

// Workgroups that the compute units hold at once (256 units, two or three each): the share
// of one of them is what a block is cut to, so that no workgroup runs much longer
// than all need together.
Plan plan_of(const ChunkProb& P) {
  Plan L;
  L.rows = P.dtype == CA_BF16 ? kWalkRows : kF32Rows;
  const int held = P.d > 64 ? 512 : P.dtype == CA_BF16 ? 768 : 1024;
  const int64_t rows = (int64_t)P.tokens * P.G;
  L.blocks = (int)(rows / L.rows + (P.B < P.tokens ? P.B : P.tokens));
  L.share = (held + P.Hk - 1) / P.Hk;
  // a cut block has more than `part` tiles, part >= all tiles / share: the parts of the cut
  // blocks are at most twice the share, and so few blocks are cut
  L.slots = 2 * L.share;
  L.cuts = L.share < L.blocks ? L.share : L.blocks;
  int64_t most = ((int64_t)P.max_pages * P.page + KT - 1) / KT + 2;  // tiles of a block
  most = (most + kPartTiles - 1) / kPartTiles;
  if (most == 1) L.slots = L.cuts = 0;
  if (L.slots > L.blocks * most) L.slots = (int)(L.blocks * most);
  L.items = L.blocks + L.slots;
  auto align = [](size_t x) { return (x + 255) & ~(size_t)255; };
  L.item_at = 256;
  L.cut_at = align(L.item_at + (size_t)L.items * sizeof(Item));
  L.part_at = align(L.cut_at + (size_t)L.cuts * sizeof(Cut));
  L.bytes = align(L.part_at + (size_t)P.Hk * L.slots * L.rows * (P.d + 4) * 4);
  return L;
}

template <typename T, int DP>
hipError_t run_join(const ChunkProb& P, const Plan& L, T* out, float* lse, const char* ws,
                    hipStream_t st) {
  if (L.slots == 0) return hipSuccess;
  const int64_t quads = (int64_t)L.cuts * P.Hk * (L.rows / 4);
  const dim3 grid((unsigned)(quads < kJoinGrid ? quads : kJoinGrid));
  hipLaunchKernelGGL((chunk_join_kernel<T, DP>), grid, dim3(256), 0, st, P, L, ws, out, lse);
  return hipGetLastError();
}

template <int D>
hipError_t run_bf16(const ChunkProb& P, const Plan& L, const bf16* q, const bf16* kp,
                    const bf16* vp, bf16* out, float* lse, char* ws, hipStream_t st) {
  const ItemOrder order = ItemOrder::of(P.Hk);
  const dim3 grid((unsigned)order.grid(L.items));
  const FastDiv by_page = FastDiv::of(P.page);
  // the rows of a page that a group of 16 takes are reached by 32-bit offsets
  if (P.page % 16 == 0 && P.k_st <= (1 << 23) && P.v_st <= (1 << 23))
    hipLaunchKernelGGL((chunk_bf16_kernel<D, true>), grid, dim3(256), 0, st, P, L, order, by_page,
                       q, kp, vp, out, lse, ws, P.scale * kLog2e);
  else
    hipLaunchKernelGGL((chunk_bf16_kernel<D, false>), grid, dim3(256), 0, st, P, L, order, by_page,
                       q, kp, vp, out, lse, ws, P.scale * kLog2e);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : run_join<bf16, D>(P, L, out, lse, ws, st);
}

template <int DP, int WAVES>
hipError_t run_f32(const ChunkProb& P, const Plan& L, const float* q, const float* kp,
                   const float* vp, float* out, float* lse, char* ws, hipStream_t st) {
  const ItemOrder order = ItemOrder::of(P.Hk);
  hipLaunchKernelGGL((chunk_f32_kernel<DP, WAVES>), dim3((unsigned)order.grid(L.items)), dim3(256), 0,
                     st, P, L, order, FastDiv::of(P.page), q, kp, vp, out, lse, ws,
                     P.scale * kLog2e);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : run_join<float, DP>(P, L, out, lse, ws, st);
}

}  // namespace

bool chunk_fits(const ChunkProb& P) {
  if ((int64_t)P.tokens * P.G >= ((int64_t)1 << 30)) return false;
  // workgroups of 256 threads, fewer than 2^32 of them
  return ItemOrder::of(P.Hk).grid(plan_of(P).items) < (1 << 24);
}

size_t chunk_bytes(const ChunkProb& P) { return plan_of(P).bytes; }

hipError_t launch_chunk(const ChunkProb& P, const void* q, const void* kp, const void* vp, void* out,
                        float* lse, char* ws, hipStream_t st) {
  const Plan L = plan_of(P);
  hipLaunchKernelGGL(chunk_plan_kernel, dim3(1), dim3(kPlan), 0, st, P, L, ws);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (P.dtype == CA_BF16) {
    const bf16 *a = (const bf16*)q, *b = (const bf16*)kp, *c = (const bf16*)vp;
    return P.d == 64 ? run_bf16<64>(P, L, a, b, c, (bf16*)out, lse, ws, st)
                     : run_bf16<128>(P, L, a, b, c, (bf16*)out, lse, ws, st);
  }
  const float *a = (const float*)q, *b = (const float*)kp, *c = (const float*)vp;
  return P.d <= 32   ? run_f32<32, 4>(P, L, a, b, c, (float*)out, lse, ws, st)
         : P.d <= 64 ? run_f32<64, 4>(P, L, a, b, c, (float*)out, lse, ws, st)
                     : run_f32<128, 2>(P, L, a, b, c, (float*)out, lse, ws, st);
}

}  // namespace ca
