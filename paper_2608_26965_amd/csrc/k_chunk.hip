// Attention of packed chunks of new tokens over a paged key-value cache.
//
// All query heads of a key head share its keys, so a sequence's rows are its new
// tokens times the G heads of the group (row r: token r / G, head r % G), taken
// in blocks; a block walks the 64-key tiles that one of its rows sees. Blocks
// have very different lengths (a prompt's beside a single token's on a long cache)
// and their number seldom fills the compute units evenly, so a first launch plans the
// work: it lists the blocks and gives every workgroup an equal share of all their
// tiles, from some tile of one block to some tile of a later one. A block that
// several workgroups share leaves its softmax states in the workspace, and a last launch
// joins them. Where there is more than a round of blocks, the first rounds are whole ones
// (the workgroups that run at a time then read the same keys at a time), and
// the shares even out the rest. Calls whose blocks have few tiles by their sizes alone go
// without a plan: a workgroup finds its block by itself.
//
// What bounds it: the matrix cores for prompts (bf16, 8,192 tokens on 24,576, 32 heads on 8 of
// 128: 3.33 to 3.52 ms, 1,090 to 1,160 TFLOP/s, four fifths of what a large matrix product reaches),
// the cache for few new tokens (16 rows on 262,144, 16 heads of 64: 222 us, 4.8 TB/s; a kernel that
// only reads reaches 5.4 over 1 GiB), the three launches for little of both (8 sequences, 5 tokens
// each on up to 16,000: 25 us, of which the plan and the joining are 12).
#include <math.h>

#include <algorithm>

#include "seq.h"
#include "walk_bf16.h"

namespace ca {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kPlan = 256;       // threads of the planning workgroup
constexpr int kF32Rows = 64;     // rows of a block, fp32
constexpr int kXcdUnits = 32;    // compute units of an XCD
constexpr int kMostHeld = 8 * kXcdUnits * 3;  // workgroups that run at a time, at most
constexpr int kShareTiles = 4;   // tiles of a share, at least
constexpr int kMostParts = 128;  // of a block, about
// What starting a block costs, in tiles. (3 in fp32: four ragged sequences 55.2 instead of 56.0 us,
// 24 of 4,565 tokens 56.9 instead of 52.1, one of 2,923 tokens 47.8 instead of 41.1.)
constexpr int kStart = 4;
constexpr int kJoinCost = 16;    // what cutting and joining costs
constexpr int kSnap = 2;         // shares begin no nearer to a block's ends, in tiles
constexpr int kMostRounds = 8;   // of whole blocks before the shares
constexpr int kIndex = 2048;     // entries of the planning workgroup's index of the blocks
constexpr int kDirectTiles = 24; // blocks of so few tiles are not planned
constexpr int kDirectBatch = 256, kDirectBlocks = 1 << 22;

// A block of a sequence's rows, for every key head. cost: of the blocks before it.
struct Block {
  int b, a, tiles, lq, lk, start;
  int64_t cost;
};
// What a workgroup does: whole blocks for `rounds` rounds, then its share, from tile t of a block of
// the hs-th of the heads that its workgroups take, up to another such place. blocks: number
// of blocks. first: the block that it begins with.
struct Turn {
  int hs, block, t, blocks;
  int hs1, block1, t1, rounds;
  Block first;
};
// A block that is cut: its first part is the end of share u - 1, the others begin shares u,
// u + 1, ..; n parts in all
struct Cut {
  int hs, u, n, a, lq, start, pad0, pad1;
};
struct PlanHead {
  int blocks, turns, cuts, whole;  // whole: no block is cut, a workgroup takes one block
};

// Workgroup w of the grid runs on XCD w % 8. The key heads are spread over the XCDs, in g
// classes (g the greatest common divisor of their number and 8); the 8 / g XCDs of a class take
// its heads one after the other, whose keys then stay in their L2.
struct Classes {
  int g, heads;  // heads of a class
  int held;      // workgroups of a class that run at a time
  static Classes of(int Hk, int per_unit) {
    int g = 8;
    while (Hk % g) g /= 2;
    return Classes{g, Hk / g, 8 / g * kXcdUnits * per_unit};
  }
};

// Bounds that the host knows, and where things lie in the workspace
struct Plan {
  int rows;        // of a block
  int slot_waves;  // wavefronts of a block that have rows, at most
  int blocks;      // at most, for one key head
  int direct;      // not planned: a workgroup takes one block, which it finds by itself
  size_t block_at, turn_at, cut_at, part_at, bytes;
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

// The order in which a block walks its tiles: the sinks', then the window's. Where the window of
// the sequence's last token begins inside this block's, from there to the last tile, and on from
// the first: blocks beside each other, whose windows are shifted, then read the same keys at a
// time (2 x 1,560 rows on windows of 4,679: 508 -> 503 us. Taken modulo the window's length
// by blocks further from the last token too: 178 -> 183 us for windows of 1,023).
struct BlockTiles {
  int ns, wrap, off, back;
  __device__ __forceinline__ BlockTiles() {}
  __device__ __forceinline__ BlockTiles(const WinMask& m, const TileList& l, int lk) {
    const int nw = l.n - l.ns, from = max(l.ns, max(0, lk - 1 - m.left) / KT) - l.b0;
    const int turn = from < nw ? from : 0;
    ns = l.ns;
    wrap = l.n - turn;
    off = l.b0 - l.ns + turn;
    back = off - nw;
  }
  __device__ __forceinline__ int tile(int t) const {
    return t + (t < ns ? 0 : t < wrap ? off : back);
  }
};

// Sum of x over the threads before this one, and over all of them
__device__ __forceinline__ int64_t plan_scan(int64_t x, int64_t (&sums)[kPlan / 64],
                                             int64_t* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int64_t in = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(in, o, 64);
    if (lane >= o) in += y;
  }
  __syncthreads();  // the sums of a scan before are read
  if (lane == 63) sums[w] = in;
  __syncthreads();
  int64_t before = in - x, all = 0;
#pragma unroll
  for (int i = 0; i < kPlan / 64; ++i) {
    if (i < w) before += sums[i];
    all += sums[i];
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

// a / b for a >= 0, b > 0: exact below 2^53, ascending in a beyond. (A division of 64-bit integers is
// a hundred instructions, which one workgroup fetches for one use: 0.4 to 0.6 us of a call.)
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (int64_t)((double)a / (double)b);
}

// One workgroup: lists the blocks by sequence, the last one (with most keys, if causal)
// first, then cuts their tiles into equal shares.
__global__ __launch_bounds__(kPlan) void chunk_plan_kernel(const ChunkProb P, const Plan L,
                                                           const Classes C, char* ws) {
  __shared__ int64_t sums[kPlan / 64];
  __shared__ int most_of[kPlan / 64];
  __shared__ int first[kPlan], s_n[kPlan], s_lq[kPlan], s_lk[kPlan], s_start[kPlan];
  __shared__ int64_t index[kIndex];  // cost of every 2^step-th block
  __shared__ int place[kMostHeld + 1], tile[kMostHeld + 1];  // where the shares begin
  __shared__ int n_cuts;
  Block* list = (Block*)(ws + L.block_at);
  Turn* turns = (Turn*)(ws + L.turn_at);
  Cut* cuts = (Cut*)(ws + L.cut_at);
  const int tid = threadIdx.x;
  int step = 0;
  while ((L.blocks >> step) >= kIndex) ++step;
  int64_t cost = 0;
  int seen = 0, longest = 0;  // seen: blocks so far, no more than the host counted
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
    int64_t total;
    const int64_t before = plan_scan(n, sums, &total);
    const int blocks = (int)min(total, (int64_t)(L.blocks - seen));
    first[tid] = (int)min(before, (int64_t)INT32_MAX);
    __syncthreads();
    for (int i0 = 0; i0 < blocks; i0 += kPlan) {
      const int i = i0 + tid;
      int tiles = 0, lo = 0, a = 0;
      if (i < blocks) {
        lo = plan_find(first, i);
        a = s_n[lo] - 1 - (i - first[lo]);
        const BlockSpan s(a, L.rows, P.G, s_lq[lo], s_lk[lo]);
        tiles = visible_tiles<KT>(P.m, s.p0, s.p1, s_lk[lo]).n;
        longest = max(longest, tiles + kStart);
      }
      const int64_t c = cost + plan_scan(i < blocks ? tiles + kStart : 0, sums, &total);
      if (i < blocks) {
        list[seen + i] = Block{b0 + lo, a, tiles, s_lq[lo], s_lk[lo], s_start[lo], c};
        if (((seen + i) & ((1 << step) - 1)) == 0) index[(seen + i) >> step] = c;
      }
      cost += total;
    }
    seen += blocks;
    __syncthreads();  // the segment's lists are read
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) longest = max(longest, __shfl_xor(longest, o, 64));
  if ((tid & 63) == 0) most_of[tid >> 6] = longest;
  if (tid == 0) n_cuts = 0;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kPlan / 64; ++x) longest = max(longest, most_of[x]);
  if (seen == 0) {
    if (tid == 0) *(PlanHead*)ws = PlanHead{0, 0, 0, 1};
    return;
  }
  // Whole blocks take as long as the longest one, and what does not fill a round leaves
  // workgroups idle: as much as a block if all are alike, next to nothing if they get
  // shorter (the shorter ones fill the gaps). Above what cutting costs (with many rounds
  // also that the workgroups no longer read the same keys at a time: a twentieth), blocks
  // are cut. (Measured while this was decided: 130 blocks of 112 tiles on each 64 workgroups 575
  // us whole, 535 cut; 64 of 33, causal, 1 to 64, 164 and 181; 256 of 450 3.58 and 3.75 ms.)
  const int64_t all = cost * C.heads, share = quotient(all, C.held);
  const int count = seen * C.heads, mean = (int)quotient(cost, seen), left = count % C.held;
  const int idle = left == 0 ? 0
                             : (int)quotient((int64_t)(C.held - left) * max(0, 2 * mean - longest), C.held);
  const bool whole = max((int64_t)longest - share, (int64_t)idle) <= kJoinCost + quotient(share, 20);
  if (whole) {
    if (tid == 0) *(PlanHead*)ws = PlanHead{seen, C.held, 0, 1};
    return;
  }
  // cost of the blocks before one
  auto before_block = [&](int i) -> int64_t {
    if (i == seen) return cost;
    if (step == 0) return index[i];
    return list[i].cost;
  };
  // cost of the class's blocks before the i-th
  auto cost_of = [&](int i) {
    const int h = i / seen;
    return h * cost + before_block(i - h * seen);
  };
  // (a share is what is left beside the whole blocks: some tiles for each workgroup, so that no two
  // shares begin at the same tile and every part of a block has some)
  int rounds = (int)max((int64_t)0, min((int64_t)kMostRounds, quotient(max(share - kShareTiles, (int64_t)0), longest)));
  int n = C.held;  // shares
  // One more round whole and the few blocks beside it in equal shares for as many workgroups as
  // get some tiles: less to join where that evens out the work as well (40 heads of 13 blocks
  // of 98 tiles, 512 at a time, 512 whole and 8 cut: 212 us; 520 cut: 231)
  int64_t rest = 0;
  bool even = true;
  if (rounds < kMostRounds && (int64_t)(rounds + 1) * C.held <= count) {
    rest = all - cost_of((rounds + 1) * C.held);
    if ((int64_t)(rounds + 1) * longest + quotient(rest, C.held) + kStart <= share + kJoinCost) {
      even = false;
      ++rounds;
      n = (int)max((int64_t)1, min((int64_t)n, min(rest / kShareTiles, quotient(kMostParts * rest, longest))));
    }
  }
  // Few tiles: fewer shares (the joining of more parts of a block costs more than they save), as
  // many on each compute unit
  if (rounds == 0) {
    const int units = 8 / C.g * kXcdUnits;
    n = (int)min((int64_t)n, min((all + kShareTiles - 1) / kShareTiles, 1 + quotient(kMostParts * all, longest)));
    if (n > units) n -= n % units;
  }
  const int turn = rounds > 0 ? C.held : n;  // workgroups that have something to do
  if (tid == 0) *(PlanHead*)ws = PlanHead{seen, turn, 0, 0};
  for (int u = tid; u <= turn; u += kPlan) {
    int hs = C.heads, block = 0, t = 0;
    if (u < n) {
      // all workgroups' whole blocks, what the shares before leave to be done by the
      // workgroups before u beside their own whole blocks
      int64_t pos = even ? quotient(all * u, n) : cost_of(rounds * C.held) + quotient(rest * u, n);
      if (even && rounds > 0) {
        pos += cost_of(rounds * C.held);
        for (int k = 0; k < rounds; ++k) pos -= cost_of(k * C.held + u) - cost_of(k * C.held);
      }
      hs = (int)quotient(pos, cost);
      const int64_t off = pos - hs * cost;
      int lo = 0, hi = ((seen - 1) >> step) + 1;  // index[lo] <= off < index[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (index[mid] <= off)
          lo = mid;
        else
          hi = mid;
      }
      hi = min((lo + 1) << step, seen);
      lo <<= step;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (list[mid].cost <= off)
          lo = mid;
        else
          hi = mid;
      }
      block = lo;
      const int64_t c = before_block(lo), e = before_block(lo + 1);
      t = max(0, (int)(off - c) - kStart);
      if (t < kSnap) t = 0;
      if (t > 0 && (int)(e - c) - kStart - t < kSnap) {  // at the next block's beginning instead
        t = 0;
        if (++block == seen) {
          block = 0;
          ++hs;
        }
      }
    }
    place[u] = hs * seen + block;
    tile[u] = t;
    Turn* x = turns + u;
    if (u < turn) {
      x->hs = hs;
      x->block = block;
      x->t = t;
      x->blocks = seen;
      x->rounds = rounds;
      x->first = list[rounds > 0 ? u % seen : block];
    }
    if (u > 0) {
      x[-1].hs1 = hs;
      x[-1].block1 = block;
      x[-1].t1 = t;
    }
  }
  __syncthreads();
  for (int u = 1 + tid; u < n; u += kPlan) {
    const int at = place[u], h = at / seen;
    if (tile[u] == 0 || (tile[u - 1] > 0 && place[u - 1] == at)) continue;
    int lo = u, hi = n;  // share lo begins in the block, share hi after it
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (place[mid] == at)
        lo = mid;
      else
        hi = mid;
    }
    const Block b = list[at - h * seen];
    cuts[atomicAdd(&n_cuts, 1)] = Cut{h, u, lo - u + 2, b.a, b.lq, b.start, 0, 0};
  }
  __syncthreads();
  if (tid == 0) ((PlanHead*)ws)->cuts = n_cuts;
}

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

// What the attention kernels are called with. They read it anew for each piece of work and after
// its walk (args()): kept in registers over the walk, which needs nearly all that there are,
// it would be spilled.
struct ChunkArgs {
  ChunkProb P;
  Plan L;
  Classes C;
  FastDiv by_page;
  float sl2;
  const void *q, *kp, *vp;
  void* out;
  float* lse;
  char* ws;
};
typedef const __attribute__((address_space(4))) ChunkArgs* Args;
__device__ __forceinline__ Args args() {
  Args a = (Args)__builtin_amdgcn_kernarg_segment_ptr();  // the only argument
  asm volatile("" : "+s"(a));
  return a;
}

// Tiles [t0, t1) of a block. slot: where the softmax state of a part goes, -1 for a whole block.
struct Piece {
  int b, a, t0, t1, slot, lq, lk, start;
};
// A workgroup's pieces of work, one after the other. (What the launch before wrote is read from
// the constant address space, by scalar loads.)
template <int ROWS>
struct Pieces {
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  typedef int i32x8 __attribute__((ext_vector_type(8)));
  typedef int i32x16 __attribute__((ext_vector_type(16)));
  typedef const __attribute__((address_space(4))) i32x4* Heads;
  typedef const __attribute__((address_space(4))) i32x8* Blocks;
  typedef const __attribute__((address_space(4))) i32x16* Turns;
  Piece it;                           // the piece
  int hs, block, t, hs1, block1, t1;  // from here to there
  int k, rounds, u, cls, n;           // k: ranges done

  __device__ __forceinline__ void set(i32x8 x) {  // x: Block
    const int end = hs == hs1 && block == block1 ? t1 : x[2];
    it = Piece{x[0], x[1], t, end, t == 0 && end == x[2] ? -1 : 2 * u + (t == 0), x[3], x[4], x[5]};
  }
  __device__ __forceinline__ void load() {
    const Args A = args();
    set(((Blocks)(A->ws + A->L.block_at))[block]);
  }
  // the i-th block of the class's as a whole
  __device__ __forceinline__ bool whole(int i) {
    hs = i / n;
    block = i - hs * n;
    hs1 = hs;
    block1 = block + 1;
    t = t1 = 0;
    return hs < args()->C.heads;
  }
  __device__ __forceinline__ void share(i32x16 x) {  // x: Turn
    hs = x[0];
    block = x[1];
    t = x[2];
    hs1 = x[4];
    block1 = x[5];
    t1 = x[6];
  }
  __device__ __forceinline__ bool more() const {
    return hs < hs1 || (hs == hs1 && (block < block1 || (block == block1 && t < t1)));
  }
  __device__ __forceinline__ int head() const { return hs * args()->C.g + cls; }

  // false: no work
  __device__ __forceinline__ bool first() {
    const Args A = args();
    const int g = A->C.g;
    cls = (blockIdx.x & 7) % g;
    u = (blockIdx.x >> 3) * (8 / g) + (blockIdx.x & 7) / g;
    k = 0;
    rounds = -1;
    if (A->L.direct) return direct(A);
    const i32x4 h = *(Heads)A->ws;  // PlanHead
    const i32x16 x = ((Turns)(A->ws + A->L.turn_at))[min(u, A->C.held - 1)];
    n = h[0];
    if (n == 0) return false;
    if (h[3]) {
      if (!whole(u)) return false;
      load();
      return true;
    }
    if (u >= h[1]) return false;
    rounds = x[7];
    if (rounds > 0)
      whole(u);
    else
      share(x);
    if (!more()) return false;
    set(i32x8{x[8], x[9], x[10], x[11], x[12], x[13], x[14], x[15]});
    return true;
  }
  __device__ __forceinline__ bool next() {
    if (hs == hs1 && block == block1) {
      t = t1;  // the end
    } else {
      t = 0;
      if (++block == n && hs < hs1) {
        block = 0;
        ++hs;
      }
    }
    if (!more()) {
      ++k;
      if (k > rounds) return false;
      if (k < rounds) {
        whole(k * args()->C.held + u);
      } else {
        const Args A = args();
        share(((Turns)(A->ws + A->L.turn_at))[u]);
        if (!more()) return false;
      }
    }
    load();
    return true;
  }
  // Block u of the class's, found from the lengths: a lane has four sequences
  __device__ __forceinline__ bool direct(const Args A) {
    constexpr int S = kDirectBatch / 64;
    const int lane = threadIdx.x & 63, B = A->P.B, T = A->P.tokens, G = A->P.G;
    int start[S], lq[S], lk[S], blocks[S], mine = 0;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const int b = S * lane + i;
      start[i] = lq[i] = lk[i] = 0;
      if (b < B) {
        start[i] = min(max(A->P.starts[b], 0), T);
        lq[i] = max(0, min(max(A->P.starts[b + 1], 0), T) - start[i]);
        lk[i] = (int)min((int64_t)max(A->P.lens[b], 0), (int64_t)A->P.max_pages * A->P.page);
      }
      // (no more than the launch can have, so that the sum of starts that do not ascend fits)
      blocks[i] = min((int)(((uint32_t)lq[i] * (uint32_t)G + ROWS - 1) / ROWS), kDirectBlocks);
      mine += blocks[i];
    }
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(sum, o, 64);
      if (lane >= o) sum += y;
    }
    n = __builtin_amdgcn_readlane(sum, 63);
    if (n <= 0 || n > A->L.blocks || !whole(u)) return false;
    const int l = __builtin_ctzll(__builtin_amdgcn_ballot_w64(sum > block));
    int i = block - (__builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(mine, l));
    bool found = false;
    it = Piece{0, 0, 0, 0, -1, 0, 0, 0};
#pragma unroll
    for (int x = 0; x < S; ++x) {
      const int c = __builtin_amdgcn_readlane(blocks[x], l);
      if (!found && i < c) {
        found = true;
        it = Piece{S * l + x, c - 1 - i, 0, 0, -1, __builtin_amdgcn_readlane(lq[x], l),
                   __builtin_amdgcn_readlane(lk[x], l), __builtin_amdgcn_readlane(start[x], l)};
      }
      i -= c;
    }
    if (!found) return false;
    const BlockSpan s(it.a, ROWS, G, it.lq, it.lk);
    it.t1 = visible_tiles<KT>(WinMask{A->P.m.left, A->P.m.right, A->P.m.sinks, A->P.m.causal}, s.p0,
                              s.p1, it.lk)
                .n;
    return true;
  }
};

// State of a part, wavefront by wavefront as its lanes hold it: `chunks` times four sums a
// lane, its row's reference (log2 units) and sum of exponentials
__device__ __forceinline__ float* part_wave(char* parts, int held, int slot_waves, int cls, int slot,
                                            int w, int chunks) {
  return (float*)parts + (((size_t)cls * 2 * held + slot) * slot_waves + w) * (64 * (4 * chunks + 2));
}

// ---- bf16 ---------------------------------------------------------------------------------

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

typedef const __attribute__((address_space(4))) int32_t* Entries;

// Copies of 1024 bytes each, one after the other in LDS, with one write of the LDS base (M0): an
// instruction's offset moves both addresses, so lane offset c is 1024 c less than where its
// bytes lie.
template <int N>
__device__ __forceinline__ void lds_dma16_run(const void* gbase, const uint32_t (&voff)[N],
                                              uint32_t lds) {
  static_assert(N == 2 || N == 4, "copies of a group of rows");
  uint32_t saved;
  if constexpr (N == 2)
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %4\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %3\n\t"
        "global_load_lds_dwordx4 %2, %3 offset:0x400\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(voff[0]), "v"(voff[1]), "s"(gbase), "s"(lds)
        : "memory");
  else
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %6\n\t"
        "s_nop 0\n\t"
        "global_load_lds_dwordx4 %1, %5\n\t"
        "global_load_lds_dwordx4 %2, %5 offset:0x400\n\t"
        "global_load_lds_dwordx4 %3, %5 offset:0x800\n\t"
        "global_load_lds_dwordx4 %4, %5 offset:0xc00\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(voff[0]), "v"(voff[1]), "v"(voff[2]), "v"(voff[3]), "s"(gbase), "s"(lds)
        : "memory");
}

// Tiles whose rows lie on pages. Wavefront w copies rows 16 w .. 16 w + 15 of a
// tile. GROUPS: pages of a multiple of 16 tokens, so that the sixteen lie on one page,
// whose entry is one scalar load (from the constant address space: no kernel writes the
// table while this one runs); else a lane looks up its row's entry. Entries are
// loaded a tile before the copies that need them. The scalar work of a tile is on its
// wavefront's path: a row group's place is found once, for keys and values, and its copies
// share one LDS base (211 -> 134 scalar instructions a tile, 2% of the time).
template <int D, bool GROUPS>
struct PagedTiles : WalkRows {
  static constexpr bool kHoles = true, kBegun = true;
  static constexpr float kMostSum = 0x1p30f;
  static constexpr int RB = 2 * D, TILE = KT * RB, NI = RB / 64, RPI = 1024 / RB;
  // Where a wavefront's rows of a tile lie: the entry (of this lane's row without GROUPS), the
  // first row's place on the page, and how many keys come after it
  struct Place {
    int e, in, last;
  };
  const bf16 *kh, *vh;  // of this key head
  const int32_t* table;
  int64_t k_sp, k_st, v_sp, v_st;
  int page, pages, most;  // most: last entry of the row
  FastDiv by_page;
  char* smem;
  uint16_t (*hole)[4];
  uint32_t lds0;
  int w, lane;
  Place pv, pk;  // of the tile whose values, and of the one whose keys are next
  BlockTiles order;

  __device__ __forceinline__ int tile(int t) const { return order.tile(t); }
  __device__ __forceinline__ int key(int t) const {
    return KT * tile(t) + 16 * w + (GROUPS ? 0 : lane & 15);
  }
  __device__ __forceinline__ Place place(int t) const {
    const int j = key(t), n = min(j, lk - 1), i = by_page.div(n), at = min(i, most);
    if constexpr (GROUPS)
      return Place{((Entries)table)[__builtin_amdgcn_readfirstlane(at)], n - i * page, lk - 1 - j};
    else
      return Place{table[at], 0, 0};  // (the others are vectors: formed anew, not kept)
  }
  // keys (V false) or values of tile t, which lies at p, into LDS tile `at`
  template <bool V>
  __device__ __forceinline__ void copy(int t, const Place& p, int at, int buf) const {
    const bf16* base = V ? vh : kh;
    const int64_t sp = V ? v_sp : k_sp, st = V ? v_st : k_st;
    const uint32_t dst = lds0 + at * TILE + 1024 * NI * w;
    const int row = lane / (RB / 16), e = p.e;
    auto chunk = [&](int c) __attribute__((always_inline)) {
      return ((lane % (RB / 16)) ^ row_key<RB>(RPI * c + row)) << 4;
    };
    auto nothing = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < NI; ++c)
        *(f32x4*)(smem + at * TILE + 1024 * (NI * w + c) + 16 * lane) = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    const bool there = e >= 0 && e < pages;
    if constexpr (GROUPS) {
      if (!V && lane == 0) hole[buf][w] = there || p.last < 0 ? 0 : 0xffff;
      if (!there || p.last < 0) {
        nothing();
        return;
      }
      // (a page takes less than 2^32 bytes)
      const char* src = (const char*)base + (uint64_t)(uint32_t)e * (uint32_t)(2 * sp) +
                        (uint64_t)(uint32_t)p.in * (uint32_t)(2 * st);
      const uint32_t rb = (uint32_t)st * 2;
      if (p.last >= 15) {
        uint32_t off[NI];
#pragma unroll
        for (int c = 0; c < NI; ++c) off[c] = (uint32_t)row * rb + chunk(c) + c * (RPI * rb - 1024);
        lds_dma16_run<NI>(src, off, __builtin_amdgcn_readfirstlane(dst));
      } else {  // rows past the last are copies of it
#pragma unroll
        for (int c = 0; c < NI; ++c)
          lds_dma16(src, (uint32_t)min(RPI * c + row, p.last) * rb + chunk(c),
                    __builtin_amdgcn_readfirstlane(dst + 1024 * c));
      }
    } else {
      const int j = key(t), n = min(j, lk - 1), in = n - by_page.div(n) * page;
      const uint32_t any = (uint32_t)__builtin_amdgcn_ballot_w64(there) & 0xffff;
      const uint32_t gone = (uint32_t)__builtin_amdgcn_ballot_w64(!there && j < lk) & 0xffff;
      if (!V && lane == 0) hole[buf][w] = (uint16_t)gone;
      if (any == 0) {
        nothing();
        return;
      }
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
  __device__ __forceinline__ void issue_k(int t, int buf) { copy<false>(t, pk, buf, buf); }
  __device__ __forceinline__ void issue_v(int t, int buf) {
    copy<true>(t, pv, 2 + buf, buf);
    pv = pk;
    pk = place(min(t + 2, t1 - 1));
  }
  // the first tile's keys and values and the second's keys, before the walk: with the queries
  __device__ __forceinline__ void begin() {
    if (t0 >= t1) return;
    const Place p = place(t0);
    pv = place(min(t0 + 1, t1 - 1));
    pk = place(min(t0 + 2, t1 - 1));
    copy<false>(t0, p, 0, 0);
    copy<true>(t0, p, 2, 0);
    if (t0 + 1 < t1) copy<false>(t0 + 1, pv, 1, 1);
  }
  __device__ __forceinline__ void issue_both(int t) const {
    const Place p = place(t);
    copy<false>(t, p, 0, 0);
    copy<true>(t, p, 2, 0);
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
    const ChunkArgs) {
  constexpr int KS = D / 16, DT = D / 32, RB = 2 * D, TILE = KT * RB;
  __shared__ __attribute__((aligned(1024))) char smem[4 * TILE];  // two tiles of keys, two of values
  __shared__ __attribute__((aligned(8))) uint16_t hole[2][4];
  __shared__ int redo;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Pieces<kWalkRows> S;
  for (bool go = S.first(); go; go = S.next()) {
    const Piece it = S.it;
    const int hk = S.head();
    __syncthreads();  // every wavefront is past the piece before
    const Args A = args();
    const int G = A->P.G, off = it.lk - it.lq, rows = it.lq * G;
    const int w0 = it.a * kWalkRows + 32 * w, wreal = max(0, min(32, rows - w0));
    // the wavefront's last row, this lane's
    const int wl = min(w0 + max(wreal, 1), rows) - 1, row = min(w0 + l32, wl);
    const BlockSpan span(it.a, kWalkRows, G, it.lq, it.lk);
    PagedTiles<D, GROUPS> T;
    T.mask = WinMask{A->P.m.left, A->P.m.right, A->P.m.sinks, A->P.m.causal};
    T.list = visible_tiles<KT>(T.mask, span.p0, span.p1, it.lk);
    T.order = BlockTiles(T.mask, T.list, it.lk);
    T.t0 = it.t0;
    T.t1 = it.t1;
    T.lk = it.lk;
    T.ra = visible_keys(T.mask, min(w0, wl) / G + off, it.lk);
    T.rz = visible_keys(T.mask, wl / G + off, it.lk);
    T.pos = row / G + off;
    T.real = wreal;
    T.block_first = span.p0;
    T.block_last = span.p1;
    T.kh = (const bf16*)A->kp + hk * A->P.k_sh;
    T.vh = (const bf16*)A->vp + hk * A->P.v_sh;
    T.table = A->P.table + it.b * A->P.table_sb;
    T.k_sp = A->P.k_sp;
    T.k_st = A->P.k_st;
    T.v_sp = A->P.v_sp;
    T.v_st = A->P.v_st;
    T.page = A->P.page;
    T.pages = A->P.pages;
    T.most = A->P.max_pages - 1;
    T.by_page = FastDiv{A->by_page.m, A->by_page.s};
    T.smem = smem;
    T.hole = hole;
    T.lds0 = lds_addr(smem);
    T.w = w;
    T.lane = lane;
    T.pv = T.pk = {0, 0, 0};

    bf16x8 qreg[KS];
    {
      const int tok = row / G, head = hk * G + row - tok * G;
      const bf16* src = (const bf16*)A->q + (it.start + tok) * A->P.q_st + head * A->P.q_sh;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) qreg[kk] = *(const bf16x8*)(src + 16 * kk + 8 * h);
    }
    T.begin();
    // Retire the loads here (a wait the compiler sees), so that no vmcnt wait of
    // theirs lands in the loop, where it would also wait for the copies in flight.
    __builtin_amdgcn_s_waitcnt(kWalkVmcnt0);
    if (tid == 0) redo = 0;  // ordered before any write by the barriers of the tiles
    f32x16 oacc[DT];
    float m, l_tot;
    walk_bf16<D>(T, smem, &redo, qreg, A->sl2, w, lane, oacc, m, l_tot);
    const Args B = args();
    if (it.slot >= 0) {
      if (wreal == 0) continue;
      // A sum far above its reference goes out against a reference at its own size: the
      // joining compares references, and adds up as many sums as there are parts
      const int up = l_tot > 0x1p22f ? __builtin_amdgcn_frexp_expf(l_tot) : 0;
      float* x = part_wave(B->ws + B->L.part_at, B->C.held, B->L.slot_waves, S.cls, it.slot, w, D / 8) +
                 4 * lane;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          f32x4 y;
#pragma unroll
          for (int j = 0; j < 4; ++j) y[j] = __builtin_amdgcn_ldexpf(oacc[dt][4 * g + j], -up);
          *(f32x4*)(x + 256 * (4 * dt + g)) = y;
        }
      x += 32 * D - 3 * lane;
      x[0] = m + (float)up;
      x[64] = __builtin_amdgcn_ldexpf(l_tot, -up);
      continue;
    }
    if (l32 >= wreal) continue;
    const bool any = l_tot != 0.f;
    const float inv = any ? 1.f / l_tot : 0.f;
    const int tok = row / G, head = hk * G + row - tok * G;
    bf16* orow = (bf16*)B->out + (it.start + tok) * B->P.o_st + head * B->P.o_sh;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        bf16x4 x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = f2bf(any ? oacc[dt][4 * g + j] * inv : 0.f);
        *(bf16x4*)(orow + 32 * dt + 8 * g + 4 * h) = x;
      }
    if (B->lse && h == 0)
      B->lse[(size_t)(it.start + tok) * B->P.H + head] =
          any ? (m + __builtin_amdgcn_logf(l_tot)) * kLn2 : -INFINITY;
  }
}

// ---- joining the parts --------------------------------------------------------------------

// A workgroup joins the rows of one wavefront, lanes as they were in the attention. Of few
// parts its wavefronts take a quarter of the chunks each, of many every fourth part, and the
// quarters are workgroups of their own. (The whole call, taken for few and for many: one block in
// 8 parts 22.0 and 21.3 us, four ragged sequences in fp32 in up to 8 55.2 and 56.0; 13 parts 22.5 and
// 21.8, 25 parts 24.9 and 21.7, 48 parts 30.4 and 23.0, 128 parts 60.5 and 40.7.)
constexpr int kJoinGrid = 8192, kFewParts = 8;

template <typename T, int D>
__global__ __launch_bounds__(256) void chunk_join_kernel(const ChunkProb P, const Plan L,
                                                         const Classes C, char* __restrict__ ws,
                                                         T* __restrict__ out,
                                                         float* __restrict__ lse) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int CH = BF ? D / 8 : D / 16, JC = CH < 4 ? 1 : CH / 4;
  constexpr int WR = BF ? 32 : 16, NG = CH / JC;  // rows of a wavefront, groups of chunks
  __shared__ __attribute__((aligned(16))) f32x4 acc[4][JC][64];
  __shared__ float ms[4][64], ls[4][64];
  const int lane = threadIdx.x & 63, lr = lane % WR;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_cuts = ((const PlanHead*)ws)->cuts, each = L.slot_waves * NG;
  for (int c = blockIdx.x; c < n_cuts * C.g * each; c += gridDim.x) {
    // (groups go slowest: of few parts the first n_cuts * g * slot_waves have work)
    const int gr = c / (n_cuts * C.g * L.slot_waves), x = c - gr * n_cuts * C.g * L.slot_waves;
    const int y = x / L.slot_waves, wv = x - y * L.slot_waves, cls = y / n_cuts;
    const Cut cut = ((const Cut*)(ws + L.cut_at))[y - cls * n_cuts];
    const int row = cut.a * L.rows + wv * WR + lr, rows = cut.lq * P.G;
    const bool few = cut.n <= kFewParts;
    // the wavefront had no rows; another workgroup's, or wavefront's
    if (row - lr >= rows || (few && gr > 0)) continue;
    const int j0 = (few ? w : gr) * JC;
    float m = -INFINITY, l = 0.f;
    f32x4 a[JC];
#pragma unroll
    for (int j = 0; j < JC; ++j) a[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto merge = [&](float m2, float l2, const f32x4* v) __attribute__((always_inline)) {
      // no key of the part is there: its reference is not one
      const float m1 = l2 == 0.f ? m : fmaxf(m, m2), ref = m1 == -INFINITY ? 0.f : m1;
      const float f = __builtin_amdgcn_exp2f(m - ref);
      const float h = l2 == 0.f ? 0.f : __builtin_amdgcn_exp2f(m2 - ref);
      l = l * f + l2 * h;
#pragma unroll
      for (int j = 0; j < JC; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) a[j][e] = a[j][e] * f + v[j][e] * h;
      m = m1;
    };
    // part 0 lies in slot 2 u - 1, parts 1, 2, .. in slots 2 u, 2 u + 2, ..
    if (!few || w < NG) {
#pragma unroll 4
      for (int i = few ? 0 : w; i < cut.n; i += few ? 1 : 4) {
        const float* p = part_wave(ws + L.part_at, C.held, L.slot_waves, cls,
                                   2 * (cut.u + i - 1) + (i == 0), wv, CH);
        f32x4 v[JC];
#pragma unroll
        for (int j = 0; j < JC; ++j) v[j] = *(const f32x4*)(p + 256 * (j0 + j) + 4 * lane);
        merge(p[256 * CH + lane], p[256 * CH + 64 + lane], v);
      }
    }
    if (!few) {
      __syncthreads();  // the states before are read
      if (w > 0) {
#pragma unroll
        for (int j = 0; j < JC; ++j) acc[w][j][lane] = a[j];
        ms[w][lane] = m;
        ls[w][lane] = l;
      }
      __syncthreads();
      if (w > 0) continue;
      for (int i = 1; i < 4; ++i) {
        f32x4 v[JC];
#pragma unroll
        for (int j = 0; j < JC; ++j) v[j] = acc[i][j][lane];
        merge(ms[i][lane], ls[i][lane], v);
      }
    }
    if (row >= rows || (few && w >= NG)) continue;
    const int tok = row / P.G, h = (cut.hs * C.g + cls) * P.G + row - tok * P.G;
    T* o = out + (cut.start + tok) * P.o_st + h * P.o_sh;
    const float inv = 1.f / l;
#pragma unroll
    for (int j = 0; j < JC; ++j) {
      const int dim = 4 * (64 / WR * (j0 + j) + lane / WR);
      if (dim >= P.d) continue;
      f32x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = l != 0.f ? a[j][e] * inv : 0.f;
      if constexpr (BF)
        *(bf16x4*)(o + dim) = bf16x4{f2bf(y[0]), f2bf(y[1]), f2bf(y[2]), f2bf(y[3])};
      else
        *(f32x4*)(o + dim) = y;
    }
    if (lse && j0 == 0 && lane < WR)
      lse[(size_t)(cut.start + tok) * P.H + h] =
          l != 0.f ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  }
}

// ---- fp32 ---------------------------------------------------------------------------------
//
// One wavefront per 16 rows, on the fp32 matrix instructions (v_mfma_f32_16x16x4_f32): S^T =
// K Q^T leaves lane l with row l % 16 and the logits of keys 4 (l / 16) + r, which is
// the P^T operand of O^T = V^T P^T as it stands. Half tiles of 32 keys go through registers
// to LDS, one ahead of the one that is computed; rows of DP + 4 floats there spread the keys'
// 16-byte reads and the values' 4-byte reads over the banks (counted: conflicts are 19% of the
// cycles in which LDS is active, these 7% of all). What bounds it: the matrix instructions, 32
// cycles each and busy 68% of the time (8,192 causal tokens, 8 heads of 64: 702 us, 98 TFLOP/s of
// the 154 of a large product), or the cache (8 single tokens on 16,000 each, 32 heads on 8 of 128:
// 237 us, 4.4 TB/s).

// The largest x of lanes l, l ^ 16, l ^ 32 and l ^ 48
__device__ __forceinline__ float max_of_groups(float x) {
  auto larger = [](uint32_t a, uint32_t b) {
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
  };
  uint32_t y = __builtin_bit_cast(uint32_t, x);
  const auto a = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  y = __builtin_bit_cast(uint32_t, larger(a[0], a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(y, y, false, false);
  return larger(b[0], b[1]);
}

template <int DP, int WAVES, bool GROUPS>
__global__ __launch_bounds__(256, WAVES) void chunk_f32_kernel(
    const ChunkArgs) {
  constexpr int HK = 32, NJ = DP / 16, LD = DP + 4, NC = DP / 4;
  constexpr int RP = 64 / NC, NP = 8 / RP;  // rows of a wavefront's pass of the copy, passes
  __shared__ __attribute__((aligned(16))) float ks[2][HK][LD], vs[2][HK][LD];
  __shared__ uint32_t gone[4], bad[4];  // keys not there, values that are not finite
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, l16 = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Pieces<kF32Rows> S;
  for (bool go = S.first(); go; go = S.next()) {
    const Piece it = S.it;
    const int hk = S.head();
    __syncthreads();  // every wavefront is past the piece before
    const Args A = args();
    const int G = A->P.G, d = A->P.d, off = it.lk - it.lq, rows = it.lq * G;
    const WinMask mask{A->P.m.left, A->P.m.right, A->P.m.sinks, A->P.m.causal};
    const BlockSpan span(it.a, kF32Rows, G, it.lq, it.lk);
    const BlockTiles list(mask, visible_tiles<KT>(mask, span.p0, span.p1, it.lk), it.lk);
    const int w0 = it.a * kF32Rows + 16 * w, wreal = max(0, min(16, rows - w0));
    // the wavefront's last row, this lane's
    const int wl = min(w0 + max(wreal, 1), rows) - 1, row = min(w0 + l16, wl);
    const KeyRange ra = visible_keys(mask, min(w0, wl) / G + off, it.lk);
    const KeyRange rz = visible_keys(mask, wl / G + off, it.lk);
    const KeyRange mine = visible_keys(mask, row / G + off, it.lk);
    const float sl2 = A->sl2;

    f32x4 qf[NJ];
    {
      const int tok = row / G, head = hk * G + row - tok * G;
      const float* src = (const float*)A->q + (it.start + tok) * A->P.q_st + head * A->P.q_sh;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int x = 16 * j + 4 * g;
        qf[j] = x < d ? *(const f32x4*)(src + x) : f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
    const int32_t* table = A->P.table + it.b * A->P.table_sb;
    const float *kh = (const float*)A->kp + hk * A->P.k_sh, *vh = (const float*)A->vp + hk * A->P.v_sh;
    const int64_t k_sp = A->P.k_sp, k_st = A->P.k_st, v_sp = A->P.v_sp, v_st = A->P.v_st;
    const int page = A->P.page, pages = A->P.pages;
    const FastDiv by_page{A->by_page.m, A->by_page.s};
    const int n = 2 * (it.t1 - it.t0);  // half tiles
    auto first_key = [&](int i) __attribute__((always_inline)) {
      return KT * list.tile(it.t0 + (i >> 1)) + HK * (i & 1);
    };
    // A wavefront copies rows 8 w .. 8 w + 7 of a half tile, RP of them a pass: this lane's piece of
    // a row, and its row in the first pass. Their entries are loaded a half tile before the rows.
    // GROUPS: pages of a multiple of 8 tokens, so that the eight lie on one page, whose entry
    // is one scalar load and whose place is found once (one for each pass: 284 us instead of 245
    // for 8 tokens on 16,000 each, 32 heads on 8 of 128).
    const int cc = 4 * (lane % NC), lr = lane / NC, cr = 8 * w + lr;
    uint32_t k_off[NP], v_off[NP];  // bytes
#pragma unroll
    for (int x = 0; x < NP; ++x) {
      k_off[x] = GROUPS ? (uint32_t)((lr + x * RP) * k_st + cc) * 4 : 0;
      v_off[x] = GROUPS ? (uint32_t)((lr + x * RP) * v_st + cc) * 4 : 0;
    }
    int ent[GROUPS ? 1 : NP], in = 0;
    auto entries = [&](int j0) __attribute__((always_inline)) {  // j0: the half tile's first key
      if constexpr (GROUPS) {
        const int j = min(j0 + 8 * w, it.lk - 1), e = by_page.div(j);
        ent[0] = ((Entries)table)[__builtin_amdgcn_readfirstlane(e)];
        in = j - e * page;
      } else {
#pragma unroll
        for (int x = 0; x < NP; ++x) ent[x] = table[by_page.div(min(j0 + cr + x * RP, it.lk - 1))];
      }
    };
    f32x4 kr[NP], vr[NP];
    uint32_t missing;
    auto load = [&](int first) __attribute__((always_inline)) {
      missing = 0;
#pragma unroll
      for (int x = 0; x < NP; ++x) kr[x] = vr[x] = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (GROUPS) {
        const int j0 = first + 8 * w, e = ent[0];
        if (j0 >= it.lk) return;
        if (e < 0 || e >= pages) {
          missing = 0xffu << (8 * w);
          return;
        }
        const char* ks0 = (const char*)kh + (uint64_t)(uint32_t)e * (uint32_t)(4 * k_sp) +
                          (uint64_t)(uint32_t)in * (uint32_t)(4 * k_st);
        const char* vs0 = (const char*)vh + (uint64_t)(uint32_t)e * (uint32_t)(4 * v_sp) +
                          (uint64_t)(uint32_t)in * (uint32_t)(4 * v_st);
        if (j0 + 8 <= it.lk && d == DP) {
#pragma unroll
          for (int x = 0; x < NP; ++x) kr[x] = *(const f32x4*)(ks0 + k_off[x]);
#pragma unroll
          for (int x = 0; x < NP; ++x) vr[x] = *(const f32x4*)(vs0 + v_off[x]);
        } else {
#pragma unroll
          for (int x = 0; x < NP; ++x)
            if (j0 + lr + x * RP < it.lk && cc < d) {
              kr[x] = *(const f32x4*)(ks0 + k_off[x]);
              vr[x] = *(const f32x4*)(vs0 + v_off[x]);
            }
        }
      } else {
        const int j0 = first + cr;
#pragma unroll
        for (int x = 0; x < NP; ++x) {
          const int j = j0 + x * RP, e = ent[x], at = j - by_page.div(min(j, it.lk - 1)) * page;
          if (j >= it.lk) continue;
          if (e < 0 || e >= pages) {
            missing |= 1u << (cr + x * RP);
          } else if (cc < d) {
            kr[x] = *(const f32x4*)(kh + e * k_sp + at * k_st + cc);
            vr[x] = *(const f32x4*)(vh + e * v_sp + at * v_st + cc);
          }
        }
      }
    };
    auto store = [&](int i) __attribute__((always_inline)) {
      if (missing) atomicOr(&gone[i & 3], missing);
#pragma unroll
      for (int x = 0; x < NP; ++x) *(f32x4*)&ks[i & 1][cr + x * RP][cc] = kr[x];
#pragma unroll
      for (int x = 0; x < NP; ++x) {
        // 0, or NaN if a value is not finite
        const float z = fmaf(vr[x][0], 0.f, vr[x][1] * 0.f) + fmaf(vr[x][2], 0.f, vr[x][3] * 0.f);
        if (__builtin_expect(z != 0.f, 0)) {
          // zero times it would reach rows that do not see it: those that do get NaN at the end
          atomicOr(&bad[i & 3], 1u << (cr + x * RP));
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!(fabsf(vr[x][e]) < INFINITY)) vr[x][e] = 0.f;
        }
        *(f32x4*)&vs[i & 1][cr + x * RP][cc] = vr[x];
      }
    };
    f32x4 o[NJ];
    float m = -INFINITY, l = 0.f;  // reference (log2 units), this lane's part of the sum
    bool poison = false;
#pragma unroll
    for (int j = 0; j < NJ; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto compute = [&](int i, int k0) __attribute__((always_inline)) {
      // no row sees a key; every row sees all
      if (k0 >= rz.s_end && (k0 >= rz.hi || k0 + HK <= ra.lo)) return;
      const uint32_t hv = __builtin_amdgcn_readfirstlane(gone[i & 3]);
      const uint32_t bv = __builtin_amdgcn_readfirstlane(bad[i & 3]);
      const bool all = (k0 + HK <= ra.s_end || (k0 >= rz.lo && k0 + HK <= ra.hi)) && hv == 0;
      const float(*kt)[LD] = ks[i & 1];
      const float(*vt)[LD] = vs[i & 1];
      // four partial sums a logit: shorter chains of rounded sums
      // products go before the other wavefronts' exponentials (1 to 2% of the time)
      __builtin_amdgcn_s_setprio(2);
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
      __builtin_amdgcn_s_setprio(0);
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
      mx = max_of_groups(mx) * sl2;
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
      int k0 = first_key(0), k1 = first_key(1);  // first keys of half tiles i and i + 1
      entries(k0);
      load(k0);
      entries(k1);
      store(0);
      __syncthreads();
      for (int i = 0; i < n; ++i) {
        const int k2 = first_key(min(i + 2, n - 1));
        if (i + 1 < n) load(k1);
        entries(k2);
        // the flags of half tile i + 2 (those of i - 2 were read before the last barrier)
        if (tid == 0) gone[(i + 2) & 3] = bad[(i + 2) & 3] = 0;
        if (wreal) compute(i, k0);
        k0 = k1;
        k1 = k2;
        if (i + 1 < n) store(i + 1);
        __syncthreads();
      }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (poison) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) o[j] = f32x4{NAN, NAN, NAN, NAN};
    }
    const Args B = args();
    if (it.slot >= 0) {
      if (wreal == 0) continue;
      float* x = part_wave(B->ws + B->L.part_at, B->C.held, B->L.slot_waves, S.cls, it.slot, w, NJ) +
                 4 * lane;
#pragma unroll
      for (int j = 0; j < NJ; ++j) *(f32x4*)(x + 256 * j) = o[j];
      x += 256 * NJ - 3 * lane;
      x[0] = m;
      x[64] = l;
      continue;
    }
    if (l16 >= wreal) continue;
    const bool any = l != 0.f;
    const int tok = row / G, head = hk * G + row - tok * G;
    float* orow = (float*)B->out + (it.start + tok) * B->P.o_st + head * B->P.o_sh;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      if (16 * j + 4 * g < d) {
        f32x4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = any ? o[j][r] / l : 0.f;
        *(f32x4*)(orow + 16 * j + 4 * g) = x;
      }
    if (B->lse && g == 0)
      B->lse[(size_t)(it.start + tok) * B->P.H + head] =
          any ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  }
}

// ---- launches -----------------------------------------------------------------------------

// Workgroups of a compute unit: LDS (bf16), registers and LDS (fp32) hold so many
int per_unit(const ChunkProb& P) { return P.d > 64 ? 2 : 3; }

Plan plan_of(const ChunkProb& P) {
  Plan L;
  L.rows = P.dtype == CA_BF16 ? kWalkRows : kF32Rows;
  const int64_t rows = (int64_t)P.tokens * P.G;
  const int wave_rows = L.rows / 4;
  L.slot_waves = (int)(rows < L.rows ? (rows + wave_rows - 1) / wave_rows : 4);
  L.blocks = (int)(rows / L.rows + (P.B < P.tokens ? P.B : P.tokens));
  const Classes C = Classes::of(P.Hk, per_unit(P));
  // tiles of a block: the table's, or those of the sinks and of the window of its tokens
  int64_t tiles = ((int64_t)P.max_pages * P.page + KT - 1) / KT;
  const int64_t span = (int64_t)P.m.left + (P.m.causal ? 0 : P.m.right) + L.rows / P.G + 2;
  tiles = std::min(tiles, span / KT + 2 + ((int64_t)P.m.sinks + KT - 1) / KT);
  L.direct = P.B <= kDirectBatch && L.blocks < kDirectBlocks && tiles <= kDirectTiles;
  if (L.direct) {
    L.block_at = L.turn_at = L.cut_at = L.part_at = L.bytes = 0;
    return L;
  }
  auto align = [](size_t x) { return (x + 255) & ~(size_t)255; };
  L.block_at = 256;
  L.turn_at = align(L.block_at + (size_t)L.blocks * sizeof(Block));
  L.cut_at = align(L.turn_at + (size_t)(C.held + 1) * sizeof(Turn));
  L.part_at = align(L.cut_at + (size_t)C.held * sizeof(Cut));
  const int dp = P.d <= 32 ? 32 : P.d <= 64 ? 64 : 128;
  const int chunks = P.dtype == CA_BF16 ? dp / 8 : dp / 16;
  L.bytes = align(L.part_at + (size_t)C.g * 2 * C.held * L.slot_waves * 256 * (4 * chunks + 2));
  return L;
}

// Workgroups that may have work: those that run at a time, or one for each block
int64_t grid_of(const ChunkProb& P, const Plan& L, const Classes& C) {
  const int64_t held = (int64_t)C.g * C.held, r = 8 / C.g;
  const int64_t each = 8 * ((L.blocks * (int64_t)C.heads + r - 1) / r);
  return each > held || L.direct ? each : held;
}

template <typename T, int DP>
hipError_t run_join(const ChunkProb& P, const Plan& L, const Classes& C, T* out, float* lse,
                    char* ws, hipStream_t st) {
  if (L.direct) return hipSuccess;
  const int64_t most = (int64_t)C.held * C.g * L.slot_waves * 4;
  const dim3 grid((unsigned)(most < kJoinGrid ? most : kJoinGrid));
  hipLaunchKernelGGL((chunk_join_kernel<T, DP>), grid, dim3(256), 0, st, P, L, C, ws, out, lse);
  return hipGetLastError();
}

template <int D>
hipError_t run_bf16(const ChunkProb& P, const Plan& L, const bf16* q, const bf16* kp,
                    const bf16* vp, bf16* out, float* lse, char* ws, hipStream_t st) {
  const Classes C = Classes::of(P.Hk, per_unit(P));
  const dim3 grid((unsigned)grid_of(P, L, C));
  const ChunkArgs A{P, L, C, FastDiv::of(P.page), P.scale * kLog2e, q, kp, vp, out, lse, ws};
  // the rows of a page that a group of 16 takes are reached by 32-bit offsets from scalar bases
  auto fits = [](int64_t sp, int64_t st) {
    return sp < ((int64_t)1 << 31) && st <= (1 << 23) && st >= D;
  };
  if (P.page % 16 == 0 && fits(P.k_sp, P.k_st) && fits(P.v_sp, P.v_st))
    hipLaunchKernelGGL((chunk_bf16_kernel<D, true>), grid, dim3(256), 0, st, A);
  else
    hipLaunchKernelGGL((chunk_bf16_kernel<D, false>), grid, dim3(256), 0, st, A);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : run_join<bf16, D>(P, L, C, out, lse, ws, st);
}

template <int DP, int WAVES>
hipError_t run_f32(const ChunkProb& P, const Plan& L, const float* q, const float* kp,
                   const float* vp, float* out, float* lse, char* ws, hipStream_t st) {
  const Classes C = Classes::of(P.Hk, per_unit(P));
  const ChunkArgs A{P, L, C, FastDiv::of(P.page), P.scale * kLog2e, q, kp, vp, out, lse, ws};
  const dim3 grid((unsigned)grid_of(P, L, C));
  // the rows of a page that a group of 8 takes are reached by 32-bit offsets from scalar bases
  auto fits = [](int64_t sp, int64_t st) { return sp < (1 << 30) && st <= (1 << 23); };
  if (P.page % 8 == 0 && fits(P.k_sp, P.k_st) && fits(P.v_sp, P.v_st))
    hipLaunchKernelGGL((chunk_f32_kernel<DP, WAVES, true>), grid, dim3(256), 0, st, A);
  else
    hipLaunchKernelGGL((chunk_f32_kernel<DP, WAVES, false>), grid, dim3(256), 0, st, A);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : run_join<float, DP>(P, L, C, out, lse, ws, st);
}

}  // namespace

bool chunk_fits(const ChunkProb& P) {
  if ((int64_t)P.tokens * P.G >= ((int64_t)1 << 30)) return false;
  // workgroups of 256 threads, fewer than 2^32 of them
  return grid_of(P, plan_of(P), Classes::of(P.Hk, per_unit(P))) < (1 << 24);
}

size_t chunk_bytes(const ChunkProb& P) { return plan_of(P).bytes; }

hipError_t launch_chunk(const ChunkProb& P, const void* q, const void* kp, const void* vp, void* out,
                        float* lse, char* ws, hipStream_t st) {
  const Plan L = plan_of(P);
  if (!L.direct) {
    hipLaunchKernelGGL(chunk_plan_kernel, dim3(1), dim3(kPlan), 0, st, P, L,
                       Classes::of(P.Hk, per_unit(P)), ws);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (P.dtype == CA_BF16) {
    const bf16 *a = (const bf16*)q, *b = (const bf16*)kp, *c = (const bf16*)vp;
    return P.d == 64 ? run_bf16<64>(P, L, a, b, c, (bf16*)out, lse, ws, st)
                     : run_bf16<128>(P, L, a, b, c, (bf16*)out, lse, ws, st);
  }
  const float *a = (const float*)q, *b = (const float*)kp, *c = (const float*)vp;
  return P.d <= 32   ? run_f32<32, 3>(P, L, a, b, c, (float*)out, lse, ws, st)
         : P.d <= 64 ? run_f32<64, 3>(P, L, a, b, c, (float*)out, lse, ws, st)
                     : run_f32<128, 2>(P, L, a, b, c, (float*)out, lse, ws, st);
}

}  // namespace ca
