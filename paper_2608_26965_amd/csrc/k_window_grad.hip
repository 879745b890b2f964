// Gradients of attention with a sliding window and sinks, bf16, on the matrix
// cores.
//
// Two kernels of one form. Each keeps a block of 64 or 128 rows (key_rows) of two
// tensors in registers, streams 64-row tiles of two others through LDS (row_tile.h) and forms
// per tile, with P = e^{s - lse},
//     S = X A^T,  E = Y B^T - D,  dS = P E,
// whose accumulators (a lane holds one kept row and several streamed ones) are the
// next products' operand as they stand:
//   queries kept (A = q, B = dout), keys streamed (X = k, Y = v):
//     dq += dS k            and the mean key  kbar += P k
//   keys kept (A = k, B = v), queries streamed (X = q, Y = dout):
//     dk += dS^T q,  dv += P^T dout
// Logits and E are formed twice that way, but every sum has one owner and a fixed
// order; adding dq up from the second kernel would need atomics or hundreds of
// megabytes of partial sums.
//
// P and dS are rounded to bf16 for their products (2^-8 each), everything else is
// fp32. A row's dS sum to zero, so that what the keys have in common drops out of
// dq; rounded ones, and a D = rowsum(dout * out) from an output that was rounded to
// bf16, leave a sum r of their own, and r times the mean key of an error. So the
// first kernel sums the dS as rounded and takes it out, dq = scale (sum dS k -
// r kbar), and D + r goes to the second. Without it dq is off by 0.0037 of its
// size (keys of one mixture, 8,192 tokens), with it 0.0023, where rounding the
// result alone is 0.0017. dk has no such sum; its dS go in as two bf16 parts (a fifth
// product), with one it was off by 0.0024 to 0.0027, so by 0.0017 to 0.0020, for 3 to
// 6% of the time.
#include <math.h>

#include "row_tile.h"
#include "seq.h"

namespace ca {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kVmcnt0 = 0x0F70;  // s_waitcnt immediate: vmcnt = 0 only
constexpr int kPad = 128;        // lse2 and delta are padded to this
constexpr int KT = 64;           // streamed rows of a tile

constexpr int NW = 4;            // wavefronts of a workgroup, W kept rows each

// Kept rows of a wavefront: 16, or 32 where keys are kept at d = 64 and the window is long.
// 16 rows leave four waves a SIMD at d = 64 with queries kept (128 registers) and three with
// keys kept (143; two with 32 rows), two at d = 128 (32 there, one wave with
// half the registers accumulation registers that operands are copied through: 793 us
// for the padded batch of three where 16 took 726), and four wavefronts of them make
// blocks of 64, of which several share a compute unit, not at the same point of a tile at the
// same time (d = 128, workgroups of 128 rows: 468 us where 64 take 430, 342 and 322, 713 to
// 720 and 703 to 710). dq takes 52 us with 32 rows and 49 with 16 (8,192 tokens, d = 64),
// 116 and 102, 68 and 57, 25 and 20. dk and dv: blocks of 128 keys waste more of a short
// window's tiles (2 x 8 heads of 6,013 tokens, 48 keys: 25 us and 21; 8,733 tokens, 295
// keys: 76 and 64), blocks of 64 read every streamed row twice as often (1,024 keys: 70
// and 74; 2,437: 68 and 93; no limit, 3,984 tokens: 121 and 145).
int key_rows(const WinProb& P) {
  return P.d == 64 && (int64_t)P.m.left + (P.m.causal ? 0 : P.m.right) >= 512 ? 32 : 16;
}
constexpr int kQueryRows = 16;
// A product of W kept rows: W x W x K, accumulator r of a lane being row 8 (r / 4) + 4 g
// + r % 4 (g = lane / W) of kept row lane % W
template <int W>
struct Mma;
template <>
struct Mma<32> {
  typedef f32x16 Acc;
  static constexpr int K = 16, N = 16;
  static __device__ __forceinline__ Acc mma(bf16x8 a, bf16x8 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mma<16> {
  typedef f32x4 Acc;
  static constexpr int K = 32, N = 4;
  static __device__ __forceinline__ Acc mma(bf16x8 a, bf16x8 b, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};

// Row blocks and the parts that their streamed tiles are cut into. Blocks 0 ..
// nsink - 1 are cut into `psink` parts (keys kept: the blocks that hold sinks,
// which every query sees), the others into `p`.
struct Parts {
  int nb, nsink, psink, p;
  __host__ __device__ int items() const { return nsink * psink + (nb - nsink) * p; }
  // places of partial sums: blocks of one part need none
  __host__ __device__ int places() const {
    return (psink > 1 ? nsink * psink : 0) + (p > 1 ? (nb - nsink) * p : 0);
  }
  // block, part and number of parts of item v; the place of its partial sums
  __device__ __forceinline__ void at(int v, int* a, int* part, int* parts, int* place) const {
    const int s = nsink * psink;
    if (v < s) {
      *a = v / psink;
      *part = v - *a * psink;
      *parts = psink;
      *place = v;
    } else {
      const int x = (v - s) / p;
      *a = nsink + x;
      *part = v - s - x * p;
      *parts = p;
      *place = (psink > 1 ? s : 0) + v - s;
    }
  }
};

// All XCDs work on one head at a time, each on a contiguous eighth of its items
// where the window is short (they read the same streamed rows), else on every
// eighth (the work of causal blocks grows or falls along the sequence).
__device__ __forceinline__ bool item_of(int wg, int n, int G, int contiguous, int* bh, int* v) {
  const int chunk = (n + 7) >> 3, loc = wg >> 3;
  *bh = loc / chunk;
  const int s = loc - *bh * chunk, x = ((wg & 7) + *bh / G) & 7;
  if (contiguous) {
    const int first = (int)((int64_t)x * n >> 3), end = (int)((int64_t)(x + 1) * n >> 3);
    *v = first + s;
    return *v < end;
  }
  *v = 8 * s + x;
  return *v < n;
}

struct GradArgs {
  const bf16 *x, *y, *a, *b;  // streamed and kept tensors
  Lay lx, ly, la, lb;
  const bf16* out;            // queries kept: the attention's output, for D
  const float* lse;
  float *lse2, *delta;        // [B H][nq padded to kPad]: lse log2(e), -D (inf and 0 past the lengths)
  bf16 *g0, *g1;
  Lay lg0, lg1;
  float* part;                // [heads][places][kRows][2][d]
  float* rpart;               // queries kept: [heads][places][kRows], sums of dS as rounded
  Parts parts;
  int contiguous;
  float sl2;
};

template <int D, bool KEYS, int W>
__global__ __launch_bounds__(64 * NW, 2) void window_grad_kernel(const WinProb P, const GradArgs g) {
  constexpr int kRows = NW * W;
  typedef Mma<W> M;
  constexpr int KK = D / M::K, DT = D / W, RB = 2 * D, TILE = KT * RB;
  __shared__ __attribute__((aligned(1024))) char smem[4 * TILE];  // X, X, Y, Y
  __shared__ __attribute__((aligned(16))) float rows[KEYS ? 2 : 1][2][KEYS ? KT : 4];
  const int nitem = g.parts.items();
  int hx, v;  // the kept tensors' head
  if (!item_of(blockIdx.x, nitem, KEYS ? 1 : P.G, g.contiguous, &hx, &v)) return;
  int blk, part, parts, place;
  g.parts.at(v, &blk, &part, &parts, &place);
  const int tid = threadIdx.x, lane = tid & 63, lw = lane % W, gr = lane / W;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int HX = KEYS ? P.Hk : P.H;
  const int b = hx / HX, lq = P.qlen(b), lk = P.klen(b), off = lk - lq;
  const int n = KEYS ? lk : lq, nmax = KEYS ? P.nk : P.nq, r0 = blk * kRows;
  const int real = max(0, min(kRows, n - r0));
  const int nqp = (P.nq + kPad - 1) / kPad * kPad;

  // the tiles that one of the block's rows sees
  TileList list{0, 0, 0};
  int first = 0, per_head = 1, ntile = 0;
  if (real > 0) {
    if constexpr (KEYS) {
      const int i0 = max(0, seeing_positions(P.m, r0).lo - off);
      const int hi = r0 < P.m.sinks ? kUnlimited : seeing_positions(P.m, r0 + real - 1).hi;
      const int i1 = min(lq, hi - off + 1);
      if (i1 > i0) {
        first = i0 / KT;
        per_head = (i1 + KT - 1) / KT - first;
        ntile = per_head * P.G;
      }
    } else {
      list = visible_tiles<KT>(P.m, r0 + off, r0 + real - 1 + off, lk);
      ntile = list.n;
    }
  }
  const int per = (ntile + parts - 1) / parts;
  const int t0 = min(ntile, part * per), t1 = min(ntile, t0 + per);

  // this wavefront's rows, and this lane's
  const int w0 = r0 + W * w, wreal = max(0, min(W, n - w0));
  const int row = min(w0 + min(lw, max(wreal, 1) - 1), nmax - 1);
  KeyRange ra, rz;       // queries kept: of the first and last row
  int plo0, plo1, phi0, phi1;  // keys kept: least and greatest bounds of their positions
  if constexpr (KEYS) {
    const int last = w0 + max(wreal, 1) - 1;
    plo0 = seeing_positions(P.m, w0).lo;
    plo1 = seeing_positions(P.m, last).lo;
    phi0 = last < P.m.sinks ? kUnlimited : max(w0, P.m.sinks) + P.m.left;
    phi1 = w0 < P.m.sinks ? kUnlimited : last + P.m.left;
  } else {
    ra = visible_keys(P.m, w0 + off, lk);
    rz = visible_keys(P.m, w0 + max(wreal, 1) - 1 + off, lk);
  }
  // 0: no pair of the wavefront's rows and the tile's is visible, 2: all, 1: else
  auto tile_class = [&](int s0) __attribute__((always_inline)) {
    if (wreal == 0) return 0;
    if constexpr (KEYS) {
      const int p0 = s0 + off, p1 = min(s0 + KT, lq) - 1 + off;
      if (p1 < plo0 || p0 > phi1) return 0;
      return plo1 <= p0 && phi0 >= p1 ? 2 : 1;
    } else {
      if (s0 >= rz.s_end && (s0 >= rz.hi || s0 + KT <= ra.lo)) return 0;
      return s0 + KT <= ra.s_end || (s0 >= rz.lo && s0 + KT <= ra.hi) ? 2 : 1;
    }
  };

  bf16x8 af[KK], bf[KK];
  float mylse = INFINITY, negdel = 0.f;
  {
    const bf16* ar = g.a + row_off(hx, row, g.la);
    const bf16* br = g.b + row_off(hx, row, g.lb);
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      af[kk] = *(const bf16x8*)(ar + M::K * kk + 8 * gr);
      bf[kk] = *(const bf16x8*)(br + M::K * kk + 8 * gr);
    }
    if constexpr (!KEYS) {
      const bf16* orow = g.out + row_off(hx, row, P.lo);
      float d = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const bf16x8 o = *(const bf16x8*)(orow + M::K * kk + 8 * gr);
#pragma unroll
        for (int j = 0; j < 8; ++j) d = fmaf(bf2f(o[j]), bf2f(bf[kk][j]), d);
      }
      if (W == 16) d += __shfl_xor(d, 16, 64);
      d += __shfl_xor(d, 32, 64);
      const float ls = g.lse[(size_t)hx * P.nq + row];
      if (lw < wreal && ls != -INFINITY) {
        mylse = ls * kLog2e;
        negdel = -d;
      }
    }
  }
  // Retire the loads here, so that no vmcnt wait of theirs lands in the loop
  __builtin_amdgcn_s_waitcnt(kVmcnt0);

  const RowCopy<RB, KT, NW> xcopy(w, lane, (uint32_t)(g.lx.sn * 2));
  const RowCopy<RB, KT, NW> ycopy(w, lane, (uint32_t)(g.ly.sn * 2));
  const uint32_t lds0 = lds_addr(smem);
  // The walk over the streamed tiles: keys kept, query head gh of the group and its
  // tile, the heads one after another
  struct Walk {
    int t, gh, tile;
  };
  auto start = [&](int t) {
    Walk x{t, 0, t};
    if constexpr (KEYS) {
      x.gh = t / per_head;
      x.tile = t - x.gh * per_head;
    }
    return x;
  };
  auto advance = [&](Walk& x) __attribute__((always_inline)) {
    ++x.t;
    ++x.tile;
    if (KEYS && x.tile == per_head) {
      x.tile = 0;
      ++x.gh;
    }
  };
  auto first_row = [&](const Walk& x) __attribute__((always_inline)) {
    return KT * (KEYS ? first + x.tile : list.tile(x.t));
  };
  const int xhead = KEYS ? b * P.H + (hx - b * P.Hk) * P.G : b * P.Hk + (hx - b * P.H) / P.G;
  const bf16 *xbase = g.x + row_off(xhead, 0, g.lx), *ybase = g.y + row_off(xhead, 0, g.ly);
  auto issue = [&](const Walk& x, int buf) __attribute__((always_inline)) {
    const int s0 = first_row(x), last = (KEYS ? lq : lk) - 1 - s0;
    xcopy.issue(xbase + x.gh * g.lx.sh + s0 * g.lx.sn, lds0 + buf * TILE, w, lane, last);
    ycopy.issue(ybase + x.gh * g.ly.sh + s0 * g.ly.sn, lds0 + (2 + buf) * TILE, w, lane, last);
    if constexpr (KEYS) {  // the rows' lse and D, 256 bytes each
      const size_t at = (size_t)(xhead + x.gh) * nqp + s0;
      const uint32_t dst = __builtin_amdgcn_readfirstlane(lds_addr(&rows[buf][w & 1][0]));
      if (w < 2 && lane < 16) lds_dma16(w ? g.delta + at : g.lse2 + at, 16 * lane, dst);
    }
  };
  // Operand offsets. Rows: this lane's chunk of row l % W of a row tile. Columns: its
  // pieces in the two transposing reads that make an operand of M::K streamed rows
  // whose other operand is 8 accumulators: W = 32, accumulators 8 u .. 8 u + 7 of a row
  // tile (col_operand); W = 16, two row tiles, element j being row 16 (j / 4) + 4 g + j % 4.
  int xoff[KK], coff[DT][2];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk)
    xoff[kk] = lw * RB + (((M::K / 8 * kk + gr) ^ row_key<RB>(lw)) << 4);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    if constexpr (W == 32) {
#pragma unroll
      for (int t = 0; t < 2; ++t) coff[dt][t] = col_operand<RB>(lane, dt, t);
    } else {
      const int r = 4 * gr + (lw >> 2), lc = 2 * dt + ((lw & 3) >> 1);
      coff[dt][0] = r * RB + ((lc ^ row_key<RB>(r)) << 4) + 8 * (lw & 1);
      coff[dt][1] = coff[dt][0] + 16 * RB;
    }
  }

  typedef typename M::Acc Acc;
  Acc acc0[DT], acc1[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int r = 0; r < M::N; ++r) acc0[dt][r] = acc1[dt][r] = 0.f;
  float rsum = 0.f;

  auto compute = [&](auto buf_tag, int s0) __attribute__((always_inline)) {
    constexpr int BUF = decltype(buf_tag)::value;
    const int c = tile_class(s0);
    if (c == 0) return;
    const char* xs = smem + BUF * TILE;
    const char* ys = smem + (2 + BUF) * TILE;
    constexpr int RT = KT / W, NO = KT / M::K;  // row tiles, and operands of 8 accumulators
    Acc s[RT], e[RT];
    bf16x8 pp[NO], dd[NO], dl[KEYS ? NO : 1];  // P, dS, what dS lost in rounding

    // Steps, a fence apart each: the operands of the next step are read before the
    // products of this one, which run beside some of the exponentials. (Left to
    // itself the compiler reads each operand right before its product and waits.)
    bf16x8 xr[2][2], yr[2][2];  // [step % 2][kk % 2]: rows
    bf16x8 xc[2][2], yc[2][2];  // [step % 2][dt % 2]: columns
    constexpr int SR = KK / 2, SC = DT / 2;  // steps of a row tile's logits, an operand's products
    auto load_rows = [&](int n) __attribute__((always_inline)) {  // step n: row tile n / SR
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int at = W * (n / SR) * RB + xoff[2 * (n % SR) + i];
        xr[n & 1][i] = *(const bf16x8*)(xs + at);
        yr[n & 1][i] = *(const bf16x8*)(ys + at);
      }
    };
    auto load_cols = [&](int n) __attribute__((always_inline)) {  // step n: operand n / SC
      const char *xo = xs + M::K * (n / SC) * RB, *yo = ys + M::K * (n / SC) * RB;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int dt = 2 * (n % SC) + i;
        xc[n & 1][i] = read_cols(xo + coff[dt][0], xo + coff[dt][1]);
        if constexpr (KEYS) yc[n & 1][i] = read_cols(yo + coff[dt][0], yo + coff[dt][1]);
      }
    };
    // keys kept: E starts from the rows' -D
    auto begin = [&](int T) __attribute__((always_inline)) {
      if constexpr (KEYS) {
#pragma unroll
        for (int x = 0; x < M::N / 4; ++x) {
          const f32x4 d = *(const f32x4*)&rows[BUF][1][W * T + 8 * x + 4 * gr];
#pragma unroll
          for (int r = 0; r < 4; ++r) e[T][4 * x + r] = d[r];
        }
      }
    };
    auto logits = [&](int n) __attribute__((always_inline)) {
      const int T = n / SR;
      Acc zero;
#pragma unroll
      for (int r = 0; r < M::N; ++r) zero[r] = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int kk = 2 * (n % SR) + i;
        s[T] = M::mma(xr[n & 1][i], af[kk], kk == 0 ? zero : s[T]);
        e[T] = M::mma(yr[n & 1][i], bf[kk], kk == 0 && !KEYS ? zero : e[T]);
      }
    };
    auto probs = [&](int o) __attribute__((always_inline)) {
      float p[8], ds[8];
#pragma unroll
      for (int x = 0; x < 2; ++x) {  // four accumulators from r on of row tile T
        const int T = W == 32 ? o / 2 : 2 * o + x, r0 = W == 32 ? 8 * (o % 2) + 4 * x : 0;
        f32x4 ls = {mylse, mylse, mylse, mylse};
        if constexpr (KEYS) ls = *(const f32x4*)&rows[BUF][0][W * T + 2 * r0 + 4 * gr];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          p[4 * x + r] = __builtin_amdgcn_exp2f(fmaf(s[T][r0 + r], g.sl2, -ls[r]));
          ds[4 * x + r] = p[4 * x + r] * (KEYS ? e[T][r0 + r] : e[T][r0 + r] + negdel);
        }
      }
      pp[o] = pack8(p);
      dd[o] = pack8(ds);
      if constexpr (KEYS) {
        float lo[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) lo[j] = ds[j] - bf2f(dd[o][j]);
        dl[o] = pack8(lo);
      } else {
        rsum = sum8(dd[o], rsum);
      }
    };
    auto products = [&](int n) __attribute__((always_inline)) {
      const int o = n / SC;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int dt = 2 * (n % SC) + i;
        acc0[dt] = M::mma(xc[n & 1][i], dd[o], acc0[dt]);
        if constexpr (KEYS) acc0[dt] = M::mma(xc[n & 1][i], dl[o], acc0[dt]);
        acc1[dt] = M::mma(KEYS ? yc[n & 1][i] : xc[n & 1][i], pp[o], acc1[dt]);
      }
    };
    // row tiles T0 .. T0 + RT / 2 - 1
    auto mask = [&](int T0) __attribute__((always_inline)) {
      int rw = row;  // (the ranges are formed here: kept over the loop they cost registers)
      asm volatile("" : "+v"(rw));
      if constexpr (KEYS) {
        const PosRange see = seeing_positions(P.m, rw);
        const uint32_t len = (uint32_t)max(0, see.hi - see.lo + 1);
        const int p0 = s0 + off + 4 * gr - see.lo;
#pragma unroll
        for (int T = T0; T < T0 + RT / 2; ++T)
#pragma unroll
          for (int r = 0; r < M::N; ++r)
            if ((uint32_t)(p0 + W * T + 8 * (r >> 2) + (r & 3)) >= len) {
              s[T][r] = -INFINITY;
              e[T][r] = 0.f;
            }
      } else {
        const KeyRange rr = visible_keys(P.m, rw + off, lk);
        const uint32_t len = (uint32_t)max(0, rr.hi - rr.lo);
        const int a0 = s0 + 4 * gr - rr.lo, b0 = rr.s_end - s0 - 4 * gr;
#pragma unroll
        for (int T = T0; T < T0 + RT / 2; ++T)
#pragma unroll
          for (int r = 0; r < M::N; ++r) {
            const int x = W * T + 8 * (r >> 2) + (r & 3);
            if (!((uint32_t)(a0 + x) < len || x < b0)) {
              s[T][r] = -INFINITY;
              e[T][r] = 0.f;
            }
          }
      }
    };
    auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
    load_rows(0);
#pragma unroll
    for (int T = 0; T < RT / 2; ++T) begin(T);
    fence();
#pragma unroll
    for (int n = 0; n < RT * SR / 2; ++n) {
      load_rows(n + 1);
      fence();
      logits(n);
      fence();
    }
    if (c == 1) mask(0);
#pragma unroll
    for (int T = RT / 2; T < RT; ++T) begin(T);
#pragma unroll
    for (int n = RT * SR / 2; n < RT * SR; ++n) {
      if (n + 1 < RT * SR)
        load_rows(n + 1);
      else
        load_cols(0);
      fence();
      logits(n);
      if (n - RT * SR / 2 < NO / 2) probs(n - RT * SR / 2);
      fence();
    }
    if (c == 1) mask(RT / 2);
#pragma unroll
    for (int n = 0; n < NO * SC; ++n) {
      if (n + 1 < NO * SC) load_cols(n + 1);
      fence();
      products(n);
      if (n < NO / 2) probs(NO / 2 + n);
      fence();
    }
  };
  // One barrier a tile: behind it tile t's copies have landed and every
  // wavefront is past tile t - 1, whose buffers take tile t + 1.
  Walk next = start(t0);
  auto step = [&](auto buf_tag, int t, int s0) __attribute__((always_inline)) {
    constexpr int BUF = decltype(buf_tag)::value;
    wait_vmcnt<0>();
    wait_lgkm();
    raw_barrier();
    int s1 = 0;
    if (t + 1 < t1) {
      advance(next);
      s1 = first_row(next);
      issue(next, BUF ^ 1);
    }
    compute(buf_tag, s0);
    return s1;
  };
  if (t0 < t1) {
    issue(next, 0);
    int s0 = first_row(next);
    for (int t = t0; t < t1; t += 2) {
      s0 = step(std::integral_constant<int, 0>{}, t, s0);
      if (t + 1 < t1) s0 = step(std::integral_constant<int, 1>{}, t + 1, s0);
    }
  }

  const int rout = w0 + lw;
  if (!KEYS) {
    if (W == 16) rsum += __shfl_xor(rsum, 16, 64);
    rsum += __shfl_xor(rsum, 32, 64);
  }
  auto dims = [&](int dt, int x) { return W * dt + 8 * x + 4 * gr; };
  if (parts > 1) {
    const size_t slot = ((size_t)hx * g.parts.places() + place) * kRows + W * w + lw;
    float* p = g.part + slot * 2 * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int x = 0; x < M::N / 4; ++x) {
        f32x4 a, b4;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          a[r] = acc0[dt][4 * x + r];
          b4[r] = acc1[dt][4 * x + r];
        }
        *(f32x4*)(p + dims(dt, x)) = a;
        *(f32x4*)(p + D + dims(dt, x)) = b4;
      }
    if (!KEYS && gr == 0) {
      g.rpart[slot] = rsum;
      if (part == 0) {
        g.lse2[(size_t)hx * nqp + rout] = mylse;
        g.delta[(size_t)hx * nqp + rout] = negdel;
      }
    }
    return;
  }
  if (!KEYS && gr == 0) {
    g.lse2[(size_t)hx * nqp + rout] = mylse;
    g.delta[(size_t)hx * nqp + rout] = negdel - rsum;
  }
  if (rout >= nmax) return;
  const bool on = lw < wreal;
  bf16* o0 = g.g0 + row_off(hx, rout, g.lg0);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int x = 0; x < M::N / 4; ++x) {
      bf16x4 y;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float a = acc0[dt][4 * x + r], d = KEYS ? a : a - rsum * acc1[dt][4 * x + r];
        y[r] = f2bf(on ? d * P.scale : 0.f);
      }
      *(bf16x4*)(o0 + dims(dt, x)) = y;
    }
  if constexpr (KEYS) {
    bf16* o1 = g.g1 + row_off(hx, rout, g.lg1);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int x = 0; x < M::N / 4; ++x) {
        bf16x4 y;
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = f2bf(on ? acc1[dt][4 * x + r] : 0.f);
        *(bf16x4*)(o1 + dims(dt, x)) = y;
      }
  }
}

// Adds up the parts of the blocks that were cut, in order: 32 lanes a row.
template <int D, bool KEYS, int W>
__global__ __launch_bounds__(256) void window_grad_join_kernel(const WinProb P, const GradArgs g,
                                                               int ncut, int first_cut) {
  constexpr int E = D / 32, kRows = NW * W;  // elements of a lane, rows of a block
  const int HX = KEYS ? P.Hk : P.H, nmax = KEYS ? P.nk : P.nq;
  const int64_t id = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  const int64_t rows = (int64_t)ncut * kRows;
  const int hx = (int)(id / rows), x = (int)(id - hx * rows);
  if (hx >= P.B * HX) return;
  const int blk = first_cut + x / kRows, r = blk * kRows + x % kRows, b = hx / HX;
  const bool sink = blk < g.parts.nsink;
  const int parts = sink ? g.parts.psink : g.parts.p;
  const int place = sink ? blk * parts
                         : (g.parts.psink > 1 ? g.parts.nsink * g.parts.psink : 0) +
                               (blk - g.parts.nsink) * parts;
  const size_t slot = ((size_t)hx * g.parts.places() + place) * kRows + x % kRows;
  float a0[E], a1[E], rs = 0.f;
#pragma unroll
  for (int i = 0; i < E; ++i) a0[i] = a1[i] = 0.f;
  for (int p = 0; p < parts; ++p) {
    const float* q = g.part + (slot + (size_t)p * kRows) * 2 * D + lane;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      a0[i] += q[32 * i];
      a1[i] += q[D + 32 * i];
    }
    if (!KEYS) rs += g.rpart[slot + (size_t)p * kRows];
  }
  const bool on = r < (KEYS ? P.klen(b) : P.qlen(b));
  if (!KEYS && lane == 0) {
    const int nqp = (P.nq + kPad - 1) / kPad * kPad;
    if (on) g.delta[(size_t)hx * nqp + r] -= rs;
  }
  if (r >= nmax) return;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const float d = KEYS ? a0[i] : a0[i] - rs * a1[i];
    g.g0[row_off(hx, r, g.lg0) + lane + 32 * i] = f2bf(on ? d * P.scale : 0.f);
    if (KEYS) g.g1[row_off(hx, r, g.lg1) + lane + 32 * i] = f2bf(on ? a1[i] : 0.f);
  }
}

// The cut of a launch of `heads` heads with nb row blocks, nsink of them with `all` tiles
// to walk and the others with `seen` (up to that many where `uneven`: causal attention
// without a window). Of the cuts below the one with the least time by this estimate, in
// tiles: a workgroup costs three tiles beside its own; equal workgroups run in rounds of
// as many as the chip holds, others fill it and leave half the longest over; partial sums
// (2 d floats a row, written and read) cost 0.015 for 128 rows and a launch 3. Twice
// that for the sums took 502 us instead of 387 for 3 heads of 7,553 tokens (d = 128, 357
// blocks on 512 places), but 252 instead of 270 for 10 heads on 2 of 3,186 (causal). 8,192 tokens on 2
// key heads take one round of 24 tiles (three parts, 159 us with the forward pass) instead
// of two of 18 (166).
Parts cut(int nb, int nsink, int64_t all, int64_t seen, int64_t heads, int rows, bool uneven) {
  static const int kCuts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
  // two workgroups a compute unit; at d = 64 three fit, but 768 here took 196 us instead of
  // 185, 321 instead of 316 and 288 instead of 302 on three shapes, others the same
  const int64_t slots = 512;
  if (nsink > nb) nsink = nb;
  Parts best{nb, nsink, 1, 1};
  double least = -1;
  for (int p : kCuts) {
    if (p > 1 && seen / p < 4) break;
    for (int ps : kCuts) {
      if (ps > 1 && (nsink == 0 || all / ps < 4)) break;
      const Parts x{nb, nsink, ps, p};
      const int64_t wgs = heads * x.items(), other = nb - nsink;
      if (p * ps > 1 && wgs > 1 << 16) break;  // enough workgroups, and bytes of partial sums
      const double each = (double)((seen + p - 1) / p) + 3;
      const double sink = nsink ? (double)((all + ps - 1) / ps) + 3 : 0;
      const double longest = each > sink ? each : sink;
      double work = (double)heads * (nsink * ps * sink + other * p * each);
      if (uneven) work *= 0.5;
      double cost;
      if (wgs <= slots)
        cost = longest;
      else if (!uneven && sink <= 1.25 * each)
        cost = (double)((wgs + slots - 1) / slots) * longest;
      else
        cost = work / slots + 0.5 * longest;
      if (x.places()) cost += 0.015 / 128 * (double)(heads * x.places() * rows) + 3;
      if (least < 0 || cost < least) {
        least = cost;
        best = x;
      }
    }
  }
  return best;
}
Parts query_parts(const WinProb& P) {
  const int kRows = NW * kQueryRows, nb = (P.nq + kRows - 1) / kRows;
  int64_t keys = (int64_t)P.m.left + (P.m.causal ? 0 : P.m.right) + kRows + P.m.sinks;
  if (keys > P.nk) keys = P.nk;
  const int64_t tiles = (keys + KT - 1) / KT;
  return cut(nb, 0, tiles, tiles, (int64_t)P.B * P.H, kRows, P.m.causal && P.m.left >= P.nk);
}
// keys kept: the blocks that hold sinks are seen by all queries
Parts key_parts(const WinProb& P) {
  const int kRows = NW * key_rows(P), nb = (P.nk + kRows - 1) / kRows;
  const int64_t all = (int64_t)(P.nq + KT - 1) / KT * P.G;
  int64_t seen = (((int64_t)P.m.left + (P.m.causal ? 0 : P.m.right) + kRows) / KT + 1) * P.G;
  if (seen > all) seen = all;
  const int nsink = P.m.sinks < P.nk ? (P.m.sinks + kRows - 1) / kRows : nb;
  return cut(nb, seen < all ? nsink : 0, all, seen, (int64_t)P.B * P.Hk, kRows,
             P.m.causal && P.m.left >= P.nk);
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

struct GradPlan {
  size_t lse2, delta, part, rpart, total;
};
GradPlan plan(const WinProb& P) {
  const size_t nqp = (size_t)(P.nq + kPad - 1) / kPad * kPad, rows = (size_t)P.B * P.H * nqp;
  // the two kernels' partial sums follow one another in the same place
  const size_t pq = (size_t)P.B * P.H * query_parts(P).places() * NW * kQueryRows;
  const size_t pk = (size_t)P.B * P.Hk * key_parts(P).places() * NW * key_rows(P);
  GradPlan g;
  g.lse2 = 0;
  g.delta = align256(rows * 4);
  g.rpart = g.delta + align256(rows * 4);
  g.part = g.rpart + align256(pq * 4);
  g.total = g.part + align256((pq > pk ? pq : pk) * 2 * P.d * 4);
  return g;
}

template <int D, bool KEYS, int W>
hipError_t run_grad(const WinProb& P, const GradArgs& g, hipStream_t st) {
  const int heads = P.B * (KEYS ? P.Hk : P.H), n = g.parts.items();
  hipLaunchKernelGGL((window_grad_kernel<D, KEYS, W>), dim3((unsigned)((int64_t)8 * ((n + 7) / 8) * heads)),
                     dim3(64 * NW), 0, st, P, g);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || g.parts.places() == 0) return e;
  const int first = g.parts.psink > 1 ? 0 : g.parts.nsink;
  const int ncut = (g.parts.p > 1 ? g.parts.nb : g.parts.nsink) - first;
  hipLaunchKernelGGL((window_grad_join_kernel<D, KEYS, W>),
                     dim3((unsigned)(((int64_t)heads * ncut * NW * W + 7) / 8)), dim3(256), 0, st, P, g,
                     ncut, first);
  return hipGetLastError();
}

template <int D>
hipError_t run_both(const WinProb& P, GradArgs& g, const bf16* q, const bf16* k, const bf16* v,
                    const bf16* dout, bf16* dq, bf16* dk, bf16* dv, hipStream_t st) {
  g.contiguous = (int64_t)P.m.left + (P.m.causal ? 0 : P.m.right) < P.nk / 2;
  g.x = k, g.lx = P.lk, g.y = v, g.ly = P.lv;
  g.a = q, g.la = P.lq, g.b = dout, g.lb = P.ldo;
  g.g0 = dq, g.lg0 = P.ldq, g.g1 = nullptr, g.lg1 = P.ldq;
  g.parts = query_parts(P);
  const hipError_t e = run_grad<D, false, kQueryRows>(P, g, st);
  if (e != hipSuccess) return e;
  g.x = q, g.lx = P.lq, g.y = dout, g.ly = P.ldo;
  g.a = k, g.la = P.lk, g.b = v, g.lb = P.lv;
  g.g0 = dk, g.lg0 = P.ldk, g.g1 = dv, g.lg1 = P.ldv;
  g.parts = key_parts(P);
  if constexpr (D == 64)
    if (key_rows(P) == 32) return run_grad<D, true, 32>(P, g, st);
  return run_grad<D, true, 16>(P, g, st);
}

}  // namespace

size_t window_grad_bf16_bytes(const WinProb& P) { return plan(P).total; }

hipError_t launch_window_grad_bf16(const WinProb& P, const void* q, const void* k, const void* v,
                                   const void* out, const float* lse, const void* dout, void* dq,
                                   void* dk, void* dv, char* ws, hipStream_t st) {
  const GradPlan p = plan(P);
  GradArgs g{};
  g.out = (const bf16*)out;
  g.lse = lse;
  g.lse2 = (float*)(ws + p.lse2);
  g.delta = (float*)(ws + p.delta);
  g.part = (float*)(ws + p.part);
  g.rpart = (float*)(ws + p.rpart);
  g.sl2 = P.scale * kLog2e;
  if (P.d == 64)
    return run_both<64>(P, g, (const bf16*)q, (const bf16*)k, (const bf16*)v, (const bf16*)dout,
                        (bf16*)dq, (bf16*)dk, (bf16*)dv, st);
  return run_both<128>(P, g, (const bf16*)q, (const bf16*)k, (const bf16*)v, (const bf16*)dout,
                       (bf16*)dq, (bf16*)dk, (bf16*)dv, st);
}

}  // namespace ca
