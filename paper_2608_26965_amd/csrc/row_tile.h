// Tiles of row-major bf16 rows in LDS, as both operands of the 32x32x16 and
// 16x16x32 matrix products: rows read 16 bytes a lane (A operand, rows on the
// matrix rows) and columns by the transposing LDS read (A operand, the rows'
// dims on the matrix rows and the rows on the contraction).
//
// 16-byte chunk lc of row r sits at chunk lc ^ row_key(r). With row bits b3 b2
// b1 b0 the key makes both reads free of bank conflicts: sixteen consecutive
// rows at one lc fall on sixteen different chunks of 256 bytes, and the four
// rows x 64 bytes that a half wavefront's transposing read takes fall on
// different 32-byte pairs of chunks. Where a product has sixteen rows, the lanes that
// are served together hold rows 0-3 and 12-15 at one chunk and rows 4-11 at its
// neighbour, lc ^ 1: the bit b2 ^ b3 keeps these two sets on chunks of their own (with
// b2 in its place every such read took twice the time).
#pragma once

#include "attn_tile.h"

namespace ca {

template <int RB>
__device__ __forceinline__ int row_key(int r) {
  static_assert(RB == 128 || RB == 256, "row width");
  const int b0 = r & 1, b1 = (r >> 1) & 1, b2 = (r >> 2) & 1, b3 = (r >> 3) & 1;
  const int m = b2 ^ b3;
  return RB == 256 ? (b1 << 3) | (b0 << 2) | (m << 1) | b3 : (b1 << 2) | (m << 1) | b3;
}

// Copies ROWS rows of RB bytes, `stride` bytes apart, into an LDS tile, NW
// wavefronts together (direct global-to-LDS copies, 1024 bytes each).
// An instruction of all wavefronts holds a multiple of sixteen rows, so every one of
// a lane's rows has the same key and its offsets differ by whole rows only.
template <int RB, int ROWS, int NW>
struct RowCopy {
  static constexpr int NI = ROWS * RB / 1024 / NW;
  static constexpr int RPI = 1024 / RB;  // rows of an instruction
  static_assert(NI * 1024 * NW == ROWS * RB && NW * RPI % 16 == 0, "tile split");
  uint32_t off;     // of this lane's first row and chunk
  uint32_t stride;  // bytes between rows

  static __device__ __forceinline__ int row0(int w, int lane) { return w * RPI + lane / (RB / 16); }
  static __device__ __forceinline__ uint32_t chunk(int w, int lane) {
    return (uint32_t)(((lane % (RB / 16)) ^ row_key<RB>(row0(w, lane))) << 4);
  }
  __device__ __forceinline__ RowCopy(int w, int lane, uint32_t stride_bytes) {
    stride = stride_bytes;
    off = (uint32_t)row0(w, lane) * stride + chunk(w, lane);
  }
  __device__ __forceinline__ static uint32_t dst(uint32_t lds, int i, int w) {
    return __builtin_amdgcn_readfirstlane(lds + (uint32_t)((i * NW + w) * 1024));
  }
  __device__ __forceinline__ void issue(const void* base, uint32_t lds, int w) const {
#pragma unroll
    for (int i = 0; i < NI; ++i)
      lds_dma16((const char*)base + (int64_t)i * NW * RPI * stride, off, dst(lds, i, w));
  }
  // rows past `last` are copies of it
  __device__ __forceinline__ void issue(const void* base, uint32_t lds, int w, int lane,
                                        int last) const {
    if (last >= ROWS - 1) {
      issue(base, lds, w);
      return;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i)
      lds_dma16(base, (uint32_t)min(row0(w, lane) + i * NW * RPI, last) * stride + chunk(w, lane),
                dst(lds, i, w));
  }
};

// Byte offset of this lane's chunk (2 kk + h) of row l % 32: the A operand of
// a 32x32x16 product over dims 16 kk .. + 15; row tiles add 32 * RB
template <int RB>
__device__ __forceinline__ int row_operand(int lane, int kk) {
  const int l32 = lane & 31;
  return l32 * RB + (((2 * kk + (lane >> 5)) ^ row_key<RB>(l32)) << 4);
}

// Byte offset of this lane's piece in the transposing read of dims 32 dt .. + 31
// and the rows 8 t + 4 h + 0 .. 3 (h = l / 32); sixteen rows further adds 16 * RB.
// Two reads (t = 0, 1) give the A operand of a 32x32x16 product whose B operand
// holds the accumulators 8 s .. 8 s + 7 of a 32x32 product: element j of half h
// is row 16 s + 8 (j / 4) + 4 h + j % 4.
template <int RB>
__device__ __forceinline__ int col_operand(int lane, int dt, int t) {
  const int i = lane & 15, g = lane >> 4, h = g >> 1;
  const int row = 8 * t + 4 * h + (i >> 2);
  const int lc = 4 * dt + 2 * (g & 1) + ((i & 3) >> 1);
  return row * RB + ((lc ^ row_key<RB>(row)) << 4) + 8 * (i & 1);
}

typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;

__device__ __forceinline__ bf16x8 read_cols(const char* a, const char* b) {
  typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
  const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(s16x4*)a);
  const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(s16x4*)b);
  typedef __attribute__((__vector_size__(8 * sizeof(short)))) short s16x8;
  const s16x8 z = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, z);
}

}  // namespace ca
