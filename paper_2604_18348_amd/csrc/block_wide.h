// What the bf16 kernels for many rows share: tiles of 32 (forward) or 64 rows staged in LDS by direct loads, read by all waves (internal).
//
// 32x32x16 products (v_mfma_f32_32x32x16_bf16): half the LDS reads a product of the 16x16 tiles.  A result holds in lane l column
// l % 32 and, in value v, row 8 (v / 4) + 4 (l / 32) + v % 4; eight consecutive values are the operand of the next product, whose
// other operand is read column-wise (two transposing reads: rows 4 (l / 32) .. + 3 and 8 further) to match.
#pragma once

#include "block.h"

namespace adac {

typedef __attribute__((address_space(3))) void lds_void_t;

constexpr int TILE = 64;               // rows of a tile of the gradients, staged as four sixteenths of pages

// Rows of D bf16 in LDS, unpadded.  Piece q (16 bytes) of row r sits in slot q ^ swz(r).  Sixteen rows that are read at one piece
// (operands that are rows) lie in sixteen different slots, and the four rows of a transposing read (operands that are columns: 64
// bytes of rows 4 i .. + 3) in four different 64-byte groups: neither read meets a bank twice.
template <int D> __device__ __forceinline__ int swz(int r) {
  return D == 128 ? ((r & 3) << 2 | ((r >> 2) & 3)) : (((r >> 1) & 1) << 2 | ((r >> 2) & 3));
}
// Byte addresses of a lane inside a tile: its row operand (row l % 32, dimensions 16 ks + 8 (l / 32) ..) and, for column block db, the
// first of its two transposing reads (rows 4 (l / 32) .. + 3 of sixteen; the second is 8 rows on, whose slots are other ones).
template <int D> __device__ __forceinline__ int row_operand(int lane, int ks) { const int c = lane & 31; return c * D * 2 + (((ks * 2 + (lane >> 5)) ^ swz<D>(c)) * 16); }
template <int D> __device__ __forceinline__ int col_operand(int lane, int db, int second) {
  const int i16 = lane & 15, r = 4 * (lane >> 5) + (i16 >> 2) + 8 * second, q = db * 4 + 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
  return r * D * 2 + ((q ^ swz<D>(r)) * 16) + 8 * (i16 & 1);
}

__device__ __forceinline__ bf16x8_t join_tr(s16x4_tr lo, s16x4_tr hi) {
  union { s16x4_tr h[2]; bf16x8_t v; } u{{lo, hi}};
  return u.v;
}
__device__ __forceinline__ s16x4_tr read_tr(const char* p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_t*)p); }

// Eight values of a result (8 s2 .. + 7) as the operand of the next product.
__device__ __forceinline__ bf16x8_t pack8(const f32x16_t& x, int s2) {
  union { uint32_t w[4]; bf16x8_t v; } u;
#pragma unroll
  for (int j = 0; j < 4; ++j) u.w[j] = pack_bf16x2(x[8 * s2 + 2 * j], x[8 * s2 + 2 * j + 1]);
  return u.v;
}
// ... and their sum, of the rounded values
__device__ __forceinline__ float sum8(const bf16x8_t& v, float c) {
  const bf16x2_t one = {(__bf16)1.0f, (__bf16)1.0f};
  union { bf16x8_t v; bf16x2_t w[4]; } u{v};
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_fdot2_f32_bf16(u.w[j], one, c, false);
  return c;
}

__device__ __forceinline__ f32x16_t mfma32(const bf16x8_t& a, const bf16x8_t& b, const f32x16_t& c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16_t zero16() {
  f32x16_t z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// A launch's workgroups go to the 8 XCDs in turn, and each XCD has an L2 of its own, which the keys (or the rows) of about one head of a
// sequence fill.  So a head's workgroups stay on one XCD, one head after the other; where the heads of all sequences are no
// multiple of 8, each goes to `split` XCDs, every split-th workgroup to each.
struct HeadItem { int head, item; };                 // head < 0: none
__device__ __forceinline__ HeadItem xcd_item(int id, int heads, int items, int split) {
  const int per = (items + split - 1) / split, unit = (id & 7) + 8 * ((id >> 3) / per), item = (id >> 3) % per * split + unit % split;
  return {item < items ? uniform(unit / split) : -1, uniform(item)};
}
static inline int xcd_split(long long heads) { return heads % 8 == 0 ? 1 : heads % 4 == 0 ? 2 : heads % 2 == 0 ? 4 : 8; }
static inline long long xcd_grid(long long heads, long long items) { const int s = xcd_split(heads); return heads * s * ((items + s - 1) / s); }

}  // namespace adac
