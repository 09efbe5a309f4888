// What the bf16 kernels for many rows share: tiles of 32 (forward) or 64 rows staged in LDS by direct loads, read by all waves; the forward walks (internal).
//
// 32x32x16 products (v_mfma_f32_32x32x16_bf16): half the LDS reads a product of the 16x16 tiles.  A result holds in lane l column
// l % 32 and, in value v, row 8 (v / 4) + 4 (l / 32) + v % 4; eight consecutive values are the operand of the next product, whose
// other operand is read column-wise (two transposing reads: rows 4 (l / 32) .. + 3 and 8 further) to match.
#pragma once

#include "prefix_part.h"

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

// NW waves of 32 rows each.  A tile's keys and values go global -> LDS directly, 16 bytes a lane, one tile ahead of the products.  Rows past
// a sequence's end are read from the last row there is in their sixteenth (or the page's first) and masked: nothing behind the end is
// touched.  Bound by what lies between the products (exponentials, roundings, LDS reads), so waves a SIMD count: tiles of 32 keys and three
// waves (two with NW = 2) against 64 keys and two, or one: 3 sequences up to 8 192 tokens, 32 pages of 64, 16 / 4 heads, d = 128 385 us
// (489), 17 776 tokens, 30 heads, d = 64 730 (744), chunks of 2 x 1 024 tokens, NW = 2, d = 128 193 (303).
template <int D, int NW, bool PART> struct WideLds {
  static constexpr int TILEB = 32 * D * 2, STAGES = PART ? 3 : 2;
  __align__(16) char lds[STAGES * 2 * TILEB];
  int2 pages_l[LIST];
  int32_t counts[NW];
};
// PART: a share of a group's or a sequence's pages (prefix_part.h), whose result is left as a partial one.  TWO: weights in two parts (block_prefix.hip).
template <int D, int NW, bool PART, bool TWO, typename Args>
__device__ __forceinline__ void wide_rows(const Args& a, int rts, int split, WideLds<D, NW, PART>& sh) {
  constexpr int NT = NW * 64, KS = D / 16, DB = D / 32, CH = D / 8, ROWB = D * 2;
  constexpr int TK = 32, PARTS = TK / 16;      // keys a tile: one product's rows
  constexpr int PT = TK * CH / NT, TILEB = TK * ROWB;
  constexpr int STAGES = WideLds<D, NW, PART>::STAGES;
  char* const lds = sh.lds;
  int2* const pages_l = sh.pages_l;
  int32_t* const counts = sh.counts;
  const BlockDims& m = a.m;
  int hk, b, i = 0, t0, rows, base_row, from = 0, to = INT32_MAX;      // pages or entries of the list
  BlockSeq s;
  Part part;
  if constexpr (PART) {
    if (!part_of(a, blockIdx.x, part)) return;
    hk = part.hk; b = part.b; s = part.s; t0 = part.t0; rows = part.rows; base_row = part.base_row; from = part.from; to = part.to;
  } else {
    const HeadItem it = xcd_item(blockIdx.x, m.B * m.Hkv, m.nb * rts, split);
    if (it.head < 0) return;
    const int rt = it.item % rts;
    i = it.item / rts; hk = it.head % m.Hkv; b = it.head / m.Hkv;
    s = block_seq(m, b);
    t0 = i * m.qblock; rows = min(m.qblock, s.nq - t0) * m.G; base_row = rt * NT / 2;
    if (t0 >= s.nq || base_row >= rows) return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, hb = lane >> 5;

  const int row = base_row + wave * 32 + c, tok = t0 + row / m.G, head = hk * m.G + row % m.G;
  QueryRow query{s.q0 + tok, -1};
  if constexpr (PART) { if (row < rows) query = part_query(a, part, tok); }
  const bool there = PART ? query.lim >= 0 : row < rows;
  bf16x8_t qf[KS];
  {
    const bf16raw* const p = (const bf16raw*)a.q + (long long)query.t * a.qs.token + (long long)head * a.qs.head + hb * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4_t w = there ? *(const u32x4_t*)(p + ks * 16) : u32x4_t{0, 0, 0, 0};
      qf[ks] = *(const bf16x8_t*)&w;
    }
  }
  const int lim = there ? (PART ? query.lim : m.causal ? min(s.n, s.first + tok + 1) : s.n) : INT32_MAX;      // (a row that is not there needs no mask)
  const int wave_first = base_row + wave * 32;
  const bool wave_has_rows = wave_first < rows;
  int minlim = m.causal ? min(s.n, s.first + t0 + wave_first / m.G + 1) : s.n;       // keys below: seen by all rows of the wave
  const int last = min(base_row + NT / 2, rows) - 1;
  int maxlim = m.causal ? min(s.n, s.first + t0 + last / m.G + 1) : s.n;
  if constexpr (PART) {
    int low = lim;
#pragma unroll
    for (int x = 1; x < 32; x *= 2) low = min(low, __shfl_xor(low, x));
    minlim = uniform(low); maxlim = s.n;
  }
  const int pages = maxlim > 0 ? (maxlim + m.page - 1) >> m.lpage : 0;
  const int32_t* const list = !PART && a.sel ? a.sel + (((long long)b * m.nb + i) * m.Hkv + hk) * m.topk : nullptr;
  const int entries = list ? m.topk : min(pages, to);

  f32x16_t oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = zero16();
  // The weights are taken relative to a reference that moves only when a tile's sum leaves its range (see below); from where it
  // starts, tiles a row sees nothing of leave sum and accumulator at zero.
  const float sc = a.scale_log2e;
  float mref = softmax_start(sc), lrun = 0.f;

  int lrow[PT], piece[PT];                         // this thread's pieces of a tile
#pragma unroll
  for (int x = 0; x < PT; ++x) {
    const int item = tid + x * NT;
    lrow[x] = item / CH;
    piece[x] = ((item % CH) ^ swz<D>(lrow[x])) * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void_t*)lds;
  const int lsub = m.lpage - 4, ktok = (int)(a.ks.token * 2), vtok = (int)(a.vs.token * 2);
  int kaddr[KS], vaddr[DB][2];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kaddr[ks] = row_operand<D>(lane, ks);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 2; ++x) vaddr[db][x] = col_operand<D>(lane, db, x);

  for (int e0 = from; e0 < entries; e0 += LIST) {
    const int n = fill_list<NT>(m, b, list, e0, 1, entries, pages, pages_l, counts);
    const int parts = n << lsub, tiles = (parts + PARTS - 1) / PARTS;
    if (!tiles) continue;
    auto issue = [&](int stage, int t) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < PT; ++x) {                // a wave's request lies inside one sixteenth of a page
        const int part = min(t * PARTS + (((wave * 64 + x * NT) / CH) >> 4), parts - 1);
        const int2 pp = pages_l[part >> lsub];
        const int pg = uniform(pp.x), phys = uniform(pp.y);
        int sub = part & ((1 << lsub) - 1), have = s.n - ((pg << m.lpage) + sub * 16);      // rows of it that exist
        if (have <= 0) { sub = 0; have = 1; }
        const int r = min(lrow[x] & 15, have - 1);
        const uint32_t dst = lds0 + stage * 2 * TILEB + (wave * 64 + x * NT) * 16;
        dma_b128(dst, (uint32_t)(r * ktok + piece[x]), uniform((const char*)a.k + row_at(m, s, a.ks, phys, pg, sub, hk) * 2));
        dma_b128(dst + TILEB, (uint32_t)(r * vtok + piece[x]), uniform((const char*)a.v + row_at(m, s, a.vs, phys, pg, sub, hk) * 2));
      }
    };
    issue(0, 0);
    if constexpr (STAGES == 2) {
      wait_vmcnt<0>();
      lds_barrier();
    } else {
      static_assert(STAGES == 3, "the waits below count the loads of one tile behind the present one");
      if (tiles > 1) issue(1, 1);
    }
    int stage = 0;
    for (int t = 0; t < tiles; ++t) {
      if constexpr (STAGES == 2) {
        if (t + 1 < tiles) issue((t + 1) & 1, t + 1);
        stage = t & 1;
      } else {                                      // two tiles on their way: the prefix of one group waits for memory, not for products
        if (t + 1 < tiles) wait_vmcnt<2 * PT>();
        else wait_vmcnt<0>();
        lds_barrier();
        if (t) stage = stage == 2 ? 0 : stage + 1;
        if (t + 2 < tiles) issue(stage == 0 ? 2 : stage - 1, t + 2);
      }
      if (wave_has_rows) {
        const char* const kt = lds + stage * 2 * TILEB;
        const char* const vt = kt + TILEB;
        f32x16_t sacc = zero16();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sacc = mfma32(*(const bf16x8_t*)(kt + kaddr[ks]), qf[ks], sacc);
        int key0[PARTS];
        bool whole = true;
#pragma unroll
        for (int x = 0; x < PARTS; ++x) {
          const int part = t * PARTS + x, pg = uniform(pages_l[min(part, parts - 1) >> lsub].x);
          key0[x] = part < parts ? (pg << m.lpage) + (part & ((1 << lsub) - 1)) * 16 : INT32_MAX - 64;
          whole = whole && key0[x] + 16 <= minlim;
        }
        if (!whole) {
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (key0[v >> 3] + 8 * ((v >> 2) & 1) + 4 * hb + (v & 3) >= lim) sacc[v] = -INFINITY;
        }
        // p = 2^((s - reference) scale): any reference gives the same result as long as nothing overflows.  The row sum of the tile
        // tells (on the first tile with a score above -inf it is infinite): only then is the tile's maximum taken, the reference
        // moved up to it and the accumulator scaled.
        bf16x8_t pf[2], rest[2];                      // weights, and TWO: what their rounding leaves
        float rsum;
        auto weights = [&]() __attribute__((always_inline)) {
          const float off = mref * sc;
          float part[2];
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2) {
            union { uint32_t w[4]; bf16x8_t v; } u, r;
            part[s2] = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float p0 = __builtin_amdgcn_exp2f(fmaf(sacc[8 * s2 + 2 * j], sc, -off)), p1 = __builtin_amdgcn_exp2f(fmaf(sacc[8 * s2 + 2 * j + 1], sc, -off));
              u.w[j] = pack_bf16x2(p0, p1);
              if constexpr (TWO) r.w[j] = rounding_rest(p0, p1, u.w[j]);
              part[s2] += p0;                       // (not the rounded ones: the sum's logarithm is an output)
              part[s2] += p1;
            }
            pf[s2] = u.v;
            if constexpr (TWO) rest[s2] = r.v;
          }
          rsum = part[0] + part[1];
        };
        weights();
        if (__any(!(rsum <= 65536.f))) {
          float top = sacc[0];
#pragma unroll
          for (int v = 0; v < 16; ++v) top = fmaxf(top, sacc[v]);
          top = fmaxf(top, __shfl_xor(top, 32));
          const float next = fmaxf(mref, top), alpha = __builtin_amdgcn_exp2f((mref - next) * sc);
          mref = next;
          lrun *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
          weights();
        }
        lrun += rsum;
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          const char* const p = vt + 16 * s2 * ROWB;
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const bf16x8_t cols = join_tr(read_tr(p + vaddr[db][0]), read_tr(p + vaddr[db][1]));
            if constexpr (TWO) oacc[db] = mfma32(cols, rest[s2], oacc[db]);
            oacc[db] = mfma32(cols, pf[s2], oacc[db]);
          }
        }
      }
      if constexpr (STAGES == 2) {
        wait_vmcnt<0>();
        lds_barrier();
      }
    }
    lds_barrier();                                  // before the list is filled again
  }

  if (!there) return;
  const float all = lrun + __shfl_xor(lrun, 32), inv = all == 0.f ? 0.f : 1.f / all;
  if constexpr (PART) {
    const long long rec = part.rec + wave * 32 + c;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *(f32x4_t*)(part.o + rec * D + db * 32 + 8 * x + 4 * hb) = f32x4_t{oacc[db][4 * x], oacc[db][4 * x + 1], oacc[db][4 * x + 2], oacc[db][4 * x + 3]};
    if (hb == 0) { part.ml[rec * 2] = mref * sc; part.ml[rec * 2 + 1] = all; }
    return;
  }
  bf16raw* const out = (bf16raw*)a.o + (long long)(s.q0 + tok) * a.os.token + (long long)head * a.os.head + 4 * hb;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *(uint2*)(out + db * 32 + 8 * x) = uint2{pack_bf16x2(oacc[db][4 * x] * inv, oacc[db][4 * x + 1] * inv), pack_bf16x2(oacc[db][4 * x + 2] * inv, oacc[db][4 * x + 3] * inv)};
  if (hb == 0 && a.lse) a.lse[(long long)(s.q0 + tok) * m.Hq + head] = all == 0.f ? -INFINITY : fmaf(mref, sc, __builtin_amdgcn_logf(all)) * LN2;
}

// The same walk over 4-bit pages, for parts.  A tile's codes come two tiles ahead into registers and go to LDS as bfloat16: those
// of keys by themselves, those of values less 8.  Per group g of 64 dimensions
//   scores   sum of step_g (c . q) + low_g sum q, scaled: the latter one more product, of (low, low, low) with three bfloat16 parts of sum q;
//   values   weights times step_g, in two bfloat16 parts or rounded to one (it weighs codes about their middle), times c - 8, and the sum of
//            weights times low_g + 8 step_g, unrounded.
// Steps are applied to 16 keys a lane, which reads them from LDS (24 of 48 wide reads a tile).  No unit is full: vector arithmetic, most of it
// from codes to bfloat16, has half of the cycles, LDS a quarter, the matrix cores a sixth; each tile ends at a barrier, and a wave waits 40 % of its
// time.  128 rows over 16 384 keys of 8 heads, d = 128, with the rows' own keys: 100 us by the kernel for few rows, 53 staged and 20 for the latter.
// Two waves a workgroup, 64 rows, where no more are there: 64 sequences in 4 groups over 8 192 keys 66 -> 52 us (weights rounded once; 55 in two parts).
template <int D, int NW> struct CodesLds {
  static constexpr int TK = 32, NG = D / 64, TILEB = TK * D * 2;
  __align__(16) char lds[4 * TILEB];
  __align__(16) float kstep_l[2][NG][TK], vstep_l[2][NG][TK], vlow_l[2][NG][TK];
  uint32_t klow_l[2][TK][NG];
  int2 pages_l[LIST];
  int32_t counts[NW];
};
template <int D, int NW, bool TWO>
__device__ __forceinline__ void wide_codes(const PrefixArgs& a, CodesLds<D, NW>& sh) {
  constexpr int NT = NW * 64, KS = D / 16, DB = D / 32, NG = D / 64, ROWB = D * 2, WORDS = D / 8;      // words of eight codes a row
  constexpr int TK = 32, PT = TK * WORDS / NT, TILEB = TK * ROWB;
  static_assert(2 * TK * NG <= NT, "a thread has one pair of a key or value and group");
  char* const lds = sh.lds;
  auto &kstep_l = sh.kstep_l, &vstep_l = sh.vstep_l, &vlow_l = sh.vlow_l;
  auto& klow_l = sh.klow_l;
  int2* const pages_l = sh.pages_l;
  int32_t* const counts = sh.counts;
  const BlockDims& m = a.m;
  Part part;
  if (!part_of(a, blockIdx.x, part)) return;
  const BlockSeq& s = part.s;
  const int hk = part.hk, b = part.b, rows = part.rows, base_row = part.base_row, from = part.from, to = part.to;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, hb = lane >> 5;

  const int row = base_row + wave * 32 + c, tok = part.t0 + row / m.G, head = hk * m.G + row % m.G;
  const QueryRow query = row < rows ? part_query(a, part, tok) : QueryRow{0, -1};
  const bool there = query.lim >= 0;
  const int lim = there ? query.lim : INT32_MAX;
  const float sc = a.scale_log2e;
  bf16x8_t qf[KS], qsum;
  {
    const bf16raw* const p = (const bf16raw*)a.q + (long long)query.t * a.qs.token + (long long)head * a.qs.head + hb * 8;
    float sum[NG];
#pragma unroll
    for (int x = 0; x < NG; ++x) sum[x] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4_t w = there ? *(const u32x4_t*)(p + ks * 16) : u32x4_t{0, 0, 0, 0};
      qf[ks] = *(const bf16x8_t*)&w;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[ks / 4] += __uint_as_float(w[j] << 16) + __uint_as_float(w[j] & 0xFFFF0000u);
    }
    uint32_t h[6] = {0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int x = 0; x < NG; ++x) {
      float v = (sum[x] + __shfl_xor(sum[x], 32)) * sc;
#pragma unroll
      for (int y = 0; y < 3; ++y) { h[3 * x + y] = __float_as_uint(v) >> 16; v -= __uint_as_float(h[3 * x + y] << 16); }      // (cut: what is left is exact)
    }
    union { uint32_t w[4]; bf16x8_t v; } u{{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, 0}};
    if (hb) u.w[0] = u.w[1] = u.w[2] = 0;
    qsum = u.v;
  }
  const bool wave_has_rows = base_row + wave * 32 < rows;
  int minlim = lim;
#pragma unroll
  for (int x = 1; x < 32; x *= 2) minlim = min(minlim, __shfl_xor(minlim, x));
  minlim = uniform(minlim);

  f32x16_t oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = zero16();
  // The weights are taken relative to a reference (scaled here) that moves only when a tile's sum leaves its range, as above.
  float mref = -3.4028e38f, lrun = 0.f, corr[NG];
#pragma unroll
  for (int x = 0; x < NG; ++x) corr[x] = 0.f;

  int kaddr[KS], vaddr[DB][2];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kaddr[ks] = row_operand<D>(lane, ks);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 2; ++x) vaddr[db][x] = col_operand<D>(lane, db, x);

  const int lsub = m.lpage - 4;
  for (int e0 = from; e0 < to; e0 += LIST) {
    const int n = fill_list<NT>(m, b, nullptr, e0, 1, to, to, pages_l, counts);
    const int parts = n << lsub, count = (parts + 1) / 2;
    if (!count) continue;
    struct Raw { uint32_t kc[PT], vc[PT], pair; } next, later;      // one and two tiles ahead
    const auto fetch = [&](Raw& f, int t) __attribute__((always_inline)) {      // (past the last: that one again, masked; behind the end lies
                                                      // anything: its weight of 0 must meet a number)
      long long at[2];                                // the rows of the pool where the sixteenths start
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int part = min(t * 2 + x, parts - 1);
        at[x] = (((long long)uniform(pages_l[part >> lsub].y) * m.Hkv + hk) << m.lpage) + (part & ((1 << lsub) - 1)) * 16;
      }
#pragma unroll
      for (int x = 0; x < PT; ++x) {
        const int item = tid + x * NT, half = ((wave * 64 + x * NT) / WORDS) >> 4;
        const uint32_t off = ((item / WORDS & 15) * WORDS + item % WORDS) * 4;
        f.kc[x] = *(const uint32_t*)((const char*)a.k + (half ? at[1] : at[0]) * (WORDS * 4) + off);
        f.vc[x] = *(const uint32_t*)((const char*)a.v + (half ? at[1] : at[0]) * (WORDS * 4) + off);
      }
      if (tid < 2 * TK * NG) {
        const int r = tid / NG % TK, part = min(t * 2 + (r >> 4), parts - 1);
        const int2 pp = pages_l[part >> lsub];
        const int in = (part & ((1 << lsub) - 1)) * 16 + (r & 15);
        f.pair = (pp.x << m.lpage) + in < s.n ? (tid < TK * NG ? a.km : a.vm)[((((long long)pp.y * m.Hkv + hk) << m.lpage) + in) * NG + tid % NG] : 0;
      }
    };
    const auto expand = [&](const Raw& f, int stage) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < PT; ++x) {
        const int item = tid + x * NT, r = item / WORDS, at = r * ROWB + ((item % WORDS) ^ swz<D>(r)) * 16;
        u32x4_t k, v;
        const uint32_t even = f.kc[x] & 0x0F0F0F0Fu, odd = f.kc[x] >> 4 & 0x0F0F0F0Fu, mid = f.vc[x] ^ 0x88888888u;      // (a code less 8: four bits with a sign)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          k[j] = __float_as_uint((float)(even >> (8 * j) & 255)) >> 16 | __float_as_uint((float)(odd >> (8 * j) & 255));
          v[j] = __float_as_uint((float)((int)(mid << (28 - 8 * j)) >> 28)) >> 16 | __float_as_uint((float)((int)(mid << (24 - 8 * j)) >> 28));
        }
        *(u32x4_t*)(lds + stage * 2 * TILEB + at) = k;
        *(u32x4_t*)(lds + stage * 2 * TILEB + TILEB + at) = v;
      }
      if (tid < 2 * TK * NG) {
        const int r = tid / NG % TK, gr = tid % NG;
        const float step = __uint_as_float(f.pair << 16), low = __uint_as_float(f.pair & 0xFFFF0000u);
        if (tid < TK * NG) { kstep_l[stage][gr][r] = step * sc; klow_l[stage][r][gr] = f.pair >> 16; }
        else { vstep_l[stage][gr][r] = step; vlow_l[stage][gr][r] = fmaf(8.f, step, low); }
      }
    };
    fetch(later, 0);
    if (count > 1) fetch(next, 1);
    expand(later, 0);
    __syncthreads();
    for (int t = 0; t < count; ++t) {
      const int stage = t & 1;
      if (t + 2 < count) fetch(later, t + 2);
      if (wave_has_rows) {
        const char* const kt = lds + stage * 2 * TILEB;
        const char* const vt = kt + TILEB;
        f32x16_t sacc;
        {
          const uint32_t l0 = klow_l[stage][c][0], l1 = NG == 2 ? klow_l[stage][c][NG - 1] : 0;
          union { uint32_t w[4]; bf16x8_t v; } u{{l0 | l0 << 16, l0 | l1 << 16, l1 | l1 << 16, 0}};
          sacc = mfma32(u.v, qsum, zero16());
          f32x16_t y[NG];
#pragma unroll
          for (int x = 0; x < NG; ++x) {
            y[x] = zero16();
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) y[x] = mfma32(*(const bf16x8_t*)(kt + kaddr[4 * x + ks]), qf[4 * x + ks], y[x]);
          }
#pragma unroll
          for (int x = 0; x < NG; ++x)
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              const f32x4_t step = *(const f32x4_t*)&kstep_l[stage][x][8 * z + 4 * hb];
#pragma unroll
              for (int j = 0; j < 4; ++j) sacc[4 * z + j] = fmaf(step[j], y[x][4 * z + j], sacc[4 * z + j]);
            }
        }
        int key0[2];
        bool whole = true;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int part = t * 2 + x, pg = uniform(pages_l[min(part, parts - 1) >> lsub].x);
          key0[x] = part < parts ? (pg << m.lpage) + (part & ((1 << lsub) - 1)) * 16 : INT32_MAX - 64;
          whole = whole && key0[x] + 16 <= minlim;
        }
        if (!whole) {
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (key0[v >> 3] + 8 * ((v >> 2) & 1) + 4 * hb + (v & 3) >= lim) sacc[v] = -INFINITY;
        }
        float p[16], rsum;
        const auto weights = [&]() __attribute__((always_inline)) {
          float part[2] = {0.f, 0.f};
#pragma unroll
          for (int v = 0; v < 16; ++v) { p[v] = __builtin_amdgcn_exp2f(sacc[v] - mref); part[v >> 3] += p[v]; }
          rsum = part[0] + part[1];
        };
        weights();
        if (__any(!(rsum <= 65536.f))) {
          float top = sacc[0];
#pragma unroll
          for (int v = 0; v < 16; ++v) top = fmaxf(top, sacc[v]);
          top = fmaxf(top, __shfl_xor(top, 32));
          const float next = fmaxf(mref, top), alpha = __builtin_amdgcn_exp2f(mref - next);
          mref = next;
          lrun *= alpha;
#pragma unroll
          for (int x = 0; x < NG; ++x) corr[x] *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
          weights();
        }
        lrun += rsum;
#pragma unroll
        for (int x = 0; x < NG; ++x) {
          bf16x8_t pf[2], rest[2];
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2) {
            union { uint32_t w[4]; bf16x8_t v; } u, r;
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const int at = 16 * s2 + 8 * z + 4 * hb, v0 = 8 * s2 + 4 * z;
              const f32x4_t step = *(const f32x4_t*)&vstep_l[stage][x][at], low = *(const f32x4_t*)&vlow_l[stage][x][at];
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const float p0 = p[v0 + 2 * j] * step[2 * j], p1 = p[v0 + 2 * j + 1] * step[2 * j + 1];
                u.w[2 * z + j] = pack_bf16x2(p0, p1);
                if constexpr (TWO) r.w[2 * z + j] = rounding_rest(p0, p1, u.w[2 * z + j]);
              }
#pragma unroll
              for (int j = 0; j < 4; ++j) corr[x] = fmaf(p[v0 + j], low[j], corr[x]);
            }
            pf[s2] = u.v;
            if constexpr (TWO) rest[s2] = r.v;
          }
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2) {
            const char* const q = vt + 16 * s2 * ROWB;
#pragma unroll
            for (int db = 2 * x; db < 2 * x + 2; ++db) {
              const bf16x8_t cols = join_tr(read_tr(q + vaddr[db][0]), read_tr(q + vaddr[db][1]));
              if constexpr (TWO) oacc[db] = mfma32(cols, rest[s2], oacc[db]);
              oacc[db] = mfma32(cols, pf[s2], oacc[db]);
            }
          }
        }
      }
      if (t + 1 < count) { expand(next, stage ^ 1); next = later; }
      __syncthreads();
    }
  }

  if (!there) return;
  const float all = lrun + __shfl_xor(lrun, 32);
#pragma unroll
  for (int x = 0; x < NG; ++x) corr[x] += __shfl_xor(corr[x], 32);
  const long long rec = part.rec + wave * 32 + c;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      f32x4_t o;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = oacc[db][4 * x + j] + corr[db / 2];
      *(f32x4_t*)(part.o + rec * D + db * 32 + 8 * x + 4 * hb) = o;
    }
  if (hb == 0) { part.ml[rec * 2] = mref; part.ml[rec * 2 + 1] = all; }
}

}  // namespace adac
