// Attention of few rows over listed pages: the walk of a workgroup (internal).
#pragma once

#include "prefix_part.h"

namespace adac {

// Keys and values of 16 rows as a lane takes them: of row lane % 16, pieces as the products want them.
//   BITS 0: the elements themselves.
//   BITS 4, bf16: of every 64 dimensions the 16 from 16 * quarter on, as two words of eight codes.  A code c becomes the bfloat16
//     128 + c (0x4300 | c: exact), two codes of a word at a time, which leaves the dimensions of a word in the order ORDER; steps
//     and lowest values enter behind the product, per group of 64:  k . q = step (k' . q) + (lo - 128 step) sum q.
//   BITS 4, fp32: the same 16 dimensions, as values lo + code * step, in order.
template <typename T, int BITS, int D> struct Raw {
  static constexpr int NF = D * sizeof(T) / 64;
  u32x4_t w[BITS == 4 ? D / 128 + (D == 64) : NF];      // 4 bits: two words of 64 dimensions
};
__host__ __device__ constexpr int code_order(int x) { return (x & 1) * 4 + (x >> 1); }      // dimension at place x of a word of codes

// piece f of a lane's row: index of its 16 bytes in a row of D elements
template <typename T, int BITS> __device__ __forceinline__ int piece_at(int f, int quarter) {
  if constexpr (BITS == 0) return 4 * f + quarter;
  else if constexpr (sizeof(T) == 2) return 8 * (f >> 1) + 2 * quarter + (f & 1);
  else return 16 * (f >> 2) + 4 * quarter + (f & 3);
}

template <typename T, int BITS, int D>
__device__ __forceinline__ void load_raw(Raw<T, BITS, D>& r, const void* base, long long row, int quarter, bool there) {
  if constexpr (BITS == 0) {
    const T* const p = (const T*)base + row;
#pragma unroll
    for (int f = 0; f < Raw<T, BITS, D>::NF; ++f) r.w[f] = there ? *(const u32x4_t*)(p + (4 * f + quarter) * Vec<T>::N) : u32x4_t{0, 0, 0, 0};
  } else {
    const uint2* const p = (const uint2*)((const char*)base + row) + quarter;      // (a row of codes is D / 2 bytes)
    uint2 a{0, 0}, b{0, 0};
    if (there) { a = p[0]; if constexpr (D == 128) b = p[4]; }
    r.w[0] = u32x4_t{a.x, a.y, b.x, b.y};
  }
}

// (4 bits, fp32: pair = (step, lowest) of the lane's row, a group)
template <typename T, int BITS, int D>
__device__ __forceinline__ void expand(RowFrag<T, D>& f, const Raw<T, BITS, D>& r, const uint32_t* pair, bool there) {
#pragma unroll
  for (int x = 0; x < Raw<T, BITS, D>::NF; ++x) {
    if constexpr (BITS == 0) f.p[x] = r.w[x];
    else if constexpr (sizeof(T) == 2) {
      const uint32_t c = r.w[0][x];
      // (constants in registers: an instruction then masks and joins, which literals do not allow)
      uint32_t mask = 0x000F000Fu, high = 0x43004300u;
      asm("" : "+v"(mask));
      asm("" : "+s"(high));
#pragma unroll
      for (int j = 0; j < 4; ++j) f.p[x][j] = (c >> (4 * j) & mask) | high;
    } else {
      const uint32_t c = r.w[0][x >> 1] >> (16 * (x & 1));
      const float step = __uint_as_float(pair[x >> 2] << 16), low = __uint_as_float(pair[x >> 2] & 0xFFFF0000u);
#pragma unroll
      for (int j = 0; j < 4; ++j) f.p[x][j] = there ? __float_as_uint(fmaf((float)(c >> (4 * j) & 15), step, low)) : 0u;
    }
  }
}

// 4 waves; a workgroup has R * 16 rows of one block of queries and a share of its list of keys, which its waves take in turns of
// 32 keys: a wave reads its keys and values straight from memory into registers (16 bytes a lane), passes the values through
// LDS of its own to have their columns, and keeps a running maximum and sum (fp32).  At the end the four waves' results are
// joined; with nsplit > 1 they are left as partial results, which block_attn_join joins.
//
// The product with V in 16 bits wants P in bfloat16 (the row sum is of the unrounded weights).  Up to 16 rows of 16-bit keys wait for memory,
// so there a weight enters in two parts, its rounding and the rounding of what that leaves (2^-16 of it): 64 sequences of up to 32 768
// tokens, 2 048 keys each, d = 128 219.9 us with one part, 220.6 with two, off from 64 bits by 0.0022 and 0.0017, of which 0.0017 is the
// rounding of O.  With more rows it is rounded (an error of half a step of bfloat16 of each weight); with 4-bit values the weights
// are multiplied by the steps of their keys first, and then rounded (in two parts 32 sequences over whole caches of up to 16 384 tokens
// 132.7 -> 140.7 us, for values that are off by half a step of 4 bits as it is).
// Attention over shared prefixes has them in two parts here, whatever the rows and bits (block_prefix.hip).
template <typename T, int BITS, int D> struct FewLds {
  static constexpr int VBYTES = 32 * D * sizeof(T), JBYTES = 4 * 16 * D * 4 + 4 * 16 * 2 * 4;
  static constexpr bool CODES = BITS == 4 && sizeof(T) == 2;
  __align__(16) char lds[4 * VBYTES > JBYTES ? 4 * VBYTES : JBYTES];
  __align__(16) float meta[CODES ? 4 : 1][2][CODES ? 32 : 1][2 * (D / 64)];      // a wave's 32 keys, values: (step, lowest), lowest of values + 8 steps
  int2 pages_l[LIST];
  int32_t counts[4];
};
// waves a SIMD that the registers are for
template <typename T, int BITS, int D, int R> constexpr int few_waves() { return R == 1 && !(sizeof(T) == 4 && BITS == 0 && D == 128) ? 2 : 1; }

// PART: a share of a group's or a sequence's pages (prefix_part.h), whose result is left as a partial one.
template <typename T, int BITS, int D, int R, bool PART, typename Args>
__device__ __forceinline__ void few_rows(const Args& a, int rts, int id, FewLds<T, BITS, D>& sh) {
  constexpr int NF = D * sizeof(T) / 64, ND = D / 16;
  constexpr bool CODES = BITS == 4 && sizeof(T) == 2;           // codes enter the products, steps behind them
  constexpr int NG = CODES ? D / 64 : 1, MW = D / 64;
  constexpr int VBYTES = FewLds<T, BITS, D>::VBYTES;
  char* const lds = sh.lds;
  auto& meta = sh.meta;
  int2* const pages_l = sh.pages_l;
  int32_t* const counts = sh.counts;
  const BlockDims& m = a.m;
  int hk, b, i = 0, t0, rows, base_row, split = 0, item = 0, e_first, every = 1, e_end = INT32_MAX;      // entries of the list: e_first, every every-th, below e_end
  BlockSeq s;
  Part part;
  if constexpr (PART) {
    if (!part_of(a, id, part)) return;
    hk = part.hk; b = part.b; s = part.s; t0 = part.t0; rows = part.rows; base_row = part.base_row;
    e_first = part.from; e_end = part.to;
  } else {
    every = a.nsplit;
    split = id % a.nsplit; id /= a.nsplit;
    item = id;
    const int rt = id % rts; id /= rts;
    i = id % m.nb; id /= m.nb;
    hk = id % m.Hkv; b = id / m.Hkv;
    s = block_seq(m, b);
    t0 = i * m.qblock; rows = min(m.qblock, s.nq - t0) * m.G; base_row = rt * R * 16;
    e_first = split;
    if (t0 >= s.nq || base_row >= rows) return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, quarter = lane >> 4;

  // queries: operand pieces, and the keys below `lim` that a row sees
  RowFrag<T, D> q[R];
  int lim[R];
  float qsum[R][NG];
  int part_min = INT32_MAX;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = base_row + r * 16 + n16, t = t0 + row / m.G;
    bool there = row < rows;
    int at = s.q0 + t;                                   // its row in the tensor
    if constexpr (PART) {
      const QueryRow query = there ? part_query(a, part, t) : QueryRow{0, -1};
      at = query.t;
      there = query.lim >= 0;
      lim[r] = there ? query.lim : INT32_MAX;
      part_min = min(part_min, lim[r]);
    } else {
      lim[r] = there ? (m.causal ? min(s.n, s.first + t + 1) : s.n) : INT32_MAX;      // (a row that is not there needs no mask)
    }
    const T* const p = (const T*)a.q + (long long)at * a.qs.token + (long long)(hk * m.G + row % m.G) * a.qs.head;
#pragma unroll
    for (int f = 0; f < NF; ++f) q[r].p[f] = there ? *(const u32x4_t*)(p + piece_at<T, BITS>(f, quarter) * Vec<T>::N) : u32x4_t{0, 0, 0, 0};
    if constexpr (CODES) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          u32x4_t& w = q[r].p[2 * g + c];
#pragma unroll
          for (int j = 0; j < 4; ++j) sum += __uint_as_float(w[j] << 16) + __uint_as_float(w[j] & 0xFFFF0000u);
          // dimensions 0..7 -> 0 4 1 5 2 6 3 7
          w = u32x4_t{(w[0] & 0xFFFFu) | w[2] << 16, w[0] >> 16 | (w[2] & 0xFFFF0000u), (w[1] & 0xFFFFu) | w[3] << 16, w[1] >> 16 | (w[3] & 0xFFFF0000u)};
        }
        qsum[r][g] = quarters_sum(sum);                  // (of 64 dimensions)
      }
    }
  }
  const int last = min(base_row + R * 16, rows) - 1;
  int maxlim = m.causal ? min(s.n, s.first + t0 + last / m.G + 1) : s.n;      // (no row sees further)
  int minlim = m.causal ? min(s.n, s.first + t0 + base_row / m.G + 1) : s.n;      // keys below: seen by all rows
  if constexpr (PART) {
#pragma unroll
    for (int x = 1; x < 16; x *= 2) part_min = min(part_min, __shfl_xor(part_min, x));
    maxlim = s.n; minlim = uniform(part_min);
  }
  const int pages = maxlim > 0 ? (maxlim + m.page - 1) >> m.lpage : 0;
  const int32_t* const list = !PART && a.sel ? a.sel + (((long long)b * m.nb + i) * m.Hkv + hk) * m.topk : nullptr;
  const int lsub = m.lpage - 4, entries = min(list ? m.topk : pages, e_end);

  // The weights are taken relative to a reference that moves only when a turn's sum leaves its range (see below); from where it
  // starts, turns a row sees nothing of leave sum and accumulator at zero.
  const float scale = a.scale_log2e;
  float ref[R], sum[R], corr[R][NG];
  f32x4_t acc[R][ND];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    ref[r] = softmax_start(scale); sum[r] = 0.f;
#pragma unroll
    for (int g = 0; g < NG; ++g) corr[r][g] = 0.f;
#pragma unroll
    for (int x = 0; x < ND; ++x) acc[r][x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  char* const vl = lds + wave * VBYTES;

  // What a turn reads, in registers one turn ahead (R > 1: in its own turn, the registers hold rows instead).
  struct Fetch {
    int key0[2];                                      // INT32_MAX - 64: no keys
    Raw<T, BITS, D> k[2], v[2];
    uint32_t pk[2][MW], pv[2][MW];                    // 4 bits: (step, lowest) of the lane's row
  };
  for (int e0 = e_first; e0 < entries; e0 += every * LIST) {
    const int halves = fill_list<256>(m, b, list, e0, every, entries, pages, pages_l, counts) << lsub, turns = (halves + 1) >> 1;
    auto fetch = [&](Fetch& f, int turn) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int half = 2 * turn + h, sub = half & ((1 << lsub) - 1);
        const bool some = half < halves;
        const int2 pp = pages_l[some ? half >> lsub : 0];
        const int pg = uniform(pp.x), phys = uniform(pp.y);
        f.key0[h] = some ? (pg << m.lpage) + sub * 16 : INT32_MAX - 64;
        const bool there = f.key0[h] + n16 < s.n;
        if constexpr (BITS == 4) {
          const long long at = ((long long)phys * m.Hkv + hk) * m.page + sub * 16 + n16;
          load_raw<T, BITS, D>(f.k[h], a.k, at * (D / 2), quarter, there);
          load_raw<T, BITS, D>(f.v[h], a.v, at * (D / 2), quarter, there);
#pragma unroll
          for (int x = 0; x < MW; ++x) {                  // (behind the end lies anything: its weight of 0 must meet a number)
            f.pk[h][x] = there ? a.km[at * MW + x] : 0;
            f.pv[h][x] = there ? a.vm[at * MW + x] : 0;
          }
        } else {
          load_raw<T, BITS, D>(f.k[h], a.k, row_at(m, s, a.ks, phys, pg, sub, hk) + n16 * a.ks.token, quarter, there);
          load_raw<T, BITS, D>(f.v[h], a.v, row_at(m, s, a.vs, phys, pg, sub, hk) + n16 * a.vs.token, quarter, there);
        }
      }
    };
    Fetch next;
    if (R == 1 && wave < turns) fetch(next, wave);
    for (int turn = wave; turn < turns; turn += 4) {
      if (R > 1) fetch(next, turn);
      int key0[2];
      RowFrag<T, D> k[2];
      float kp[2][4][2 * MW], vp[2][4][2 * MW];         // CODES: of keys 4 * quarter + j
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        key0[h] = next.key0[h];
        const bool there = key0[h] + n16 < s.n;
        expand<T, BITS, D>(k[h], next.k[h], next.pk[h], there);
        RowFrag<T, D> v;
        expand<T, BITS, D>(v, next.v[h], next.pv[h], there);
        compiler_fence();
#pragma unroll
        for (int f = 0; f < NF; ++f) *(u32x4_t*)(vl + lds_piece<T, D>(16 * h + n16, piece_at<T, BITS>(f, quarter))) = v.p[f];
        if constexpr (CODES) {
          if (quarter == 0) {
#pragma unroll
            for (int x = 0; x < MW; ++x) {
              const float ks = __uint_as_float(next.pk[h][x] << 16), vs = __uint_as_float(next.pv[h][x] << 16);
              meta[wave][0][16 * h + n16][2 * x] = ks;
              meta[wave][0][16 * h + n16][2 * x + 1] = __uint_as_float(next.pk[h][x] & 0xFFFF0000u);
              meta[wave][1][16 * h + n16][2 * x] = vs;
              meta[wave][1][16 * h + n16][2 * x + 1] = fmaf(8.f, vs, __uint_as_float(next.pv[h][x] & 0xFFFF0000u));
            }
          }
        }
      }
      compiler_fence();
      if constexpr (CODES) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int x = 0; x < 2 * MW; ++x) { kp[h][j][x] = meta[wave][0][16 * h + 4 * quarter + j][x]; vp[h][j][x] = meta[wave][1][16 * h + 4 * quarter + j][x]; }
      }
      if (R == 1 && turn + 4 < turns) fetch(next, turn + 4);

#pragma unroll
      for (int r = 0; r < R; ++r) {
        f32x4_t sc[2], p[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          sc[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          if constexpr (CODES) {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              const float start = -128.f * qsum[r][g];     // what the 128 of every code adds to a product
              f32x4_t x{start, start, start, start};
              x = mma(T{}, k[h].p[2 * g], q[r].p[2 * g], x);
              x = mma(T{}, k[h].p[2 * g + 1], q[r].p[2 * g + 1], x);
#pragma unroll
              for (int j = 0; j < 4; ++j)
                sc[h][j] = fmaf(kp[h][j][2 * g], x[j], fmaf(kp[h][j][2 * g + 1], qsum[r][g], sc[h][j]));
            }
          } else {
            sc[h] = dots(k[h], q[r]);
          }
          if (key0[h] + 16 > minlim) {
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[h][j] = key0[h] + 4 * quarter + j < lim[r] ? sc[h][j] : -INFINITY;
          }
        }
        // p = 2^((s - reference) scale): any reference gives the same result as long as nothing overflows.  The turn's sum tells (it
        // is infinite at a row's first score above -inf): only then is the maximum taken, the reference moved up to it and what
        // has been summed scaled.
        float rsum;
        auto weights = [&]() __attribute__((always_inline)) {
          const float off = ref[r] * scale;
          rsum = 0.f;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) { p[h][j] = __builtin_amdgcn_exp2f(fmaf(sc[h][j], scale, -off)); rsum += p[h][j]; }
        };
        weights();
        if (__any(!(rsum <= 65536.f))) {
          float top = ref[r];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, sc[h][j]);
          top = quarters_max(top);
          const float alpha = __builtin_amdgcn_exp2f((ref[r] - top) * scale);
          ref[r] = top;
          sum[r] *= alpha;
#pragma unroll
          for (int g = 0; g < NG; ++g) corr[r][g] *= alpha;
#pragma unroll
          for (int x = 0; x < ND; ++x) acc[r][x] *= alpha;
          weights();
        }
        sum[r] += rsum;
        if constexpr (CODES) {
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            // weights times steps, rounded here: what is taken off for the 128 has to be what the product adds.  8 more are taken off
            // and come back unrounded: the rounding then weighs codes about their middle, not from 0 up.
            const bf16x2_t one = {(__bf16)1.0f, (__bf16)1.0f};
            union { uint32_t w[4]; bf16x2_t b[4]; bf16x8_t v; } u, rest;
            float c = 0.f, back = corr[r][g];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int h = x >> 1, j = 2 * (x & 1);
              const float p0 = p[h][j] * vp[h][j][2 * g], p1 = p[h][j + 1] * vp[h][j + 1][2 * g];
              u.w[x] = pack_bf16x2(p0, p1);
              c = __builtin_amdgcn_fdot2_f32_bf16(u.b[x], one, c, false);
              if constexpr (PART) {
                rest.w[x] = rounding_rest(p0, p1, u.w[x]);
                c = __builtin_amdgcn_fdot2_f32_bf16(rest.b[x], one, c, false);
              }
              back = fmaf(p[h][j + 1], vp[h][j + 1][2 * g + 1], fmaf(p[h][j], vp[h][j][2 * g + 1], back));
            }
            corr[r][g] = fmaf(-136.f, c, back);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              if constexpr (PART) acc[r][4 * g + x] = mma_cols<D>(vl, 64 * g + 16 * x, lane, u.v, rest.v, acc[r][4 * g + x]);
              else acc[r][4 * g + x] = mma_cols<D>(vl, 64 * g + 16 * x, lane, u.v, acc[r][4 * g + x]);
            }
          }
        } else if constexpr (sizeof(T) == 2) {
          union { uint32_t w[4]; bf16x8_t v; } u{{pack_bf16x2(p[0][0], p[0][1]), pack_bf16x2(p[0][2], p[0][3]), pack_bf16x2(p[1][0], p[1][1]), pack_bf16x2(p[1][2], p[1][3])}};
          union { uint32_t w[4]; bf16x8_t v; } rest;
          constexpr bool TWO = PART || R == 1;
          if constexpr (TWO) {
#pragma unroll
            for (int x = 0; x < 4; ++x) rest.w[x] = rounding_rest(p[x >> 1][2 * (x & 1)], p[x >> 1][2 * (x & 1) + 1], u.w[x]);
          }
#pragma unroll
          for (int x = 0; x < ND; ++x) {
            if constexpr (TWO) acc[r][x] = mma_cols<D>(vl, 16 * x, lane, u.v, rest.v, acc[r][x]);
            else acc[r][x] = mma_cols<D>(vl, 16 * x, lane, u.v, acc[r][x]);
          }
        } else {
#pragma unroll
          for (int x = 0; x < ND; ++x) acc[r][x] = mma_cols<D>(T{}, vl, 16 * x, lane, p[0], p[1], acc[r][x]);
        }
      }
      compiler_fence();
    }
    __syncthreads();                                  // before the list is filled again
  }

  // join the four waves, 16 rows at a time: [wave][row][d], [wave][row] x {maximum, sum}
  float* const jo = (float*)lds;
  float* const jm = jo + 4 * 16 * D;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    __syncthreads();
    const float tot = quarters_sum(sum[r]);
    float c[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) c[g] = CODES ? quarters_sum(corr[r][g]) : 0.f;
#pragma unroll
    for (int x = 0; x < ND; ++x)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = 16 * x + 4 * quarter + j;
        const int dim = CODES ? (at & ~7) + code_order(at & 7) : at;
        jo[(wave * 16 + n16) * D + dim] = acc[r][x][j] + c[CODES ? x / 4 : 0];
      }
    if (quarter == 0) { jm[(wave * 16 + n16) * 2] = ref[r] * scale; jm[(wave * 16 + n16) * 2 + 1] = tot; }
    __syncthreads();
    const int jr = tid >> 4, row = base_row + r * 16 + jr, d0 = (tid & 15) * (D / 16);
    float top = -INFINITY, all = 0.f, o[D / 16];
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, jm[(w * 16 + jr) * 2]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int x = 0; x < D / 16; ++x) o[x] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(jm[(w * 16 + jr) * 2] - ref);
      all += f * jm[(w * 16 + jr) * 2 + 1];
#pragma unroll
      for (int x = 0; x < D / 16; ++x) o[x] = fmaf(f, jo[(w * 16 + jr) * D + d0 + x], o[x]);
    }
    if (row >= rows) continue;
    if (PART || a.nsplit > 1) {
      const long long rec = (PART ? part.rec : ((long long)item * a.nsplit + split) * (16 * R)) + r * 16 + jr;
      float *po = a.part_o, *pml = a.part_ml;
      if constexpr (PART) { po = part.o; pml = part.ml; }
#pragma unroll
      for (int x = 0; x < D / 16; x += 4) *(f32x4_t*)(po + rec * D + d0 + x) = f32x4_t{o[x], o[x + 1], o[x + 2], o[x + 3]};
      if (d0 == 0) { pml[rec * 2] = top; pml[rec * 2 + 1] = all; }
    } else {
      const int t = t0 + row / m.G, head = hk * m.G + row % m.G;
      const float inv = all == 0.f ? 0.f : 1.f / all;
#pragma unroll
      for (int x = 0; x < D / 16; ++x) o[x] *= inv;
      T* const out = (T*)a.o + (long long)(s.q0 + t) * a.os.token + (long long)head * a.os.head + d0;
#pragma unroll
      for (int x = 0; x < D / 16; x += 4) {
        if constexpr (sizeof(T) == 2) *(uint2*)(out + x) = uint2{pack_bf16x2(o[x], o[x + 1]), pack_bf16x2(o[x + 2], o[x + 3])};
        else *(f32x4_t*)(out + x) = f32x4_t{o[x], o[x + 1], o[x + 2], o[x + 3]};
      }
      if (d0 == 0 && a.lse) a.lse[(long long)(s.q0 + t) * m.Hq + head] = all == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(all)) * LN2;
    }
  }
}

}  // namespace adac
