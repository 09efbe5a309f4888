// Attention over a paged cache for groups of sequences that share their first pages: the shared pages meet the rows of the whole group
// at once, every sequence's rows its own pages behind them, both in one launch; then a row's partial results are joined.
//   o = sum_z 2^(m_z - m) o_z / sum_z 2^(m_z - m) l_z,  m = max_z m_z: every part z leaves o_z unnormalised, l_z and m_z, in fp32.
// Bound by the pages' bytes as long as a group has few hundred rows (one token of 32 sequences, 16 384 shared keys and up to 1 616 own, 32 / 8 heads, d = 128:
// 66 us for 176 MB and 25 MB of partial results, 3.0 TB/s; 89 by the kernel for few rows), then by what lies between the walk's products (128 sequences,
// 32 768 shared keys, 4 heads of keys: 141 us, 0.49 PFLOP/s, matrix cores 40 % of the cycles, vector arithmetic 42 %; 334).
//
// Weights of 16-bit and 4-bit calls enter the product with V in two parts, their rounding to bfloat16 and the rounding of what that leaves (up to 2^-16 of
// a weight): results are then off by their own rounding alone, 0.00166 relative to 64 bits, however many rows share the keys.  Rounded once they
// are off by 0.0020 to 0.0023, and take (whole calls, two parts -> one) 75 -> 71 us in the first call above, 159 -> 140 in the second, 36 -> 33.5 for 16 rows
// over 16 384 keys, 87 -> 80 for 64 sequences in 4 groups over 8 192 of 4 bits.  Blocks of 128 rows, chunks of a prompt, are rounded once, as by block_attn_wide: they
// are bound by products (16 sequences of up to 64 queries over 8 192 keys 185 -> 157 us, 4 bits 316 -> 266).
#include "block_few.h"
#include "block_wide.h"

namespace adac {

namespace {

template <typename T, int BITS, int D, int R>
__global__ __launch_bounds__(256, (few_waves<T, BITS, D, R>())) void prefix_few(PrefixArgs a, int first) {
  __shared__ FewLds<T, BITS, D> sh;
  few_rows<T, BITS, D, R, true>(a, 1, first + blockIdx.x, sh);
}
template <int D, bool TWO>
__global__ __launch_bounds__(256, 3) void prefix_wide(PrefixArgs a) {
  __shared__ WideLds<D, 4, true> sh;
  wide_rows<D, 4, true, TWO>(a, 1, 1, sh);
}
template <int D, int NW, bool TWO>
__global__ __launch_bounds__(NW * 64, 2) void prefix_codes(PrefixArgs a) {
  __shared__ CodesLds<D, NW> sh;
  wide_codes<D, NW, TWO>(a, sh);
}

// Joins a row's partial results: those of the pages its group shares, then those of its own.  D / 4 lanes read a result; `per` such
// slots share a row's results, each every per-th with a running maximum, and are joined through LDS.  Bound by waiting: 35 results of 1 024 rows,
// d = 128, 8.7 us (24 with one slot a row, 11 with an address a result in 64 bits).
template <typename T, int D>
__global__ __launch_bounds__(256) void prefix_join(PrefixArgs a, int per) {
  constexpr int LPR = D / 4, SLOTS = 256 / LPR;
  __shared__ __align__(16) float jo[SLOTS][D];
  __shared__ float jm[SLOTS][2];
  const BlockDims& m = a.m;
  const int slot = threadIdx.x / LPR, d0 = threadIdx.x % LPR * 4, part = slot % per;
  uint32_t id = blockIdx.x * (SLOTS / per) + slot / per;      // (a launch has below 2^24 workgroups)
  const int head = id % (uint32_t)m.Hq; id /= (uint32_t)m.Hq;
  const int i = id % (uint32_t)m.max_q; id /= (uint32_t)m.max_q;
  const int b = min((int)id, m.B - 1), hk = head / m.G;
  const BlockSeq s = block_seq(m, b);
  const bool there = (int)id < m.B && i < s.nq;
  const int t = s.q0 + i;
  int parts = 0, own = 0;
  long long rec = 0, trec = 0;
  int g = -1;                                          // the group, looked up by every lane: a wave's rows may be several sequences'
  if (a.gr.groups) {
    int lo = 0, hi = a.gr.groups;
    while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (a.gr.cu_group[mid] <= b) lo = mid; else hi = mid; }
    if (a.gr.cu_group[lo] <= b && b < a.gr.cu_group[lo + 1]) g = lo;
  }
  if (there) {
    Group group{0, 0, 0, 0, 0};
    if (g >= 0) {
      group = group_at(m, a.gr, g);
      const int query = a.gr.slots ? b * a.gr.slots + i : t, x = (query - group.q0) * m.G + head % m.G;
      rec = ((long long)(first_tile(m, group.q0, g, a.TR) + x / a.TR) * m.Hkv + hk) * a.shares * a.TR + x % a.TR;
      parts = group.pages && query >= group.q0 && query < group.q1 ? splits_of(m, group.pages, a.shares, a.gkeys) : 0;      // (else rows do not ascend)
    }
    own = splits_of(m, ((s.n + m.page - 1) >> m.lpage) - group.pages, a.tshares, a.tkeys);
    const int blk = i / m.qblock, row = (i - blk * m.qblock) * m.G + head % m.G, rt = row / a.TT;
    trec = (((((long long)b * m.Hkv + hk) * m.nb + blk) * a.rts + rt) * a.tshares) * a.TT + row % a.TT;
  }
  float top = -INFINITY, all = 0.f;
  f32x4_t o{0.f, 0.f, 0.f, 0.f};
  // every per-th of `count` results, `rows` rows apart, from the z-th on
  const auto add = [&](const float* po, const float* pml, int z, int count, int rows) __attribute__((always_inline)) {
    for (; z < count; z += 2 * per) {
      float mx[2], sum[2];
      f32x4_t v[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        mx[u] = -INFINITY; sum[u] = 0.f; v[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        if (z + u * per < count) {
          const uint32_t x = (uint32_t)(z + u * per) * rows;      // (below 2^32 / 4 D: a launch has no more workgroups than places)
          v[u] = *(const f32x4_t*)(po + x * D);
          mx[u] = pml[x * 2]; sum[u] = pml[x * 2 + 1];
        }
      }
      const float next = fmaxf(fmaxf(mx[0], mx[1]), top);      // (finite: a result's reference is)
      const float f0 = __builtin_amdgcn_exp2f(top - next);
      all *= f0; o *= f0;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const float f = __builtin_amdgcn_exp2f(mx[u] - next);
        all = fmaf(f, sum[u], all);
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = fmaf(f, v[u][j], o[j]);
      }
      top = next;
    }
  };
  add(a.group_o + rec * D + d0, a.group_ml + rec * 2, part, parts, a.TR);
  add(a.tail_o + trec * D + d0, a.tail_ml + trec * 2, (part - parts) & (per - 1), own, a.TT);
  if (per > 1) {
    *(f32x4_t*)&jo[slot][d0] = o;
    if (d0 == 0) { jm[slot][0] = top; jm[slot][1] = all; }
    __syncthreads();
    if (part) return;
    for (int z = 1; z < per; ++z) {
      const float other = jm[slot + z][0], next = fmaxf(top, other);
      if (other == -INFINITY) continue;                // (a slot without a result)
      const float f0 = __builtin_amdgcn_exp2f(top - next), f = __builtin_amdgcn_exp2f(other - next);
      all = fmaf(f, jm[slot + z][1], all * f0);
      const f32x4_t v = *(const f32x4_t*)&jo[slot + z][d0];
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = fmaf(f, v[j], o[j] * f0);
      top = next;
    }
  }
  if (!there) return;
  o *= all == 0.f ? 0.f : 1.f / all;
  T* const out = (T*)a.o + (long long)t * a.os.token + (long long)head * a.os.head + d0;
  if constexpr (sizeof(T) == 2) *(uint2*)out = uint2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
  else *(f32x4_t*)out = o;
  if (d0 == 0 && a.lse) a.lse[(long long)t * m.Hq + head] = all == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(all)) * LN2;
}

// Which kernel, what it is given: fills a's shape.  `rows`, `trows`: of partial results.
constexpr long long FAR = 1 << 25;                    // tokens this far apart: offsets inside a page pass 32 bits
struct PrefixShape { bool wide, two; int R; size_t rows, trows; };      // two: weights in two parts
PrefixShape shape_of(int dtype, int bits, PrefixArgs* a) {
  const BlockDims& m = a->m;
  PrefixShape s;
  const long long most = (long long)m.B * m.max_q, queries = m.q_rows < most ? m.q_rows : most;
  const int groups = a->gr.groups, block = m.qblock * m.G;
  const long long rows = groups ? (queries * m.G + groups - 1) / groups : block;      // of a group, on average
  const long long keys = (long long)m.max_pages << m.lpage;
  // Tiles of 128 rows staged for four waves (d = 128, 8 heads of keys, before the join): 16 rows over 16 384 keys 30 us (41 by prefix_few), over 2 048 and
  // 1 024 (d = 64) 17 and 9 (15, 10); 8 rows 29 (28); 8 groups of 4 rows over 8 192 62 (54).  4 bits need a second launch for the rows' own keys
  // and spread 32 KB of bfloat16 a tile: 32 rows over 16 384 keys 43 (64), over 2 048 28 (29), over 1 024 (d = 64) 19 (13); 16 rows over 4 096 30 (22).
  s.wide = dtype == ADACLUSTER_BF16 && (block > 16 || (bits ? rows > 16 && rows * keys > (1 << 16) : rows > 4)) &&
           (bits || (a->ks.token < FAR && a->vs.token < FAR));
  s.two = block < 128;
  s.R = rows > 16 || block > 16 ? 2 : 1;
  a->TR = s.wide ? (bits && rows <= 64 && block <= 64 ? 64 : 128) : 16 * s.R;
  a->TT = s.wide ? (bits && block <= 16 ? 16 : bits ? a->TR : block > 32 ? 128 : 32) : 16 * s.R;
  a->gr.slots = m.q_rows > most ? m.max_q : 0;
  a->tiles = groups ? (int)(queries * m.G / a->TR) + groups : 0;
  a->rts = (block + a->TT - 1) / a->TT;
  const long long items = (long long)a->rts * m.nb * m.Hkv * m.B, busy = (rows + a->TR - 1) / a->TR * groups * m.Hkv;
  // Few tiles: the pages are split among the workgroups that the GPU holds at a time (three a CU; 128 own rows of up to 1 616 keys beside 32 768 x 128 rows
  // and 32 beside 16 384: 134 and 62 us; for two a CU 134 and 64, four 138 and 60, but 35 -> 41 for 16).  A share has four times as many keys as rows,
  // so that a partial result (four bytes a value) stays a quarter of what it is made of (128 rows over 16 384 keys: 43 us with 256 keys each, 36 with
  // 512), or 256; if that leaves CUs without one, as few as 128 (128 rows over 1 024 keys, d = 64: 21 -> 14 us; 64 over 4 096, d = 128: 27 -> 22).
  // (Both sides measured with weights rounded once.)  Keys are counted by the width of page_table, which the host knows, not by the sequences.
  const int places = s.wide ? (bits ? 512 : 768) : s.R == 1 ? 512 : 256;
  const auto share = [&](long long items, int rows, int* least) {
    const long long most = rows > 64 ? 4 * rows : 256, fill = keys * items / 256;
    *least = (int)(!s.wide || rows == 16 || fill > most ? most : fill < 128 ? 128 : fill);      // (few rows: a quarter for each wave of the 256)
    long long n = items > 0 ? places / items : 1;
    if (n > (keys + *least - 1) / *least) n = (keys + *least - 1) / *least;
    return (int)(n < 1 ? 1 : n);
  };
  a->shares = share(busy, a->TR, &a->gkeys);
  a->tshares = share(items, a->TT, &a->tkeys);
  a->split = xcd_split(m.Hkv);
  s.rows = (size_t)a->tiles * m.Hkv * a->shares * a->TR;
  s.trows = (size_t)items * a->tshares * a->TT;
  return s;
}

template <typename T, int BITS, int D>
void go(hipStream_t st, const PrefixShape& s, int wg, const PrefixArgs& a) {
  if constexpr (sizeof(T) == 2 && BITS == 0) {
    if (s.wide) { if (s.two) prefix_wide<D, true><<<wg, 256, 0, st>>>(a); else prefix_wide<D, false><<<wg, 256, 0, st>>>(a); return; }
  }
  if constexpr (sizeof(T) == 2 && BITS == 4) {
    if (s.wide) {
      // a sequence's own few rows take codes straight into their products, in a launch of their own
      const int n = a.TT == 16 ? a.grid : wg;
      if (n) {
        if (a.TR == 64) prefix_codes<D, 2, true><<<n, 128, 0, st>>>(a);      // (blocks of 64 rows at most)
        else if (s.two) prefix_codes<D, 4, true><<<n, 256, 0, st>>>(a);
        else prefix_codes<D, 4, false><<<n, 256, 0, st>>>(a);
      }
      if (wg > n) prefix_few<T, BITS, D, 1><<<wg - n, 256, 0, st>>>(a, n);
      return;
    }
  }
  if (s.R == 1) prefix_few<T, BITS, D, 1><<<wg, 256, 0, st>>>(a, 0);
  else prefix_few<T, BITS, D, 2><<<wg, 256, 0, st>>>(a, 0);
}

}  // namespace

size_t prefix_attn_bytes(int dtype, int bits, int d, const PrefixArgs& a) {
  size_t most = 0;
  for (const long long token : {0ll, FAR}) {            // (of any strides: who asks may not have them yet)
    PrefixArgs x = a;
    x.ks.token = x.vs.token = token;
    const PrefixShape s = shape_of(dtype, bits, &x);
    const size_t n = align_up(s.rows * d * 4, 256) + align_up(s.rows * 8, 256) + align_up(s.trows * d * 4, 256) + align_up(s.trows * 8, 256);
    if (n > most) most = n;
  }
  return most;
}

int launch_prefix_attn(hipStream_t st, int dtype, int bits, int d, PrefixArgs a, void* ws) {
  const PrefixShape s = shape_of(dtype, bits, &a);
  char* p = (char*)ws;
  const auto take = [&](size_t n) { char* const x = p; p += align_up(n, 256); return (float*)x; };
  a.group_o = take(s.rows * d * 4);
  a.group_ml = take(s.rows * 8);
  a.tail_o = take(s.trows * d * 4);
  a.tail_ml = take(s.trows * 8);
  const long long grid = a.tiles ? xcd_grid(a.m.Hkv, (long long)a.tiles * a.shares) : 0, wg = grid + (long long)a.rts * a.m.nb * a.m.Hkv * a.m.B * a.tshares;
  // the join: up to eight results a slot, and two workgroups a CU
  const int slots = 1024 / d;
  const long long rows = (long long)a.m.B * a.m.max_q * a.m.Hq;
  int per = 1;
  while (per < slots && (per * 8 < a.shares + a.tshares || rows * per < 512 * slots)) per *= 2;
  const long long jwg = (rows * per + slots - 1) / slots;
  if (!grid_fits(wg) || !grid_fits(jwg)) return ADACLUSTER_E_UNSUPPORTED;
  a.grid = (int)grid;
#define GO(T, D) if (bits) go<T, 4, D>(st, s, (int)wg, a); else go<T, 0, D>(st, s, (int)wg, a)
  if (dtype == ADACLUSTER_BF16) { if (d == 64) { GO(bf16raw, 64); } else { GO(bf16raw, 128); } }
  else { if (d == 64) { GO(float, 64); } else { GO(float, 128); } }
#undef GO
  if (int rc = launched()) return rc;
#define JOIN(T, D) prefix_join<T, D><<<(int)jwg, 256, 0, st>>>(a, per)
  if (dtype == ADACLUSTER_BF16) { if (d == 64) JOIN(bf16raw, 64); else JOIN(bf16raw, 128); }
  else { if (d == 64) JOIN(float, 64); else JOIN(float, 128); }
#undef JOIN
  return launched();
}

}  // namespace adac
