// Attention over a paged cache for groups of sequences that share their first pages: the shared pages meet the rows of the whole group
// at once, every sequence's rows its own pages behind them, and a row's partial results are joined.
#include "block.h"

namespace adac {

namespace {

struct PrefixShape {
  int TR;                          // rows of a tile of a group: 16 or 32 (block_attn), 64 or 128 (block_attn_wide)
  bool wide;
  int tiles, nsplit;               // of all groups at most; workgroups that share a group's pages
  BlockDims tail;                  // blocks of queries of a sequence
  int R, rts, tsplit;
  long long items;                 // of the tails
  size_t rows, trows;              // of partial results
};

PrefixShape shape_of(int dtype, int bits, const BlockAttnArgs& a) {
  const BlockDims& m = a.m;
  PrefixShape s;
  const long long most = (long long)m.B * m.max_q, queries = m.q_rows < most ? m.q_rows : most;
  const long long rows = (queries * m.G + a.gr.groups - 1) / (a.gr.groups > 0 ? a.gr.groups : 1);      // of a group, on average
  s.wide = dtype == ADACLUSTER_BF16 && rows > 32 && (bits || (a.ks.token < (1 << 25) && a.vs.token < (1 << 25)));
  s.TR = s.wide ? (rows <= 64 && bits ? 64 : 128) : rows <= 16 ? 16 : 32;
  s.tiles = a.gr.groups ? (int)((long long)m.q_rows * m.G / s.TR) + a.gr.groups : 0;
  // Few tiles: the pages are split among the workgroups that the GPU holds at a time.
  const long long busy = (rows + s.TR - 1) / s.TR * a.gr.groups * m.Hkv, keys = (long long)m.max_pages << m.lpage;
  const auto share = [&](long long items, int places, int tile) {
    const int least = share_keys(tile);
    long long n = items > 0 ? places / items : 1;
    if (n > (keys + least - 1) / least) n = (keys + least - 1) / least;
    return (int)(n < 1 ? 1 : n);
  };
  s.nsplit = share(busy, s.wide ? (bits ? 512 : 768) : s.TR == 16 ? 512 : 256, s.TR);
  s.tail = m;
  const int r = m.qblock * m.G;
  s.R = r <= 16 ? 1 : 2;
  s.rts = (r + 16 * s.R - 1) / (16 * s.R);
  s.items = (long long)s.rts * m.nb * m.Hkv * m.B;
  s.tsplit = share(s.items, s.R == 1 ? 512 : 256, 16 * s.R);
  s.rows = (size_t)s.tiles * m.Hkv * s.nsplit * s.TR;
  s.trows = (size_t)s.items * s.tsplit * 16 * s.R;
  return s;
}

// Joins a row's partial results: those of the pages its group shares, then those of its own.  D / 4 lanes read a result; `per` such
// slots share a row's results, each every per-th with a running maximum, and are joined through LDS.
template <typename T, int D>
__global__ __launch_bounds__(256) void prefix_join(BlockAttnArgs a, int rts, int R, int TR, int nsplit, int per, const float* __restrict__ shared_o,
                                                   const float* __restrict__ shared_ml) {
  constexpr int LPR = D / 4, SLOTS = 256 / LPR;
  __shared__ __align__(16) float jo[SLOTS][D];
  __shared__ float jm[SLOTS][2];
  const BlockDims& m = a.m;
  const int slot = threadIdx.x / LPR, d0 = threadIdx.x % LPR * 4, part = slot % per;
  long long id = (long long)blockIdx.x * (SLOTS / per) + slot / per;
  const int head = (int)(id % m.Hq); id /= m.Hq;
  const int i = (int)(id % m.max_q), b = (int)min(id / m.max_q, (long long)m.B - 1), hk = head / m.G;
  const BlockSeq s = block_seq(m, b);
  const bool there = id / m.max_q < m.B && i < s.nq;
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
      const int x = (t - group.q0) * m.G + head % m.G;
      rec = ((long long)(first_tile(m, group.q0, g, TR) + x / TR) * m.Hkv + hk) * nsplit * TR + x % TR;
      parts = group.pages && t >= group.q0 && t < group.q1 ? splits_of(m, group.pages, nsplit, TR) : 0;      // (else rows do not ascend)
    }
    own = splits_of(m, ((s.n + m.page - 1) >> m.lpage) - group.pages, a.nsplit, 16 * R);
    const int blk = i / m.qblock, row = (i - blk * m.qblock) * m.G + head % m.G, rt = row / (16 * R);
    trec = (((((long long)b * m.Hkv + hk) * m.nb + blk) * rts + rt) * a.nsplit) * (16 * R) + row % (16 * R);
  }
  const auto at = [&](int z, const float*& ml) __attribute__((always_inline)) {
    const bool sh = z < parts;
    const long long x = sh ? rec + (long long)z * TR : trec + (long long)(z - parts) * 16 * R;
    ml = (sh ? shared_ml : a.part_ml) + x * 2;
    return (sh ? shared_o : a.part_o) + x * D + d0;
  };
  float top = -INFINITY, all = 0.f;
  f32x4_t o{0.f, 0.f, 0.f, 0.f};
  const int count = parts + own;
  for (int z0 = part; z0 < count; z0 += 4 * per) {
    float mx[4], sum[4];
    f32x4_t v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int z = z0 + u * per;
      mx[u] = -INFINITY; sum[u] = 0.f; v[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if (z < count) { const float* ml; v[u] = *(const f32x4_t*)at(z, ml); mx[u] = ml[0]; sum[u] = ml[1]; }
    }
    const float next = fmaxf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), top);      // (finite: a result's reference is)
    const float f0 = __builtin_amdgcn_exp2f(top - next);
    all *= f0; o *= f0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float f = __builtin_amdgcn_exp2f(mx[u] - next);
      all = fmaf(f, sum[u], all);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = fmaf(f, v[u][j], o[j]);
    }
    top = next;
  }
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

}  // namespace

size_t prefix_attn_bytes(int dtype, int bits, int d, const BlockAttnArgs& a) {
  const PrefixShape s = shape_of(dtype, bits, a);
  return align_up(s.rows * d * 4, 256) + align_up(s.rows * 8, 256) + align_up(s.trows * d * 4, 256) + align_up(s.trows * 8, 256);
}

int launch_prefix_attn(hipStream_t st, int dtype, int bits, int d, BlockAttnArgs a, void* ws) {
  const PrefixShape s = shape_of(dtype, bits, a);
  if (!grid_fits((long long)s.tiles * a.m.Hkv * s.nsplit) || !grid_fits(s.items * (s.tsplit > s.R ? s.tsplit : s.R))) return ADACLUSTER_E_UNSUPPORTED;
  char* p = (char*)ws;
  const auto take = [&](size_t n) { char* const x = p; p += align_up(n, 256); return (float*)x; };
  float* const so = take(s.rows * d * 4);
  float* const sml = take(s.rows * 8);
  if (s.tiles) {
    BlockAttnArgs x = a;
    x.nsplit = s.nsplit; x.part_o = so; x.part_ml = sml;
    if (s.wide) launch_block_attn_wide_part(st, bits, d, s.TR, s.tiles, x);
    else launch_block_attn_part(st, dtype, bits, d, Rows::GROUP, s.TR / 16, 1, (long long)s.tiles * a.m.Hkv, x);
    if (int rc = launched()) return rc;
  }
  a.nsplit = s.tsplit;
  a.part_o = take(s.trows * d * 4);
  a.part_ml = take(s.trows * 8);
  launch_block_attn_part(st, dtype, bits, d, Rows::TAIL, s.R, s.rts, s.items, a);
  if (int rc = launched()) return rc;
  // up to eight results a slot, and two workgroups a CU
  const int slots = 1024 / d;
  const long long rows = (long long)a.m.B * a.m.max_q * a.m.Hq;
  int per = 1;
  while (per < slots && (per * 8 < s.nsplit + s.tsplit || rows * per < 512 * slots)) per *= 2;
  const long long wg = (rows * per + slots - 1) / slots;
  if (!grid_fits(wg)) return ADACLUSTER_E_UNSUPPORTED;
#define JOIN(T, D) prefix_join<T, D><<<(int)wg, 256, 0, st>>>(a, s.rts, s.R, s.TR, s.nsplit, per, so, sml)
  if (dtype == ADACLUSTER_BF16) { if (d == 64) JOIN(bf16raw, 64); else JOIN(bf16raw, 128); }
  else { if (d == 64) JOIN(float, 64); else JOIN(float, 128); }
#undef JOIN
  return launched();
}

}  // namespace adac
