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
  s.wide = dtype == ADACLUSTER_BF16 && !bits && rows > 32 && a.ks.token < (1 << 25) && a.vs.token < (1 << 25);
  s.TR = s.wide ? (rows <= 64 ? 64 : 128) : rows <= 16 ? 16 : 32;
  s.tiles = a.gr.groups ? (int)((long long)m.q_rows * m.G / s.TR) + a.gr.groups : 0;
  // Few tiles: the pages are split until the launch has four workgroups a CU, 256 keys each at least.
  const long long busy = (rows + s.TR - 1) / s.TR * a.gr.groups * m.Hkv, keys = (long long)m.max_pages << m.lpage;
  const auto share = [&](long long items) {
    long long n = items > 0 ? (1024 + items - 1) / items : 1;
    if (n > (keys + 255) / 256) n = (keys + 255) / 256;
    return (int)n;
  };
  s.nsplit = share(busy);
  s.tail = m;
  const int r = m.qblock * m.G;
  s.R = r <= 16 ? 1 : 2;
  s.rts = (r + 16 * s.R - 1) / (16 * s.R);
  s.items = (long long)s.rts * m.nb * m.Hkv * m.B;
  s.tsplit = share(s.items);
  s.rows = (size_t)s.tiles * m.Hkv * s.nsplit * s.TR;
  s.trows = (size_t)s.items * s.tsplit * 16 * s.R;
  return s;
}

// A wave's 16 lanes a row: the partial results of the pages its group shares, then those of its own.
template <typename T, int D>
__global__ __launch_bounds__(256) void prefix_join(BlockAttnArgs a, int rts, int R, int TR, int nsplit, const float* __restrict__ shared_o, const float* __restrict__ shared_ml) {
  const BlockDims& m = a.m;
  const int item = blockIdx.x / R, r = blockIdx.x % R;
  int id = item;
  const int rt = id % rts; id /= rts;
  const int i = id % m.nb; id /= m.nb;
  const int hk = id % m.Hkv, b = id / m.Hkv;
  const BlockSeq s = block_seq(m, b);
  const int g = group_of(a.gr, b);
  const int t0 = i * m.qblock, rows = min(m.qblock, s.nq - t0) * m.G;
  const int jr = threadIdx.x >> 4, row = (rt * R + r) * 16 + jr, d0 = (threadIdx.x & 15) * (D / 16);
  if (t0 >= s.nq || row >= rows) return;
  const int t = t0 + row / m.G;
  Group group{0, 0, 0, 0, 0};
  int parts = 0;
  long long rec = 0;
  if (g >= 0) {
    group = group_at(m, a.gr, g);
    const int x = (s.q0 + t - group.q0) * m.G + row % m.G;
    rec = ((long long)(first_tile(m, group.q0, g, TR) + x / TR) * m.Hkv + hk) * nsplit * TR + x % TR;
    parts = group.pages && s.q0 >= group.q0 && s.q0 + t < group.q1 ? splits_of(m, group.pages, nsplit) : 0;      // (else rows do not ascend)
  }
  const int own = splits_of(m, ((s.n + m.page - 1) >> m.lpage) - group.pages, a.nsplit);
  const long long trec = (long long)item * a.nsplit * (16 * R) + r * 16 + jr;
  float top = -INFINITY, all = 0.f, o[D / 16];
  for (int z = 0; z < parts; ++z) top = fmaxf(top, shared_ml[(rec + (long long)z * TR) * 2]);
  for (int z = 0; z < own; ++z) top = fmaxf(top, a.part_ml[(trec + (long long)z * 16 * R) * 2]);
  const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int x = 0; x < D / 16; ++x) o[x] = 0.f;
  const auto add = [&](const float* po, const float* pml, long long at) __attribute__((always_inline)) {
    const float f = __builtin_amdgcn_exp2f(pml[at * 2] - ref);
    all += f * pml[at * 2 + 1];
#pragma unroll
    for (int x = 0; x < D / 16; x += 4) {
      const f32x4_t v = *(const f32x4_t*)(po + at * D + d0 + x);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[x + j] = fmaf(f, v[j], o[x + j]);
    }
  };
  for (int z = 0; z < parts; ++z) add(shared_o, shared_ml, rec + (long long)z * TR);
  for (int z = 0; z < own; ++z) add(a.part_o, a.part_ml, trec + (long long)z * 16 * R);
  const int head = hk * m.G + row % m.G;
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
    if (s.wide) launch_block_attn_wide_part(st, d, s.TR, s.tiles, x);
    else launch_block_attn_part(st, dtype, bits, d, Rows::GROUP, s.TR / 16, 1, (long long)s.tiles * a.m.Hkv, x);
    if (int rc = launched()) return rc;
  }
  a.nsplit = s.tsplit;
  a.part_o = take(s.trows * d * 4);
  a.part_ml = take(s.trows * 8);
  launch_block_attn_part(st, dtype, bits, d, Rows::TAIL, s.R, s.rts, s.items, a);
  if (int rc = launched()) return rc;
  const int wg = (int)(s.items * s.R);
#define JOIN(T, D) prefix_join<T, D><<<wg, 256, 0, st>>>(a, s.rts, s.R, s.TR, s.nsplit, so, sml)
  if (dtype == ADACLUSTER_BF16) { if (d == 64) JOIN(bf16raw, 64); else JOIN(bf16raw, 128); }
  else { if (d == 64) JOIN(float, 64); else JOIN(float, 128); }
#undef JOIN
  return launched();
}

}  // namespace adac
