// Groups of sequences that share their first pages, and the parts that their attention is made of (internal).
#pragma once

#include "block.h"

namespace adac {

// Sequences [b0, b1) of group g, its queries [q0, q1), and the whole pages of what they share (of what the first one holds).  Queries are counted
// as their rows lie in the tensor; where that has more rows than the call can have queries, B * max_q, in places instead, max_q for every
// sequence: tiles and partial results are as many as either count may need.
struct Group { int b0, b1, q0, q1, pages; };
__device__ __forceinline__ Group group_at(const BlockDims& m, const BlockGroups& gr, int g) {
  Group x{0, 0, 0, 0, 0};
  x.b0 = min(max(gr.cu_group[g], 0), m.B);
  x.b1 = min(max(gr.cu_group[g + 1], x.b0), m.B);
  if (gr.slots) {
    x.q0 = x.b0 * gr.slots;
    x.q1 = x.b1 * gr.slots;
  } else {
    x.q0 = min(max(m.cu_q[x.b0], 0), m.q_rows);
    x.q1 = min(max(m.cu_q[x.b1], x.q0), m.q_rows);
  }
  if (x.b0 < x.b1) x.pages = min(max(gr.prefix[g], 0), min(max(m.seq_lens[x.b0], 0), m.max_pages << m.lpage)) >> m.lpage;
  return x;
}
// The last of the groups for which `at_most` holds, or -1: by whole waves, of a condition that holds for the first ones.
template <typename F> __device__ __forceinline__ int last_group(int groups, F at_most) {
  int n = 0;
  for (int g0 = 0; g0 < groups; g0 += 64) {
    const int g = g0 + (threadIdx.x & 63);
    n += __popcll(__ballot(g < groups && at_most(min(g, groups - 1))));
  }
  return n - 1;
}
// The group of sequence b, or -1.
__device__ __forceinline__ int group_of(const BlockGroups& gr, int b) {
  const int g = last_group(gr.groups, [&](int x) { return gr.cu_group[x] <= b; });
  return g >= 0 && b < gr.cu_group[g + 1] ? g : -1;
}
// Tiles of TR rows (a query of a head each) start anew at every group: the first tile of a group whose queries start at q0.  Groups
// that follow each other have different ones, and all lie below min(q_rows, B * max_q) * G / TR + groups.
__device__ __forceinline__ int first_tile(const BlockDims& m, int q0, int g, int TR) { return q0 * m.G / TR + g; }

// Query x of the group, counted as above: its row in the tensor, and the key below which it sees, or -1 (a row of no sequence).
struct QueryRow { int t, lim; };
__device__ __forceinline__ QueryRow group_query(const BlockDims& m, const BlockGroups& gr, const Group& g, int x) {
  int b, t;
  BlockSeq s;
  if (gr.slots) {
    b = min(x / gr.slots, m.B - 1);
    s = block_seq(m, b);
    t = s.q0 + x % gr.slots;
  } else {
    t = x;
    b = g.b0 + (t - g.q0);                             // (one query a sequence)
    if (m.max_q > 1 || b >= g.b1 || m.cu_q[b] > t || m.cu_q[b + 1] <= t) {
      int lo = g.b0, hi = g.b1;                        // cu_q[lo] <= t < cu_q[hi]
      while (hi - lo > 1) { const int mid = (lo + hi) >> 1; if (m.cu_q[mid] <= t) lo = mid; else hi = mid; }
      b = lo;
    }
    s = block_seq(m, b);
  }
  const int i = t - s.q0;
  if (i < 0 || i >= s.nq) return {0, -1};
  return {t, m.causal ? max(0, min(s.n, s.first + i + 1)) : s.n};
}
// How many of `nsplit` workgroups share `pages` pages, `keys` keys each at least.
__device__ __forceinline__ int splits_of(const BlockDims& m, int pages, int nsplit, int keys) {
  return min(nsplit, max(1, ((pages << m.lpage) + keys - 1) / keys));
}

// What a workgroup walks: rows of a group over a share of the pages that it shares, or rows of a block of queries of a sequence over a
// share of the pages behind them.
struct Part {
  BlockSeq s;                      // shared: the group's queries, as Group counts them, and as keys the pages that it shares
  Group group;
  int hk, b, t0, rows, base_row;   // rows from base_row on below `rows`; row r is query t0 + r / G
  int from, to;                    // pages
  bool shared;
  long long rec;                   // its first partial result, in rows
  float *o, *ml;
};
__device__ __forceinline__ bool part_of(const PrefixArgs& a, int id, Part& p) {
  const BlockDims& m = a.m;
  p.shared = id < a.grid;
  int pages, shares, share;
  if (p.shared) {
                                   // a share of the keys is walked by all tiles side by side
    const int per = (a.tiles * a.shares + a.split - 1) / a.split, unit = (id & 7) + 8 * ((id >> 3) / per), item = (id >> 3) % per * a.split + unit % a.split;
    if (item >= a.tiles * a.shares) return false;
    const int tile = uniform(item % a.tiles);
    share = uniform(item / a.tiles);
    p.hk = uniform(unit / a.split);
    const int g = a.gr.groups == 1 ? 0 : last_group(a.gr.groups, [&](int x) { return first_tile(m, group_at(m, a.gr, x).q0, x, a.TR) <= tile; });
    if (g < 0) return false;
    p.group = group_at(m, a.gr, g);
    p.b = p.group.b0;
    p.t0 = 0;
    p.base_row = (tile - first_tile(m, p.group.q0, g, a.TR)) * a.TR;      // (below 0: groups that do not ascend)
    p.rows = (p.group.q1 - p.group.q0) * m.G;
    p.from = 0; p.to = pages = p.group.pages;
    p.s = BlockSeq{p.group.q0, p.group.q1 - p.group.q0, 0, pages << m.lpage, 0};
    shares = splits_of(m, pages, a.shares, a.gkeys);
    p.rec = (((long long)tile * m.Hkv + p.hk) * a.shares + share) * a.TR;
    p.o = a.group_o; p.ml = a.group_ml;
  } else {
    id -= a.grid;
    const int item = uniform(id / a.tshares);
    share = uniform(id % a.tshares);
    id = item;
    const int rt = uniform(id % a.rts); id = uniform(id / a.rts);
    const int i = uniform(id % m.nb); id = uniform(id / m.nb);
    p.hk = uniform(id % m.Hkv); p.b = uniform(id / m.Hkv);
    p.s = block_seq(m, p.b);
    p.t0 = i * m.qblock;
    p.rows = min(m.qblock, p.s.nq - p.t0) * m.G;
    p.base_row = p.t0 < p.s.nq ? rt * a.TT : p.rows;
    const int g = group_of(a.gr, p.b);
    p.from = g >= 0 ? group_at(m, a.gr, g).pages : 0;
    const int last = min(p.base_row + a.TT, p.rows) - 1, lim = m.causal ? min(p.s.n, p.s.first + p.t0 + last / m.G + 1) : p.s.n;      // (no row sees further)
    p.to = lim > 0 ? (lim + m.page - 1) >> m.lpage : 0;
    pages = ((p.s.n + m.page - 1) >> m.lpage) - p.from;
    shares = splits_of(m, pages, a.tshares, a.tkeys);
    p.rec = ((long long)item * a.tshares + share) * a.TT;
    p.o = a.tail_o; p.ml = a.tail_ml;
  }
  if (p.base_row < 0 || p.base_row >= p.rows || share >= shares) return false;
  const int n = max(0, p.to - p.from), first = p.from;
  p.from = uniform(first + (int)((long long)n * share / shares));
  p.to = uniform(first + (int)((long long)n * (share + 1) / shares));
  return true;
}
// Its query x, from the first of p.s: the row in the tensor, and the key below which it sees, or -1 (no such row).
__device__ __forceinline__ QueryRow part_query(const PrefixArgs& a, const Part& p, int x) {
  const BlockDims& m = a.m;
  if (p.shared) return group_query(m, a.gr, p.group, p.s.q0 + x);
  return {p.s.q0 + x, max(0, m.causal ? min(p.s.n, p.s.first + x + 1) : p.s.n)};
}

}  // namespace adac
