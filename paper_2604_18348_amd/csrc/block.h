// Attention over pages of keys: what its kernels share (internal).
//
// A workgroup's unit is a block of queries: `qblock` consecutive queries of a sequence, of all the query heads that share
// one head of keys.  Its rows are counted token by token, the heads of the group inside a token, so that the causal limit
// never falls from one row to the next.
//
// All products run on 16x16 matrix-core tiles (v_mfma_f32_16x16x32_bf16, v_mfma_f32_16x16x4_f32): lane l holds row l % 16 of
// an operand and, of every run of the inner dimension, the 16 bytes that belong to quarter l / 16; of a result it holds
// column l % 16 and the rows 4 (l / 16) .. + 3.  Scores are formed as S^T = K Q^T, so that a lane holds one query and four
// keys of a tile, and what it holds of P^T is what the product O^T = V^T P^T wants from it: P never leaves the registers.
// That product's other operand, columns of V, comes out of LDS (transposing reads in 16 bits, plain ones in 32).
#pragma once

#include "common.h"

namespace adac {

typedef __attribute__((__vector_size__(4 * sizeof(uint32_t)))) uint32_t u32x4_t;

// What all kernels need of the parameters and the batch.
struct BlockDims {
  int B, Hq, Hkv, G;               // G: query heads of a head of keys
  int page, lpage;                 // tokens of a page, and their log2
  int num_pages;                   // of the pool; 0: packed keys
  int max_pages, max_q, qblock, nb;      // nb: blocks of queries a sequence at most
  int causal, topk, keep_first;
  int q_rows, k_rows;
  const int32_t *cu_q, *cu_k, *seq_lens, *table;
};

// Every figure that comes from device memory is held to the buffers it points into.
struct BlockSeq {
  int q0, nq;          // first query row, queries
  int k0, n;           // first key row (packed), keys
  int first;           // position of query 0: the last query is the last key
};
__device__ __forceinline__ BlockSeq block_seq(const BlockDims& m, int b) {
  BlockSeq s;
  s.q0 = min(max(m.cu_q[b], 0), m.q_rows);
  s.nq = min(max(m.cu_q[b + 1], s.q0), m.q_rows) - s.q0;
  const int most = m.max_pages << m.lpage;
  if (m.num_pages) {
    s.k0 = 0;
    s.n = min(max(m.seq_lens[b], 0), most);
  } else {
    s.k0 = min(max(m.cu_k[b], 0), m.k_rows);
    s.n = min(min(max(m.cu_k[b + 1], s.k0), m.k_rows) - s.k0, most);
  }
  s.first = s.n - s.nq;
  s.nq = min(s.nq, m.max_q);
  return s;
}

// Page of the pool that holds page pg of sequence b, or -1 (a table entry that names none).
__device__ __forceinline__ int pool_page(const BlockDims& m, int b, int pg) {
  const int t = m.table[(size_t)b * m.max_pages + pg];
  return (unsigned)t < (unsigned)m.num_pages ? t : -1;
}

// Groups of sequences that share their first pages (prefix_part.h); groups 0: none.  slots: 0, or how many places every sequence has among its
// group's queries (Group).
struct BlockGroups { int groups, slots; const int32_t *cu_group, *prefix; };

// Entry e of a list of pages (NULL: all pages in order), or -1: past the pages, or not above the entry before it.
__device__ __forceinline__ int list_page(const int32_t* __restrict__ list, int e, int pages) {
  if (!list) return e < pages ? e : -1;
  const int v = list[e], before = e > 0 ? list[e - 1] : -1;
  return v >= 0 && v > before && v < pages ? v : -1;
}

// a value that all lanes share, where the compiler keeps it in a vector register (divisions are made there)
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t v = (uint64_t)p;
  return (const char*)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}

// Entries e0, e0 + every, .. below e1 of a list, LIST at most, that name keys of pages below `pages`, in order: {page, place in the
// pool}.  Returns how many.  A list is looked up once by all threads, so that no load of a key waits for an entry and its page.
constexpr int LIST = 512;
template <int NT>
__device__ __forceinline__ int fill_list(const BlockDims& m, int b, const int32_t* list, int e0, int every, int e1, int pages, int2* out, int32_t* counts) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int n = 0;
  const int end = (int)min((long long)e1, e0 + (long long)every * LIST);
  for (int base = e0; base < end; base += NT * every) {
    const int e = base + tid * every;
    int pg = e < end ? list_page(list, e, pages) : -1, phys = 0;
    if (pg >= 0 && m.num_pages) { phys = pool_page(m, b, pg); if (phys < 0) pg = -1; }
    const uint64_t some = __ballot(pg >= 0);
    if (lane == 0) counts[wave] = __popcll(some);
    __syncthreads();
    int at = n + __popcll(some & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) { if (w < wave) at += counts[w]; n += counts[w]; }
    if (pg >= 0) out[at] = int2{pg, phys};
    __syncthreads();
  }
  return __builtin_amdgcn_readfirstlane(n);
}

// Where the 16 keys of a sixteenth `sub` of page pg start, in elements from the tensor's base: keys of one head.
struct KeyStride { long long page, token, head; };
__device__ __forceinline__ long long row_at(const BlockDims& m, const BlockSeq& s, const KeyStride& st, int phys, int pg, int sub, int hk) {
  return m.num_pages ? phys * st.page + (sub * 16) * st.token + hk * st.head
                     : (s.k0 + (long long)(pg << m.lpage) + sub * 16) * st.token + hk * st.head;
}

template <typename T> struct Vec { static constexpr int N = 16 / sizeof(T); };      // elements of 16 bytes

// 16-byte pieces of a row of D elements in LDS: piece u of row r lies in slot u ^ swz(r).  The 16 rows of a tile then lie in
// 16 different slots (writes), and the transposing reads (4 rows x 32 bytes a quarter wave) meet no bank twice.
template <typename T, int D> __device__ __forceinline__ int lds_piece(int r, int u) {
  constexpr int UPR = D * (int)sizeof(T) / 16;
  return (r * UPR + (UPR >= 16 ? u ^ (r & 15) : u ^ ((r >> 1) & 7))) * 16;
}

typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4_tr;
typedef __attribute__((address_space(3))) s16x4_tr lds_tr_t;

// acc += A B over one 16-byte piece of the inner dimension.  fp32 takes four products of four: both operands hold the same
// dimension in the same element, whatever their order.
__device__ __forceinline__ f32x4_t mma(bf16raw, const u32x4_t& a, const u32x4_t& b, f32x4_t acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8_t*)&a, *(const bf16x8_t*)&b, acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mma(float, const u32x4_t& a, const u32x4_t& b, f32x4_t acc) {
  const f32x4_t x = *(const f32x4_t*)&a, y = *(const f32x4_t*)&b;
#pragma unroll
  for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], acc, 0, 0, 0);
  return acc;
}

// acc[16 columns of X from d0][.] += X^T W over 32 rows of X in LDS (row-major, lds_piece); w0, w1: what the lane holds of W's
// rows 4 quarter .. + 3 of either half, as a result tile leaves it.
template <int D>
__device__ __forceinline__ bf16x8_t read_cols(const char* lds, int d0, int lane) {
  const int r = 4 * (lane >> 4) + ((lane >> 2) & 3), u = d0 / 8 + ((lane >> 1) & 1), in = (lane & 1) * 8;
  const s16x4_tr lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_t*)(lds + lds_piece<bf16raw, D>(r, u) + in));
  const s16x4_tr hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr_t*)(lds + lds_piece<bf16raw, D>(r + 16, u) + in));
  union { struct { s16x4_tr lo, hi; } s; bf16x8_t v; } a{{lo, hi}};
  return a.v;
}
template <int D>
__device__ __forceinline__ f32x4_t mma_cols(const char* lds, int d0, int lane, const bf16x8_t& w, f32x4_t acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(read_cols<D>(lds, d0, lane), w, acc, 0, 0, 0);
}
// ... with W in two parts, of which the columns of X are read once
template <int D>
__device__ __forceinline__ f32x4_t mma_cols(const char* lds, int d0, int lane, const bf16x8_t& w, const bf16x8_t& rest, f32x4_t acc) {
  const bf16x8_t a = read_cols<D>(lds, d0, lane);
  acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, rest, acc, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, w, acc, 0, 0, 0);
}
template <int D>
__device__ __forceinline__ f32x4_t mma_cols(bf16raw, const char* lds, int d0, int lane, const f32x4_t& w0, const f32x4_t& w1, f32x4_t acc) {
  union { uint32_t w[4]; bf16x8_t v; } b{{pack_bf16x2(w0[0], w0[1]), pack_bf16x2(w0[2], w0[3]), pack_bf16x2(w1[0], w1[1]), pack_bf16x2(w1[2], w1[3])}};
  return mma_cols<D>(lds, d0, lane, b.v, acc);
}
template <int D>
__device__ __forceinline__ f32x4_t mma_cols(float, const char* lds, int d0, int lane, const f32x4_t& w0, const f32x4_t& w1, f32x4_t acc) {
  const int r = 4 * (lane >> 4), u = d0 / 4 + ((lane >> 2) & 3), in = (lane & 3) * 4;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(*(const float*)(lds + lds_piece<float, D>(16 * h + r + i, u) + in), h ? w1[i] : w0[i], acc, 0, 0, 0);
  return acc;
}

// The lane's pieces of 16 rows: row lane % 16, piece 4 f + lane / 16 of it.
template <typename T, int D> struct RowFrag { u32x4_t p[D * sizeof(T) / 64]; };
// The 16 x 16 products of two tiles' rows.  128 dimensions in 32 bits are two sums: a single chain of them is off by twice as much (fp32
// attention against 64 bits 1.9e-6, with two 1.0e-6 at 0.1 to 0.8 % more time, with four 0.65e-6 at up to 5 %; a product library
// 0.7e-6 to 1.9e-6).  The gradients form their scores the same way: weights then agree with the row's sum to the last bits.
template <typename T, int D>
__device__ __forceinline__ f32x4_t dots(const RowFrag<T, D>& a, const RowFrag<T, D>& b) {
  constexpr int NF = D * sizeof(T) / 64;
  constexpr bool TWO = sizeof(T) == 4 && D == 128;
  const f32x4_t zero{0.f, 0.f, 0.f, 0.f};
  f32x4_t sum = zero, other = zero;
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    f32x4_t& s = TWO && f % 2 ? other : sum;
    s = mma(T{}, a.p[f], b.p[f], s);
  }
  return TWO ? sum + other : sum;
}
template <typename T, int D>
__device__ __forceinline__ void load_frag(RowFrag<T, D>& f, const T* row, int quarter, bool there) {
#pragma unroll
  for (int x = 0; x < (int)(D * sizeof(T) / 64); ++x)
    f.p[x] = there ? *(const u32x4_t*)(row + (4 * x + quarter) * Vec<T>::N) : u32x4_t{0, 0, 0, 0};
}
template <typename T, int D>
__device__ __forceinline__ void store_frag(char* lds, int row, int quarter, const RowFrag<T, D>& f) {
#pragma unroll
  for (int x = 0; x < (int)(D * sizeof(T) / 64); ++x) *(u32x4_t*)(lds + lds_piece<T, D>(row, 4 * x + quarter)) = f.p[x];
}

// What the rounding of x, y to `packed` (pack_bf16x2) leaves of them, rounded: up to 2^-8 of a value, off by up to 2^-16 of it.
__device__ __forceinline__ uint32_t rounding_rest(float x, float y, uint32_t packed) {
  return pack_bf16x2(x - __uint_as_float(packed << 16), y - __uint_as_float(packed & 0xFFFF0000u));
}

__device__ __forceinline__ void compiler_fence() { asm volatile("" ::: "memory"); }

__device__ __forceinline__ float quarters_sum(float v) { v += __shfl_xor(v, 16); return v + __shfl_xor(v, 32); }
__device__ __forceinline__ float quarters_max(float v) { v = fmaxf(v, __shfl_xor(v, 16)); return fmaxf(v, __shfl_xor(v, 32)); }

// 16-byte stores of N floats as T
template <typename T> __device__ __forceinline__ void store_vec(T* p, const float* v);
template <> __device__ __forceinline__ void store_vec<float>(float* p, const float* v) { *(f32x4_t*)p = f32x4_t{v[0], v[1], v[2], v[3]}; }
template <> __device__ __forceinline__ void store_vec<bf16raw>(bf16raw* p, const float* v) {
  *(u32x4_t*)p = u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// ---- launches (block_cache.hip, block_attn.hip, block_grad.hip): 0 or an ADACLUSTER_E_* code ----
struct CacheArgs {
  BlockDims m;                               // cu_q: rows of the new tokens; seq_lens: tokens held before
  const void *k, *v;                         // new rows (append)
  void *ko, *vo;                             // values read (read)
  KeyStride new_k, new_v;                    // (page 0)
  void *kp, *vp, *boxes;                     // the pool
  uint32_t *km, *vm;                         // 4 bits: (scale, lo) pairs
  KeyStride ks, vs;
};
int launch_cache_append(hipStream_t s, int dtype, int bits, int d, const CacheArgs& a);
int launch_cache_read(hipStream_t s, int dtype, int bits, int d, const CacheArgs& a);
int launch_block_boxes(hipStream_t s, int dtype, int d, const BlockDims& m, const void* k, KeyStride ks, void* boxes);
size_t block_select_bytes(const BlockDims& m, int dtype);
int launch_block_select(hipStream_t s, int dtype, int d, const BlockDims& m, const void* q, KeyStride qs, const void* boxes,
                        int32_t* sel_idx, int32_t* sel_cnt, void* ws);

struct BlockAttnArgs {
  BlockDims m;
  const void *q, *k, *v;
  const uint32_t *km, *vm;
  const int32_t* sel;
  void* o;
  float* lse;                                // NULL: not wanted
  KeyStride qs, os, ks, vs;
  float scale_log2e;
  int nsplit;
  float *part_o, *part_ml;                   // [item][split][rows][d], [item][split][rows][2]
};
size_t block_attn_bytes(const BlockDims& m, int d, bool listed);
int launch_block_attn(hipStream_t s, int dtype, int bits, int d, BlockAttnArgs a, void* ws);
bool block_wide_takes(const BlockAttnArgs& a, int dtype, int bits);      // (block_wide.hip)
int launch_block_attn_wide(hipStream_t s, int d, const BlockAttnArgs& a);

// (block_prefix.hip)
// Two kinds of partial results, [item][share][rows][d] and [item][share][rows][2]: of tiles of a group's rows over the pages it shares, and of a
// sequence's rows over its pages behind them.
struct PrefixArgs : BlockAttnArgs {
  BlockGroups gr;
  int grid, split;                           // workgroups of the former, which come first, and their division among the XCDs
  int tiles, TR, shares;                     // tiles of all groups at most, rows of a tile, workgroups that share a group's pages at most
  int rts, TT, tshares;                      // of the latter: tiles of a block of queries, their rows, shares
  int gkeys, tkeys;                          // keys of a share at least
  float *group_o, *group_ml, *tail_o, *tail_ml;
};
size_t prefix_attn_bytes(int dtype, int bits, int d, const PrefixArgs& a);
int launch_prefix_attn(hipStream_t s, int dtype, int bits, int d, PrefixArgs a, void* ws);

// (block_weights.hip)
struct WeightsArgs {
  BlockDims m;
  const void *q, *k;
  const uint32_t* km;
  const float *lse, *w;                      // w: what was there (NULL: nothing)
  float* out;                                // [B][Hkv][max_pages * page]
  KeyStride qs, ks;
  float scale_log2e, decay;
  const u32x4_t* sums;                       // 4 bits: two records a row and head (weights_sums)
  float* part;                               // [nsplit] like out: sums over a share of the rows
  int nsplit;
};
size_t cache_weights_bytes(int dtype, int bits, int d, const BlockDims& m, const KeyStride& qs);
int launch_cache_weights(hipStream_t s, int dtype, int bits, int d, WeightsArgs a, void* ws);
// (block_evict.hip)
struct EvictArgs {
  BlockDims m;
  const float* w;
  const int32_t* new_table;
  int keep, recent;
  int32_t *kept, *new_lens;
  float* new_w;
  void *kp, *vp, *boxes;
  uint32_t *km, *vm;
  KeyStride ks, vs;
};
int launch_cache_evict(hipStream_t s, int dtype, int bits, int d, const EvictArgs& a);

struct BlockGradArgs {
  BlockDims m;
  const void *q, *k, *v, *o, *d_o;
  const float* lse;
  const int32_t* sel;
  void *dq, *dk, *dv;
  KeyStride qs, ks, vs, os, dos, dqs, dks, dvs;
  float scale, scale_log2e;
  float* delta;                              // [q_rows][Hq]
  uint32_t* marks;                           // [B][Hkv][max_pages][words]: blocks of queries that list a page
  int words;
  float* sums;                               // of pages that many blocks list, a share each: [group][np][..]
  int groups, wg, np, limit;
};
size_t block_grad_bytes(const BlockDims& m, int dtype, int d, bool listed);
int launch_block_attn_backward(hipStream_t s, int dtype, int d, BlockGradArgs a, void* ws);

// a launch of more workgroups than a grid may have threads for is refused before it is made
static inline bool grid_fits(long long workgroups) { return workgroups <= (1ll << 32) / 256 - 1; }

}  // namespace adac
