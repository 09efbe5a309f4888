// Pages of keys and values: new tokens written into them (in the inputs' type or in 4 bits) with the pages' boxes, tokens read
// back, boxes of packed keys, and the selection of pages for blocks of queries by the scores of their boxes (Eq. 1).
#include "block.h"

namespace adac {

namespace {

template <typename T> __device__ __forceinline__ void unpack16(const u32x4_t& w, float* v);
template <> __device__ __forceinline__ void unpack16<float>(const u32x4_t& w, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
}
template <> __device__ __forceinline__ void unpack16<bf16raw>(const u32x4_t& w, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}

// Bits of the bfloat16 next to x in the direction of minus infinity, and of plus infinity for x >= 0 (x finite; either may be infinite).
__device__ __forceinline__ uint32_t bf16_down(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u + ((u >> 31) && (u & 0xFFFF) ? 0x10000u : 0u)) >> 16;
}
__device__ __forceinline__ uint32_t bf16_up(float x) { return (__float_as_uint(x) + 0xFFFFu) >> 16; }
__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// 4 bits: 64 dimensions of a row share a step and a lowest value, both bfloat16, rounded so that the sixteen values
// lo + code * step span the group: lo down, the step (max - lo) * (1/15, as a float) up.  A value is then off by half a step at most.  A
// group that holds a NaN or an infinity, or whose span or step no float or bfloat16 holds, is kept as NaN.
// The lanes of a group are neighbours, VEC values each.
template <int VEC>
__device__ __forceinline__ uint32_t quantise(const float* v, uint32_t* pair) {
  float lo = v[0], hi = v[0];
  bool good = true;
#pragma unroll
  for (int i = 0; i < VEC; ++i) { lo = fminf(lo, v[i]); hi = fmaxf(hi, v[i]); good = good && finite(v[i]); }
  int ok = good;
#pragma unroll
  for (int x = 1; x < 64 / VEC; x <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, x)); hi = fmaxf(hi, __shfl_xor(hi, x));
    ok &= __shfl_xor(ok, x);
  }
  const uint32_t lob = bf16_down(lo);
  const float low = __uint_as_float(lob << 16), span = hi - low;
  const uint32_t stb = bf16_up(span * (1.0f / 15.0f));
  const float step = __uint_as_float(stb << 16);
  if (!(ok && finite(span) && finite(step))) { *pair = 0x7FC07FC0u; return 0; }
  *pair = lob << 16 | stb;
  uint32_t codes = 0;
  if (step > 0.f) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) codes |= (uint32_t)fminf(fmaxf(rintf((v[i] - low) / step), 0.f), 15.f) << (4 * i);
  }
  return codes;
}

// New tokens of one page of one head: memory-bound, 16 bytes a lane in and out.  A page belongs to one workgroup, so its box is
// the old one (where the page held tokens before) joined with the new keys' in a fixed order, without atomics.
template <typename T, int BITS, int D>
__global__ __launch_bounds__(256) void cache_append(CacheArgs a, int touched) {
  constexpr int VEC = Vec<T>::N, LPR = D / VEC, RPI = 256 / LPR;          // lanes a row, rows a turn
  const BlockDims& m = a.m;
  const int j = blockIdx.x % touched, hk = blockIdx.x / touched % m.Hkv, b = blockIdx.x / touched / m.Hkv;
  const int r0 = min(max(m.cu_q[b], 0), m.q_rows), nn = min(min(max(m.cu_q[b + 1], r0), m.q_rows) - r0, m.max_q);
  const int most = m.max_pages << m.lpage, old = min(max(m.seq_lens[b], 0), most), end = (int)min((long long)old + nn, (long long)most);
  const int pg = (old >> m.lpage) + j, p0 = max(old, pg << m.lpage), p1 = min(end, (pg + 1) << m.lpage);
  if (p0 >= p1) return;
  const int phys = pool_page(m, b, pg);
  if (phys < 0) return;
  const int tid = threadIdx.x, col = tid % LPR * VEC;
  float mx[VEC], mn[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) { mx[i] = -INFINITY; mn[i] = INFINITY; }
  for (int p = p0 + tid / LPR; p - tid / LPR < p1; p += RPI) {
    const bool there = p < p1;                                 // (whole groups of lanes quantise together)
    const long long row = r0 + (p - old);
    const int in = p & (m.page - 1);
    u32x4_t kw{0, 0, 0, 0}, vw{0, 0, 0, 0};
    if (there) {
      kw = *(const u32x4_t*)((const T*)a.k + row * a.new_k.token + hk * a.new_k.head + col);
      vw = *(const u32x4_t*)((const T*)a.v + row * a.new_v.token + hk * a.new_v.head + col);
    }
    float kv[VEC];
    unpack16<T>(kw, kv);
    if constexpr (BITS == 4) {
      float vv[VEC];
      unpack16<T>(vw, vv);
      uint32_t kp, vp;
      const uint32_t kc = quantise<VEC>(kv, &kp), vc = quantise<VEC>(vv, &vp);
      if (there) {
        const long long at = ((long long)phys * m.Hkv + hk) * m.page + in;
        if constexpr (VEC == 8) {
          ((uint32_t*)a.kp)[at * (D / 8) + col / 8] = kc;
          ((uint32_t*)a.vp)[at * (D / 8) + col / 8] = vc;
        } else {
          ((uint16_t*)a.kp)[at * (D / 4) + col / 4] = (uint16_t)kc;
          ((uint16_t*)a.vp)[at * (D / 4) + col / 4] = (uint16_t)vc;
        }
        if (col % 64 == 0) { a.km[at * (D / 64) + col / 64] = kp; a.vm[at * (D / 64) + col / 64] = vp; }
      }
    } else if (there) {
      *(u32x4_t*)((T*)a.kp + phys * a.ks.page + in * a.ks.token + hk * a.ks.head + col) = kw;
      *(u32x4_t*)((T*)a.vp + phys * a.vs.page + in * a.vs.token + hk * a.vs.head + col) = vw;
    }
    if (there) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) { mx[i] = fmaxf(mx[i], kv[i]); mn[i] = fminf(mn[i], kv[i]); }
    }
  }
  __shared__ float s_mx[256 * VEC], s_mn[256 * VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) { s_mx[tid * VEC + i] = mx[i]; s_mn[tid * VEC + i] = mn[i]; }
  __syncthreads();
  T* const box = (T*)a.boxes + ((long long)phys * m.Hkv + hk) * 2 * D;
  const bool joined = (pg << m.lpage) < old;
  for (int c = tid; c < D; c += 256) {
    float x = s_mx[c], y = s_mn[c];
    for (int r = 1; r < RPI; ++r) { x = fmaxf(x, s_mx[r * D + c]); y = fminf(y, s_mn[r * D + c]); }
    if (joined) { x = fmaxf(x, Elem<T>::load(box + c)); y = fminf(y, Elem<T>::load(box + D + c)); }
    if constexpr (sizeof(T) == 2) { box[c] = (T)(__float_as_uint(x) >> 16); box[D + c] = (T)(__float_as_uint(y) >> 16); }      // (bfloat16 values: exact)
    else { box[c] = x; box[D + c] = y; }
  }
}

// Tokens of the cache as values: a lane 16 bytes of the output.
template <typename T, int BITS, int D>
__global__ __launch_bounds__(256) void cache_read(CacheArgs a, int pieces) {
  constexpr int VEC = Vec<T>::N, LPR = D / VEC, RPI = 256 / LPR;
  const BlockDims& m = a.m;
  const int j = blockIdx.x % pieces, b = blockIdx.x / pieces;
  const int r0 = min(max(m.cu_q[b], 0), m.q_rows), nn = min(min(max(m.cu_q[b + 1], r0), m.q_rows) - r0, m.max_q);
  const int most = m.max_pages << m.lpage, old = min(max(m.seq_lens[b], 0), most), end = (int)min((long long)old + nn, (long long)most);
  const int x = j * RPI + threadIdx.x / LPR, hk = x % m.Hkv, t = x / m.Hkv, col = threadIdx.x % LPR * VEC;
  const int p = old + t;
  if (t >= nn || p >= end) return;
  const int phys = pool_page(m, b, p >> m.lpage), in = p & (m.page - 1);
  const long long to = ((long long)(r0 + t) * m.Hkv + hk) * D + col;
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    T* const out = (T*)(side ? a.vo : a.ko) + to;
    u32x4_t w{0, 0, 0, 0};
    if (phys >= 0) {
      if constexpr (BITS == 4) {
        const long long at = ((long long)phys * m.Hkv + hk) * m.page + in;
        const uint32_t pair = (side ? a.vm : a.km)[at * (D / 64) + col / 64];
        const uint32_t c = VEC == 8 ? ((const uint32_t*)(side ? a.vp : a.kp))[at * (D / 8) + col / 8] : ((const uint16_t*)(side ? a.vp : a.kp))[at * (D / 4) + col / 4];
        const float step = __uint_as_float(pair << 16), low = __uint_as_float(pair & 0xFFFF0000u);
        float v[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = fmaf((float)(c >> (4 * i) & 15), step, low);       // (the product is exact: one rounding)
        store_vec<T>(out, v);
        continue;
      } else {
        const KeyStride& st = side ? a.vs : a.ks;
        w = *(const u32x4_t*)((const T*)(side ? a.vp : a.kp) + phys * st.page + in * st.token + hk * st.head + col);
      }
    }
    *(u32x4_t*)out = w;
  }
}

// Boxes of packed keys: a workgroup a page and head, as in cache_append.
template <typename T, int D>
__global__ __launch_bounds__(256) void block_boxes(BlockDims m, const T* __restrict__ k, KeyStride ks, T* __restrict__ boxes) {
  constexpr int VEC = Vec<T>::N, LPR = D / VEC, RPI = 256 / LPR;
  const int pg = blockIdx.x % m.max_pages, hk = blockIdx.x / m.max_pages % m.Hkv, b = blockIdx.x / m.max_pages / m.Hkv;
  const int k0 = min(max(m.cu_k[b], 0), m.k_rows), n = min(max(m.cu_k[b + 1], k0), m.k_rows) - k0;
  const int p0 = pg << m.lpage, p1 = min(n, p0 + m.page);
  const int tid = threadIdx.x, col = tid % LPR * VEC;
  float mx[VEC], mn[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) { mx[i] = -INFINITY; mn[i] = INFINITY; }
  for (int p = p0 + tid / LPR; p < p1; p += RPI) {
    float v[VEC];
    unpack16<T>(*(const u32x4_t*)(k + (long long)(k0 + p) * ks.token + hk * ks.head + col), v);
#pragma unroll
    for (int i = 0; i < VEC; ++i) { mx[i] = fmaxf(mx[i], v[i]); mn[i] = fminf(mn[i], v[i]); }
  }
  __shared__ float s_mx[256 * VEC], s_mn[256 * VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) { s_mx[tid * VEC + i] = mx[i]; s_mn[tid * VEC + i] = mn[i]; }
  __syncthreads();
  T* const box = boxes + (((long long)b * m.max_pages + pg) * m.Hkv + hk) * 2 * D;
  for (int c = tid; c < D; c += 256) {
    float x = s_mx[c], y = s_mn[c];
    for (int r = 1; r < RPI; ++r) { x = fmaxf(x, s_mx[r * D + c]); y = fminf(y, s_mn[r * D + c]); }
    if (p0 >= p1) x = y = 0.f;                     // a page past the sequence
    if constexpr (sizeof(T) == 2) { box[c] = (T)(__float_as_uint(x) >> 16); box[D + c] = (T)(__float_as_uint(y) >> 16); }
    else { box[c] = x; box[D + c] = y; }
  }
}

// What a block of queries can list of a sequence: pages [0, seen), of which [lo, hi) hold its own positions.
struct Seen { int lo, hi, seen; };
__device__ __forceinline__ Seen block_seen(const BlockDims& m, const BlockSeq& s, int i) {
  const int t0 = i * m.qblock;
  if (t0 >= s.nq) return {0, 0, 0};
  if (!m.causal) return {0, 0, (s.n + m.page - 1) >> m.lpage};
  const int first = max(s.first + t0, 0), last = s.first + min(t0 + m.qblock, s.nq) - 1;
  if (last < 0) return {0, 0, 0};
  return {first >> m.lpage, (last >> m.lpage) + 1, (last >> m.lpage) + 1};
}

// Scores of a block of queries against the boxes of pages: S(h, p) = sum_d max(u_d max_pd, u_d min_pd), u the sum of the
// block's queries of head h, and the largest over the heads that share the keys.  In 64 bits: products of the sums with
// bfloat16 boxes and their sums are then exact but for terms 2^-50 of the largest, and the list does not hang on the order
// of a sum.  A lane holds VEC dimensions of u for every head of its group (up to SCORE_HEADS at a time) and reads VEC
// of either side of a box.  A score that is NaN counts as minus infinity.
constexpr int SCORE_HEADS = 4;
template <typename T, int D>
__global__ __launch_bounds__(256) void block_scores(BlockDims m, const T* __restrict__ q, KeyStride qs, const T* __restrict__ boxes,
                                                    double* __restrict__ scores, int pieces, int per) {
  constexpr int VEC = Vec<T>::N, LPR = D / VEC, RPI = 256 / LPR;
  const int piece = blockIdx.x % pieces, rest = blockIdx.x / pieces, i = rest % m.nb, hk = rest / m.nb % m.Hkv, b = rest / m.nb / m.Hkv;
  const BlockSeq s = block_seq(m, b);
  const Seen see = block_seen(m, s, i);
  const int p0 = piece * per, p1 = min(p0 + per, m.causal ? see.lo : see.seen);      // own pages need no score
  if (p0 >= p1 || see.seen <= m.topk) return;
  const int t0 = i * m.qblock, t1 = min(t0 + m.qblock, s.nq);
  const int tid = threadIdx.x, col = tid % LPR * VEC;
  double* const out = scores + (((long long)b * m.nb + i) * m.Hkv + hk) * m.max_pages;
  for (int h0 = 0; h0 < m.G; h0 += SCORE_HEADS) {
    const int H = min(SCORE_HEADS, m.G - h0);
    double u[SCORE_HEADS][VEC];
#pragma unroll
    for (int h = 0; h < SCORE_HEADS; ++h) {
#pragma unroll
      for (int x = 0; x < VEC; ++x) u[h][x] = 0.0;
      if (h < H)
        for (int t = t0; t < t1; ++t) {
          float v[VEC];
          unpack16<T>(*(const u32x4_t*)(q + (long long)(s.q0 + t) * qs.token + (hk * m.G + h0 + h) * qs.head + col), v);
#pragma unroll
          for (int x = 0; x < VEC; ++x) u[h][x] += (double)v[x];
        }
    }
    for (int p = p0 + tid / LPR; p < p1; p += RPI) {
      const int row = m.num_pages ? pool_page(m, b, p) : b * m.max_pages + p;
      double best = -INFINITY;
      if (row >= 0) {
        const T* const box = boxes + ((long long)row * m.Hkv + hk) * 2 * D + col;
        float mx[VEC], mn[VEC];
        unpack16<T>(*(const u32x4_t*)box, mx);
        unpack16<T>(*(const u32x4_t*)(box + D), mn);
#pragma unroll
        for (int h = 0; h < SCORE_HEADS; ++h) {
          double c = 0.0;
#pragma unroll
          for (int x = 0; x < VEC; ++x) c = fma(u[h][x], (double)(u[h][x] >= 0.0 ? mx[x] : mn[x]), c);
#pragma unroll
          for (int o = 1; o < LPR; o <<= 1) c += __shfl_xor(c, o);
          if (h < H && c > best) best = c;
        }
      }
      if (col == 0) out[p] = h0 ? fmax(out[p], best) : best + 0.0;      // (-0 + 0 = 0: equal to it in the order below)
    }
  }
}

// The larger score has the larger key.
__device__ __forceinline__ uint64_t order_key(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

// Pages of one block of queries and head of keys: its own pages and the first ones, and of the others those of the largest
// scores, ties to the lowest page, in ascending order.  The border is found digit by digit (8 bits) from the top.
__global__ __launch_bounds__(256) void block_topk(BlockDims m, const double* __restrict__ scores, int32_t* __restrict__ sel_idx, int32_t* __restrict__ sel_cnt) {
  const int hk = blockIdx.x % m.Hkv, i = blockIdx.x / m.Hkv % m.nb, b = blockIdx.x / m.Hkv / m.nb;
  const BlockSeq s = block_seq(m, b);
  const Seen see = block_seen(m, s, i);
  const long long rec = ((long long)b * m.nb + i) * m.Hkv + hk;
  int32_t* const idx = sel_idx + rec * m.topk;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (see.seen <= m.topk) {
    for (int j = tid; j < m.topk; j += 256) idx[j] = j < see.seen ? j : -1;
    if (tid == 0) sel_cnt[rec] = see.seen;
    return;
  }
  const double* const sc = scores + rec * m.max_pages;
  const int c0 = min(m.keep_first, m.causal ? see.lo : see.seen), c1 = m.causal ? see.lo : see.seen;       // pages [c0, c1) are chosen from
  const int need = m.topk - (see.seen - (c1 - c0));                                                       // (not below 0: the host has seen to it)
  __shared__ int32_t s_hist[256], s_wave[4];
  __shared__ int32_t s_digit, s_left, s_in;
  uint64_t prefix = 0, mask = 0;
  int left = need;                                   // of those that agree with the prefix
  if (need <= 0) prefix = mask = ~0ull;              // no score reaches it
  for (int shift = 56; shift >= 0 && need > 0; shift -= 8) {
    s_hist[tid] = 0;
    __syncthreads();
    for (int p = c0 + tid; p < c1; p += 256) {
      const uint64_t key = order_key(sc[p]);
      if ((key & mask) == prefix) atomicAdd(&s_hist[key >> shift & 255], 1);
    }
    __syncthreads();
    // counts from the top: thread t takes digit 255 - t
    const int n = s_hist[255 - tid];
    int incl = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int u = __shfl_up(incl, o); if (lane >= o) incl += u; }
    if (lane == 63) s_wave[wave] = incl;
    __syncthreads();
    for (int w = 0; w < wave; ++w) incl += s_wave[w];
    if (incl >= left && incl - n < left) { s_digit = 255 - tid; s_left = left - (incl - n); s_in = n; }
    __syncthreads();
    prefix |= (uint64_t)s_digit << shift;
    mask |= 255ull << shift;
    left = s_left;
    const bool all = s_left == s_in;                 // the whole digit is taken: the order inside it does not matter
    __syncthreads();
    if (all) break;
  }
  int written = 0, equal = 0;
  for (int base = 0; base < see.seen; base += 256) {
    const int p = base + tid;
    bool take = p < see.seen && (p < c0 || p >= c1), tie = false;
    if (p < see.seen && !take) {
      const uint64_t key = order_key(sc[p]) & mask;
      take = key > prefix;
      tie = key == prefix;
    }
    const uint64_t ties = __ballot(tie);
    if (lane == 0) s_wave[wave] = __popcll(ties);
    __syncthreads();
    int before = equal + __popcll(ties & ((1ull << lane) - 1));
    for (int w = 0; w < 4; ++w) { if (w < wave) before += s_wave[w]; equal += s_wave[w]; }
    take = take || (tie && before < left);
    __syncthreads();
    const uint64_t takes = __ballot(take);
    if (lane == 0) s_wave[wave] = __popcll(takes);
    __syncthreads();
    int at = written + __popcll(takes & ((1ull << lane) - 1));
    for (int w = 0; w < 4; ++w) { if (w < wave) at += s_wave[w]; written += s_wave[w]; }
    if (take) idx[at] = p;
    __syncthreads();
  }
  if (tid == 0) sel_cnt[rec] = m.topk;
}

}  // namespace

#define BY_TYPE(dtype, d, CALL)                                                           \
  if (dtype == ADACLUSTER_BF16) { if (d == 64) { CALL(bf16raw, 64); } else { CALL(bf16raw, 128); } } \
  else { if (d == 64) { CALL(float, 64); } else { CALL(float, 128); } }

int launch_cache_append(hipStream_t s, int dtype, int bits, int d, const CacheArgs& a) {
  const int touched = a.m.max_q >= 1 ? ((a.m.max_q - 1) >> a.m.lpage) + 2 : 0;
  const long long wg = (long long)touched * a.m.Hkv * a.m.B;
  if (!grid_fits(wg)) return ADACLUSTER_E_UNSUPPORTED;
#define CALL(T, D) if (bits == 4) cache_append<T, 4, D><<<(int)wg, 256, 0, s>>>(a, touched); else cache_append<T, 0, D><<<(int)wg, 256, 0, s>>>(a, touched)
  BY_TYPE(dtype, d, CALL)
#undef CALL
  return launched();
}

int launch_cache_read(hipStream_t s, int dtype, int bits, int d, const CacheArgs& a) {
  const int rpi = 256 * (dtype == ADACLUSTER_BF16 ? 8 : 4) / d;
  const long long pieces = ((long long)a.m.max_q * a.m.Hkv + rpi - 1) / rpi, wg = pieces * a.m.B;
  if (!grid_fits(wg) || pieces * rpi > INT32_MAX) return ADACLUSTER_E_UNSUPPORTED;
#define CALL(T, D) if (bits == 4) cache_read<T, 4, D><<<(int)wg, 256, 0, s>>>(a, (int)pieces); else cache_read<T, 0, D><<<(int)wg, 256, 0, s>>>(a, (int)pieces)
  BY_TYPE(dtype, d, CALL)
#undef CALL
  return launched();
}

int launch_block_boxes(hipStream_t s, int dtype, int d, const BlockDims& m, const void* k, KeyStride ks, void* boxes) {
  const long long wg = (long long)m.max_pages * m.Hkv * m.B;
  if (!grid_fits(wg)) return ADACLUSTER_E_UNSUPPORTED;
#define CALL(T, D) block_boxes<T, D><<<(int)wg, 256, 0, s>>>(m, (const T*)k, ks, (T*)boxes)
  BY_TYPE(dtype, d, CALL)
#undef CALL
  return launched();
}

size_t block_select_bytes(const BlockDims& m) { return (size_t)m.B * m.nb * m.Hkv * m.max_pages * sizeof(double); }

int launch_block_select(hipStream_t s, int dtype, int d, const BlockDims& m, const void* q, KeyStride qs, const void* boxes,
                        int32_t* sel_idx, int32_t* sel_cnt, void* ws) {
  const long long recs = (long long)m.B * m.nb * m.Hkv;
  const int per = 256, pieces = (m.max_pages + per - 1) / per;
  if (!grid_fits(recs * pieces)) return ADACLUSTER_E_UNSUPPORTED;
  if (m.max_pages > m.topk) {
#define CALL(T, D) block_scores<T, D><<<(int)(recs * pieces), 256, 0, s>>>(m, (const T*)q, qs, (const T*)boxes, (double*)ws, pieces, per)
    BY_TYPE(dtype, d, CALL)
#undef CALL
    if (int rc = launched()) return rc;
  }
  block_topk<<<(int)recs, 256, 0, s>>>(m, (const double*)ws, sel_idx, sel_cnt);
  return launched();
}

}  // namespace adac
