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
  const auto join = [&](auto ctrl) __attribute__((always_inline)) {      // with the lane that the DPP control names
    constexpr int C = decltype(ctrl)::value;
    lo = fminf(lo, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(lo), C, 0xF, 0xF, false)));
    hi = fmaxf(hi, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(hi), C, 0xF, 0xF, false)));
    ok &= __builtin_amdgcn_update_dpp(0, ok, C, 0xF, 0xF, false);
  };
  join(std::integral_constant<int, 0xB1>{});        // lanes 1 apart
  join(std::integral_constant<int, 0x4E>{});        // 2 apart
  join(std::integral_constant<int, 0x141>{});       // the other four of eight
  if constexpr (VEC == 4) join(std::integral_constant<int, 0x140>{});      // the other eight of sixteen
  const uint32_t lob = bf16_down(lo);
  const float low = __uint_as_float(lob << 16), span = hi - low;
  const uint32_t stb = bf16_up(span * (1.0f / 15.0f));
  const float step = __uint_as_float(stb << 16);
  if (!(ok && finite(span) && finite(step))) { *pair = 0x7FC07FC0u; return 0; }
  *pair = lob << 16 | stb;
  uint32_t codes = 0;
  if (step >= 0x1p-100f && step <= 0x1p100f) {
    // (v - low) / step as the division rounds it, from one reciprocal: with y = 1 / step rounded to nearest and q near the quotient,
    // q + (x - q step) y, the remainder exact by an fma, is the quotient rounded to nearest (Markstein, "Computation of elementary
    // functions on the IBM RISC System/6000 processor", 1990).  Divisions: 25 000 tokens of 8 heads, d = 128 40 us, 32 so.
    const float y = 1.0f / step;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const float x = v[i] - low, q = x * y, r = fmaf(fmaf(-q, step, x), y, q);
      codes |= (uint32_t)fminf(fmaxf(rintf(r), 0.f), 15.f) << (4 * i);
    }
  } else if (step > 0.f) {
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

// Scores of a block of queries against the boxes of pages: S(h, p) = sum_d u_d (u_d >= 0 ? max_pd : min_pd), u the sum of the block's
// queries of head h, and the largest over the heads that share the keys.  In 64 bits: products of the sums with bfloat16 boxes
// and their sums are then exact but for terms 2^-50 of the largest, and the list does not hang on the order of a sum.  A
// lane holds VEC dimensions of u for up to SCORE_HEADS heads and reads VEC of either side of a box; LPR lanes a page.
// A score that is NaN counts as minus infinity.
constexpr int SCORE_HEADS = 4;
template <typename T, int D>
__device__ __forceinline__ void load_box(const BlockDims& m, int b, int hk, int p, const T* __restrict__ boxes, int col, float* mx, float* mn, bool* there) {
  const int row = m.num_pages ? pool_page(m, b, p) : b * m.max_pages + p;
  *there = row >= 0;
  const T* const box = boxes + ((long long)max(row, 0) * m.Hkv + hk) * 2 * D + col;
  unpack16<T>(*(const u32x4_t*)box, mx);
  unpack16<T>(*(const u32x4_t*)(box + D), mn);
}
template <int CTRL> __device__ __forceinline__ double add_lane(double v) {      // + the value of the lane that CTRL names (DPP)
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xF, 0xF, false), hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xF, 0xF, false);
  return v + __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
template <int VEC, int LPR>
__device__ __forceinline__ double box_score(const double (*u)[VEC], int H, const float* mx, const float* mn) {
  double best = -INFINITY, c[SCORE_HEADS];
#pragma unroll
  for (int h = 0; h < SCORE_HEADS; ++h) {            // (all of them, whatever H: no branch between the sums, which then overlap)
    c[h] = 0.0;
#pragma unroll
    for (int x = 0; x < VEC; ++x) c[h] = fma(u[h][x], (double)(u[h][x] >= 0.0 ? mx[x] : mn[x]), c[h]);
  }
#pragma unroll
  for (int h = 0; h < SCORE_HEADS; ++h) c[h] = add_lane<0xB1>(c[h]);          // lanes 1 apart
#pragma unroll
  for (int h = 0; h < SCORE_HEADS; ++h) c[h] = add_lane<0x4E>(c[h]);          // 2 apart
#pragma unroll
  for (int h = 0; h < SCORE_HEADS; ++h) c[h] = add_lane<0x141>(c[h]);         // the other four of eight
  if constexpr (LPR >= 16)
#pragma unroll
    for (int h = 0; h < SCORE_HEADS; ++h) c[h] = add_lane<0x140>(c[h]);       // the other eight of sixteen
  if constexpr (LPR >= 32)
#pragma unroll
    for (int h = 0; h < SCORE_HEADS; ++h) c[h] += __shfl_xor(c[h], 16);
#pragma unroll
  for (int h = 0; h < SCORE_HEADS; ++h) if (h < H && c[h] > best) best = c[h];
  return best + 0.0;                                 // (-0 + 0 = 0: equal to it in the order below)
}

// The larger score has the larger key.
__device__ __forceinline__ uint64_t order_key(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);
  return u >> 63 ? ~u : u | 0x8000000000000000ull;
}

// The list of one block of queries and head of keys from its scores: its own pages and the first ones, and of the others those of the
// largest scores, ties to the lowest page, in ascending order.  The border is found digit by digit (8 bits) from the top.
template <int NT>
__device__ __forceinline__ void choose(const BlockDims& m, const Seen& see, const double* sc, int32_t* __restrict__ idx, int32_t* __restrict__ cnt) {
  constexpr int NW = NT / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c1 = m.causal ? see.lo : see.seen, c0 = min(m.keep_first, c1);       // pages [c0, c1) are chosen from
  const int need = m.topk - (see.seen - (c1 - c0));                            // (not below 0: the host has seen to it)
  __shared__ int32_t s_hist[256], s_wave[NW];
  __shared__ int32_t s_digit, s_left, s_in;
  uint64_t prefix = 0, mask = 0;
  int left = need;                                   // of those that agree with the prefix
  if (need <= 0) prefix = mask = ~0ull;              // no score reaches it
  const bool few = c1 - c0 <= NT;                    // a page a thread: those before it are counted
  for (int shift = 56; shift >= 0 && need > 0 && !few; shift -= 8) {
    if (tid < 256) s_hist[tid] = 0;
    __syncthreads();
    for (int p = c0 + tid; p < c1; p += NT) {
      const uint64_t key = order_key(sc[p]);
      if ((key & mask) == prefix) atomicAdd(&s_hist[key >> shift & 255], 1);
    }
    __syncthreads();
    // counts from the top: thread t takes digit 255 - t
    const int n = tid < 256 ? s_hist[255 - tid] : 0;
    int incl = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int u = __shfl_up(incl, o); if (lane >= o) incl += u; }
    if (lane == 63) s_wave[wave] = incl;
    __syncthreads();
    for (int w = 0; w < wave; ++w) incl += s_wave[w];
    if (tid < 256 && incl >= left && incl - n < left) { s_digit = 255 - tid; s_left = left - (incl - n); s_in = n; }
    __syncthreads();
    prefix |= (uint64_t)s_digit << shift;
    mask |= 255ull << shift;
    left = s_left;
    const bool all = s_left == s_in;                 // the whole digit is taken: the order inside it does not matter
    __syncthreads();
    if (all) break;
  }
  if (few) {
    __shared__ uint64_t s_take[NW], s_tie[NW];
    const int p = c0 + tid;
    const bool from = p < c1 && need > 0;
    const uint64_t key = order_key(sc[min(p, max(c1 - 1, 0))]);
    int above = 0;
    __shared__ uint64_t s_key[NT];
    s_key[tid] = p < c1 ? key : 0;                   // (0: above nothing)
    __syncthreads();
    if (__any(from))
      for (int x0 = 0; x0 < c1 - c0; x0 += 8) {      // (eight reads on their way at a time; NT is a multiple of it)
        uint64_t v[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) v[y] = s_key[x0 + y];
#pragma unroll
        for (int y = 0; y < 8; ++y) above += v[y] > key;
      }
    // taken: those with fewer than `need` above them, and of the last ones that tie as many as there is room for, in order
    const uint64_t w = __ballot(from && above < need);
    if (lane == 0) s_take[wave] = w;
    if (tid == 0) { s_left = 0; s_in = 0; }
    __syncthreads();
    int all = 0;
    for (int x = 0; x < NW; ++x) all += __popcll(s_take[x]);
    if (all > need && from && above < need) atomicMax(&s_left, above);           // the tie: the largest count
    __syncthreads();
    const bool tie = all > need && from && above == s_left, sure = from && above < need && !tie;
    const uint64_t ws = __ballot(sure), wt = __ballot(tie);
    __syncthreads();
    if (lane == 0) { s_take[wave] = ws; s_tie[wave] = wt; }
    __syncthreads();
    int room = need, at = c0, before = 0;            // (the first c0 pages are all taken)
    for (int x = 0; x < NW; ++x) room -= __popcll(s_take[x]);
    for (int x = 0; x < wave; ++x) { at += __popcll(s_take[x]); before += __popcll(s_tie[x]); }
    at += __popcll(ws & ((1ull << lane) - 1));
    before += __popcll(wt & ((1ull << lane) - 1));
    if (sure || (tie && before < room)) idx[at + min(before, room)] = p;
    for (int x = tid; x < c0; x += NT) idx[x] = x;
    for (int x = c1 + tid; x < see.seen; x += NT) idx[m.topk - see.seen + x] = x;
    if (tid == 0) *cnt = m.topk;
    return;
  }
  int written = 0, equal = 0;
  for (int base = 0; base < see.seen; base += NT) {
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
    for (int w = 0; w < NW; ++w) { if (w < wave) before += s_wave[w]; equal += s_wave[w]; }
    take = take || (tie && before < left);
    __syncthreads();
    const uint64_t takes = __ballot(take);
    if (lane == 0) s_wave[wave] = __popcll(takes);
    __syncthreads();
    int at = written + __popcll(takes & ((1ull << lane) - 1));
    for (int w = 0; w < NW; ++w) { if (w < wave) at += s_wave[w]; written += s_wave[w]; }
    if (take) idx[at] = p;
    __syncthreads();
  }
  if (tid == 0) *cnt = m.topk;
}

// All pages that can be listed fit: no score is asked.
template <int NT>
__device__ __forceinline__ void list_all(const BlockDims& m, const Seen& see, int32_t* __restrict__ idx, int32_t* __restrict__ cnt) {
  for (int j = threadIdx.x; j < m.topk; j += NT) idx[j] = j < see.seen ? j : -1;
  if (threadIdx.x == 0) *cnt = see.seen;
}

// u of a record: sums of the block's queries of every head, in 64 bits, to u_l [G][D] (parts: NT * VEC doubles of scratch).
template <typename T, int D, int NT>
__device__ __forceinline__ void block_sums(const BlockDims& m, const BlockSeq& s, int i, int hk, const T* __restrict__ q, const KeyStride& qs, double* u_l, double* parts) {
  constexpr int VEC = Vec<T>::N, LPR = D / VEC;
  const int tid = threadIdx.x, t0 = i * m.qblock, t1 = min(t0 + m.qblock, s.nq);
  // vectors of VEC dimensions; where there are fewer than threads, the tokens go to groups of threads whose sums are added in order
  const int vecs = m.G * LPR, groups = max(1, min(NT / vecs, t1 - t0)), g = tid / vecs;
  for (int v = tid % vecs; v < vecs && g < groups; v += NT) {              // (vecs > threads: one group, several vectors)
    const int h = v / LPR, c = v % LPR * VEC;
    double sum[VEC];
#pragma unroll
    for (int x = 0; x < VEC; ++x) sum[x] = 0.0;
    const T* const at = q + (long long)s.q0 * qs.token + (hk * m.G + h) * qs.head + c;
    for (int t = t0 + g; t < t1; t += 4 * groups) {                        // (four loads on their way at a time)
      u32x4_t w[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) w[y] = *(const u32x4_t*)(at + (long long)min(t + y * groups, t1 - 1) * qs.token);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        float f[VEC];
        unpack16<T>(w[y], f);
#pragma unroll
        for (int x = 0; x < VEC; ++x) sum[x] += t + y * groups < t1 ? (double)f[x] : 0.0;
      }
    }
#pragma unroll
    for (int x = 0; x < VEC; ++x) (groups > 1 ? parts + g * m.G * D : u_l)[h * D + c + x] = sum[x];
  }
  __syncthreads();
  if (groups > 1) {
    for (int x = tid; x < m.G * D; x += NT) {
      double sum = parts[x];
      for (int y = 1; y < groups; ++y) sum += parts[y * m.G * D + x];
      u_l[x] = sum;
    }
    __syncthreads();
  }
}

// Scores of pages [p0, p1) from u in LDS to sc, in 64 bits: LPR lanes a page.  list: the pages, or NULL: p0 .. in order.
template <typename T, int D, int NT>
__device__ __forceinline__ void exact_scores(const BlockDims& m, int b, int hk, const T* __restrict__ boxes, const double* u_l, int p0, int p1, const int32_t* list, double* sc) {
  constexpr int VEC = Vec<T>::N, LPR = D / VEC, RPI = NT / LPR, AHEAD = 2;
  const int tid = threadIdx.x, col = tid % LPR * VEC;
  for (int h0 = 0; h0 < m.G; h0 += SCORE_HEADS) {
    double u[SCORE_HEADS][VEC];
    const int H = min(SCORE_HEADS, m.G - h0);
#pragma unroll
    for (int h = 0; h < SCORE_HEADS; ++h)
#pragma unroll
      for (int x = 0; x < VEC; ++x) u[h][x] = h < H ? u_l[(h0 + h) * D + col + x] : 0.0;
    for (int p = p0 + tid / LPR; p < p1; p += RPI * AHEAD) {
      float mx[AHEAD][VEC], mn[AHEAD][VEC];
      bool there[AHEAD];
#pragma unroll
      for (int y = 0; y < AHEAD; ++y) {
        const int at = min(p + y * RPI, p1 - 1);
        load_box<T, D>(m, b, hk, list ? list[at] : at, boxes, col, mx[y], mn[y], &there[y]);
      }
#pragma unroll
      for (int y = 0; y < AHEAD; ++y) {
        const int at = p + y * RPI;
        double best = box_score<VEC, LPR>(u, H, mx[y], mn[y]);
        if (!there[y]) best = -INFINITY;
        if (col == 0 && at < p1) sc[at] = h0 ? fmax(sc[at], best) : best;
      }
    }
  }
  __syncthreads();
}

// A workgroup a record: sums of the block's queries, scores and list in one launch, u and the scores in LDS.
constexpr int PICK_PAGES = 4096, PICK_HEADS = 16;
template <typename T, int D, int PICK_NT>
__global__ __launch_bounds__(PICK_NT) void block_pick(BlockDims m, const T* __restrict__ q, KeyStride qs, const T* __restrict__ boxes,
                                                      int32_t* __restrict__ sel_idx, int32_t* __restrict__ sel_cnt) {
  extern __shared__ __align__(16) double lds[];      // [G][D] sums, then [max_pages] scores; before them the parts of the sums
  const int hk = blockIdx.x % m.Hkv, i = blockIdx.x / m.Hkv % m.nb, b = blockIdx.x / m.Hkv / m.nb;
  const BlockSeq s = block_seq(m, b);
  const Seen see = block_seen(m, s, i);
  const long long rec = ((long long)b * m.nb + i) * m.Hkv + hk;
  int32_t* const idx = sel_idx + rec * m.topk;
  if (see.seen <= m.topk) { list_all<PICK_NT>(m, see, idx, sel_cnt + rec); return; }
  double* const sc = lds + m.G * D;
  block_sums<T, D, PICK_NT>(m, s, i, hk, q, qs, lds, sc);
  exact_scores<T, D, PICK_NT>(m, b, hk, boxes, lds, 0, m.causal ? see.lo : see.seen, nullptr, sc);      // (own pages need no score)
  choose<PICK_NT>(m, see, sc, idx, sel_cnt + rec);
}

// Largest value over the 16 lanes that share lane / 16.
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, false)));       // lanes 1 apart
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xF, 0xF, false)));       // 2 apart
  v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xF, 0xF, false)));      // the other four of eight
  return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xF, 0xF, false)));   // the other eight
}
__device__ __forceinline__ uint32_t order_key32(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

// block_pick for bfloat16, with the scores bounded on the matrix cores first and formed in 64 bits only where the border of the list
// runs.  S = u+ max + u- min (u+, u-: u where it is >= 0, < 0), u as one or two bfloat16 (LO: sums of several queries; what is left out is
// below 2^-16 |u|), 16 pages x 16 heads a tile, and with the same products of absolute values the sum A of what was added.  S is off
// by at most 2^-12 A + 2^-70: at most 4 D products of exact factors added in fp32, each addition by 2^-22 of what it has, and
// products or factors below 2^-126 taken for 0 (u is held to 2^-60 .. 2^40 here; a record outside is scored in 64 bits throughout).
// With lo = S - e, hi = S + e (infinite where they are no numbers): a page whose hi is below the need-th largest lo is not
// taken, one whose lo is above the (need + 1)-th largest hi is, and the others, a handful, are scored in 64 bits.  Bound by the
// boxes it reads: 32 x 8 records of 1 640 pages on average (0.2 GB), 62 us; in 64 bits throughout 108.
constexpr int PICK_BORDER = 512;
template <int D, bool LO, int PICK_NT>
__global__ __launch_bounds__(PICK_NT, LO && D == 128 ? 3 : 4) void block_pick_bounds(BlockDims m, const bf16raw* __restrict__ q, KeyStride qs, const bf16raw* __restrict__ boxes,
                                                             int32_t* __restrict__ sel_idx, int32_t* __restrict__ sel_cnt) {
  constexpr int NF = D / 32, NW = PICK_NT / 64, PER = 8;
  extern __shared__ __align__(16) double lds[];      // [G][D] sums, then [max_pages] pairs of bounds; before them the parts of the sums
  __shared__ double border_sc[PICK_BORDER];
  __shared__ int32_t border_l[PICK_BORDER];
  __shared__ unsigned long long taken[PICK_PAGES / 64];
  __shared__ int32_t first_at[PICK_PAGES / 64], counts[2][NW][6], s_border, s_in, s_odd;
  const int hk = blockIdx.x % m.Hkv, i = blockIdx.x / m.Hkv % m.nb, b = blockIdx.x / m.Hkv / m.nb;
  const BlockSeq s = block_seq(m, b);
  const Seen see = block_seen(m, s, i);
  const long long rec = ((long long)b * m.nb + i) * m.Hkv + hk;
  int32_t* const idx = sel_idx + rec * m.topk;
  if (see.seen <= m.topk) { list_all<PICK_NT>(m, see, idx, sel_cnt + rec); return; }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n16 = lane & 15, quarter = lane >> 4;
  double* const u_l = lds;
  float2* const bound = (float2*)(lds + m.G * D);
  if (tid == 0) s_border = s_in = s_odd = 0;
  block_sums<bf16raw, D, PICK_NT>(m, s, i, hk, q, qs, u_l, lds + m.G * D);
  {
    bool odd = false;
    for (int x = tid; x < m.G * D; x += PICK_NT) { const double v = fabs(u_l[x]); odd = odd || !(v == 0.0 || (v >= 0x1p-60 && v <= 0x1p40)); }
    if (odd) s_odd = 1;
  }
  __syncthreads();
  const int c1 = m.causal ? see.lo : see.seen, c0 = min(m.keep_first, c1), need = m.topk - (see.seen - (c1 - c0));
  const auto exact = [&]() {
    __syncthreads();
    exact_scores<bf16raw, D, PICK_NT>(m, b, hk, boxes, u_l, 0, c1, nullptr, (double*)bound);
    choose<PICK_NT>(m, see, (const double*)bound, idx, sel_cnt + rec);
  };
  if (s_odd) { exact(); return; }
  if (need > 0) {
    // operands: column n16 is head n16
    RowFrag<bf16raw, D> ph, pl, nh, nl, pa, na;      // u+ and u-: upper and lower parts, and bounds of |u|
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t o[6] = {0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const double v = n16 < m.G ? u_l[n16 * D + 32 * f + 8 * quarter + 2 * w + x] : 0.0;
          const float vf = (float)v;
          const uint32_t h = f32_to_bf16(vf), l = LO ? f32_to_bf16((float)(v - (double)__uint_as_float(h << 16))) : 0, a = (h & 0x7FFF) + (vf != 0.f);
          const bool neg = vf < 0.f;
          o[neg ? 2 : 0] |= h << (16 * x);
          o[neg ? 3 : 1] |= l << (16 * x);
          o[neg ? 5 : 4] |= a << (16 * x);
        }
        ph.p[f][w] = o[0]; pl.p[f][w] = o[1]; nh.p[f][w] = o[2]; nl.p[f][w] = o[3]; pa.p[f][w] = o[4]; na.p[f][w] = o[5];
      }
    const int tiles = (c1 + 15) >> 4;
    auto row_of = [&](int t) __attribute__((always_inline)) {      // of the lane's page; -1: none
      const int p = min(t * 16 + n16, c1 - 1);
      return m.num_pages ? pool_page(m, b, p) : b * m.max_pages + p;
    };
    auto load = [&](RowFrag<bf16raw, D>& x, RowFrag<bf16raw, D>& y, int row) __attribute__((always_inline)) {
      const bf16raw* const box = boxes + ((long long)max(row, 0) * m.Hkv + hk) * 2 * D;
      load_frag(x, box, quarter, true);
      load_frag(y, box + D, quarter, true);
    };
    RowFrag<bf16raw, D> mx, mn;
    int row = wave < tiles ? row_of(wave) : -1, row1 = wave + NW < tiles ? row_of(wave + NW) : -1;
    if (wave < tiles) load(mx, mn, row);
    for (int t = wave; t < tiles; t += NW) {
      f32x4_t sc{0.f, 0.f, 0.f, 0.f}, ab = sc;
#pragma unroll
      for (int f = 0; f < NF; ++f) {
        sc = mma(bf16raw{}, mx.p[f], ph.p[f], sc);
        sc = mma(bf16raw{}, mn.p[f], nh.p[f], sc);
        if constexpr (LO) { sc = mma(bf16raw{}, mx.p[f], pl.p[f], sc); sc = mma(bf16raw{}, mn.p[f], nl.p[f], sc); }
        ab = mma(bf16raw{}, mx.p[f] & 0x7FFF7FFFu, pa.p[f], ab);
        ab = mma(bf16raw{}, mn.p[f] & 0x7FFF7FFFu, na.p[f], ab);
      }
      const bool none = row < 0;
      const int row2 = t + 2 * NW < tiles ? row_of(t + 2 * NW) : -1;
      if (t + NW < tiles) load(mx, mn, row1);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = fmaf(0x1p-12f, ab[j], 0x1p-70f);
        float lo = sc[j] - e, hi = sc[j] + e;
        if (!(finite(lo) && finite(hi))) { lo = -INFINITY; hi = INFINITY; }
        if (n16 >= m.G) lo = hi = -INFINITY;
        if (__shfl((int)none, 4 * quarter + j)) lo = hi = -INFINITY;      // (the page's row is looked up by lane page % 16)
        lo = row16_max(lo);
        hi = row16_max(hi);
        const int p = t * 16 + 4 * quarter + j;
        if (n16 == 0 && p < c1) bound[p] = float2{lo, hi};
      }
      row = row1; row1 = row2;
    }
  }
  __syncthreads();
  // what is taken for certain, and the border
  const auto settle = [&](int p, bool in, bool edge) {            // (all lanes of a wave, pages of 64 aligned to 64)
    const unsigned long long sure = __ballot(in), w = sure | __ballot(p < see.seen && (p < c0 || p >= c1));
    if (lane == 0) { taken[p >> 6] = w; if (sure) atomicAdd(&s_in, __popcll(sure)); }
    if (edge) { const int at = atomicAdd(&s_border, 1); if (at < PICK_BORDER) border_l[at] = p; }      // (in any order: pages decide ties)
  };
  // the need-th largest lo and the (need + 1)-th largest hi, two bits a turn, by counting what is not below three values in between
  uint32_t kl[PER], kh[PER];
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    const int p = c0 + tid + x * PICK_NT;
    kl[x] = kh[x] = 0;                               // (below all keys)
    if (need > 0 && p < c1) { const float2 v = bound[p]; kl[x] = order_key32(v.x); kh[x] = order_key32(v.y); }
  }
  uint32_t lth = 0, hth = 0;
  if (need > 0) {
    const int mine = (c1 - c0 + PICK_NT - 1) / PICK_NT;
    for (int shift = 30; shift >= 0; shift -= 2) {
      int n[6] = {0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int x = 0; x < PER; ++x) {
        if (x >= mine) break;
#pragma unroll
        for (int y = 0; y < 3; ++y) {
          n[y] += __popcll(__ballot(kl[x] >= (lth | (uint32_t)(y + 1) << shift)));
          n[3 + y] += __popcll(__ballot(kh[x] >= (hth | (uint32_t)(y + 1) << shift)));
        }
      }
      const int turn = (shift >> 1) & 1;             // (a slot is read before the barrier that the next writer of it passes)
      if (lane < 6) counts[turn][wave][lane] = lane == 0 ? n[0] : lane == 1 ? n[1] : lane == 2 ? n[2] : lane == 3 ? n[3] : lane == 4 ? n[4] : n[5];
      __syncthreads();
      int sum = 0;
      if (lane < 6) {
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += counts[turn][w][lane];
      }
      const unsigned long long up = __ballot(lane < 3 ? sum >= need : lane < 6 && sum >= need + 1);
      lth |= (uint32_t)__popcll(up & 7) << shift;
      hth |= (uint32_t)__popcll(up & 56) << shift;
    }
  }
#pragma unroll
  for (int x = 0; x < PER; ++x) {
    const int p = tid + x * PICK_NT;
    if (x * PICK_NT >= see.seen) break;
    bool in = false, edge = false;
    if (need > 0 && p >= c0 && p < c1) {
      const float2 v = bound[p];
      in = order_key32(v.x) > hth;
      edge = !in && order_key32(v.y) >= lth;
    }
    settle(p, in, edge);
  }
  __syncthreads();
  const int nb = s_border, left = need - s_in;
  if (nb > PICK_BORDER) { exact(); return; }
  if (nb == left) {
    for (int x = tid; x < nb; x += PICK_NT) atomicOr(&taken[border_l[x] >> 6], 1ull << (border_l[x] & 63));
  } else if (left > 0) {
    exact_scores<bf16raw, D, PICK_NT>(m, b, hk, boxes, u_l, 0, nb, border_l, border_sc);
    for (int x = tid; x < nb; x += PICK_NT) {
      const uint64_t key = order_key(border_sc[x]);
      const int p = border_l[x];
      int before = 0;
      for (int y = 0; y < nb; ++y) { const uint64_t other = order_key(border_sc[y]); before += other > key || (other == key && border_l[y] < p); }
      if (before < left) atomicOr(&taken[p >> 6], 1ull << (p & 63));
    }
  }
  __syncthreads();
  const int words = (see.seen + 63) >> 6;
  if (wave == 0) {
    const int n = lane < words ? __popcll(taken[lane]) : 0;
    int incl = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(incl, o); if (lane >= o) incl += v; }
    first_at[lane] = incl - n;
  }
  __syncthreads();
  for (int p = tid; p < see.seen; p += PICK_NT) {
    const unsigned long long w = taken[p >> 6], bit = 1ull << (p & 63);
    if (w & bit) idx[first_at[p >> 6] + __popcll(w & (bit - 1))] = p;
  }
  if (tid == 0) sel_cnt[rec] = m.topk;
}

// Few records over long contexts: scores by many workgroups, to memory, and the lists from there.
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
      float mx[VEC], mn[VEC];
      bool there;
      load_box<T, D>(m, b, hk, p, boxes, col, mx, mn, &there);
      double best = box_score<VEC, LPR>(u, H, mx, mn);
      if (!there) best = -INFINITY;
      if (col == 0) out[p] = h0 ? fmax(out[p], best) : best;
    }
  }
}

__global__ __launch_bounds__(256) void block_topk(BlockDims m, const double* __restrict__ scores, int32_t* __restrict__ sel_idx, int32_t* __restrict__ sel_cnt) {
  const int hk = blockIdx.x % m.Hkv, i = blockIdx.x / m.Hkv % m.nb, b = blockIdx.x / m.Hkv / m.nb;
  const BlockSeq s = block_seq(m, b);
  const Seen see = block_seen(m, s, i);
  const long long rec = ((long long)b * m.nb + i) * m.Hkv + hk;
  if (see.seen <= m.topk) list_all<256>(m, see, sel_idx + rec * m.topk, sel_cnt + rec);
  else choose<256>(m, see, scores + rec * m.max_pages, sel_idx + rec * m.topk, sel_cnt + rec);
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

// Whether a workgroup a record does (its u and scores in LDS): bfloat16 scores are bounds first; in 64 bits there have to be enough
// records to fill the chip, or few pages.
static bool picks(const BlockDims& m, int dtype) {
  const long long recs = (long long)m.B * m.nb * m.Hkv;
  return m.max_pages <= PICK_PAGES && m.G <= PICK_HEADS && (dtype == ADACLUSTER_BF16 || recs >= 128 || m.max_pages <= 1024);
}

size_t block_select_bytes(const BlockDims& m, int dtype) { return picks(m, dtype) ? 0 : (size_t)m.B * m.nb * m.Hkv * m.max_pages * sizeof(double); }

int launch_block_select(hipStream_t s, int dtype, int d, const BlockDims& m, const void* q, KeyStride qs, const void* boxes,
                        int32_t* sel_idx, int32_t* sel_cnt, void* ws) {
  const long long recs = (long long)m.B * m.nb * m.Hkv;
  const int per = 256, pieces = (m.max_pages + per - 1) / per;
  if (!grid_fits(recs * (picks(m, dtype) ? 2 : pieces))) return ADACLUSTER_E_UNSUPPORTED;
  if (picks(m, dtype)) {
    // Threads: 512 where a launch has few records, so that a CU has loads on their way (256 records of 2 048 pages 62 us, with 256
    // threads 76), 256 (more records a CU) else (512 records 116, with 512 threads 136).  Bounds pay from some 600 pages on (records of
    // 512 pages: 35 us in 64 bits, 42 with bounds; of 750: 31 and 29; of 2 048: 108 and 62).
    const bool wide = recs <= 256 || m.max_pages > 2048, bounds = dtype == ADACLUSTER_BF16 && m.max_pages > 512;
    const int nt = wide ? 512 : 256, parts = nt * (dtype == ADACLUSTER_BF16 ? 8 : 4);      // sums, then scores or the parts of the sums
    const size_t lds = ((size_t)m.G * d + (m.max_pages > parts ? m.max_pages : parts)) * sizeof(double);
#define CALL(T, D)                                                                                                                              \
  {                                                                                                                                             \
    if (wide) block_pick<T, D, 512><<<(int)recs, 512, lds, s>>>(m, (const T*)q, qs, (const T*)boxes, sel_idx, sel_cnt);                       \
    else block_pick<T, D, 256><<<(int)recs, 256, lds, s>>>(m, (const T*)q, qs, (const T*)boxes, sel_idx, sel_cnt);                            \
  }
#define BOUNDS(D, LO)                                                                                                                           \
  {                                                                                                                                             \
    if (wide) block_pick_bounds<D, LO, 512><<<(int)recs, 512, lds, s>>>(m, (const bf16raw*)q, qs, (const bf16raw*)boxes, sel_idx, sel_cnt);   \
    else block_pick_bounds<D, LO, 256><<<(int)recs, 256, lds, s>>>(m, (const bf16raw*)q, qs, (const bf16raw*)boxes, sel_idx, sel_cnt);        \
  }
    if (bounds) {
      if (m.qblock == 1) { if (d == 64) BOUNDS(64, false) else BOUNDS(128, false) }
      else { if (d == 64) BOUNDS(64, true) else BOUNDS(128, true) }
    } else {
      BY_TYPE(dtype, d, CALL)
    }
#undef CALL
#undef BOUNDS
    return launched();
  }
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
