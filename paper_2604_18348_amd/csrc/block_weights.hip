// The weight that every key of a paged cache gets from attention's rows.
#include "block_wide.h"

namespace adac {

namespace {

// w_j = decay w_j + sum over the rows r that see key j of 2^(scale log2(e) q_r . k_j - log2(e) lse_r): lse is the logarithm of the row's sum, so
// no maximum runs along.  No two workgroups add to a weight, and a call repeats bit for bit.
//
// Few rows: bound by the keys' bytes (one token of 32 sequences up to 16 384, 8 heads, d = 128: 173 us, 4.9 TB/s).  A wave has H sixteens of keys a
// turn, the next turn's on their way, and 16 rows at a time; a result tile holds in a lane one key and four rows, so that a key's step and
// lowest value, its sum and its weight are one lane's (4 bits, the same call: 256 us with a lane's four keys and one row, 93 so, bound by what
// becomes of a code).
//
// 4 bits, bf16: a code c enters as the bfloat16 16 + c (0x4180 | c << 3: exact), which leaves the dimensions of a word of eight in the
// order 0 4 1 5 2 6 3 7; the accumulator starts at -16 sum q, and steps and lowest values come behind the product, a group of 64.  (Attention
// takes 128 + c, a shift less; that is off by five times as much, which its sums over keys average out.)
template <typename T, int BITS, int D> struct RawKeys {      // of one row
  static constexpr int NF = D * sizeof(T) / 64, NG = D / 64;
  u32x4_t f[BITS ? 1 : NF];
  uint2 c[BITS ? NG : 1];
  uint32_t pair[BITS ? NG : 1];
};
// piece x of a lane's row: its place in a row of D elements
template <typename T, int BITS> __device__ __forceinline__ int piece_of(int x, int quarter) {
  if constexpr (BITS == 0) return 4 * x + quarter;
  else if constexpr (sizeof(T) == 2) return 8 * (x >> 1) + 2 * quarter + (x & 1);
  else return 16 * (x >> 2) + 4 * quarter + (x & 3);
}
template <typename T, int BITS, int D>
__device__ __forceinline__ void expand_keys(RowFrag<T, D>& f, const RawKeys<T, BITS, D>& r) {
#pragma unroll
  for (int x = 0; x < RawKeys<T, BITS, D>::NF; ++x) {
    if constexpr (BITS == 0) f.p[x] = r.f[x];
    else if constexpr (sizeof(T) == 2) {
      const uint32_t w = x & 1 ? r.c[x >> 1].y : r.c[x >> 1].x;
      f.p[x] = u32x4_t{(w << 3 & 0x00780078u) | 0x41804180u, (w >> 1 & 0x00780078u) | 0x41804180u, (w >> 5 & 0x00780078u) | 0x41804180u,
                       (w >> 9 & 0x00780078u) | 0x41804180u};
    } else {
      const uint32_t pair = r.pair[x >> 2], w = ((x >> 1) & 1 ? r.c[x >> 2].y : r.c[x >> 2].x) >> (16 * (x & 1));
      const float step = __uint_as_float(pair << 16), low = __uint_as_float(pair & 0xFFFF0000u);
#pragma unroll
      for (int j = 0; j < 4; ++j) f.p[x][j] = __float_as_uint(fmaf((float)(w >> (4 * j) & 15), step, low));
    }
  }
}

constexpr int KEY_TILES = 2;                          // of 16 keys a wave and turn
template <typename T, int BITS, int D>
__global__ __launch_bounds__(256, D == 128 && sizeof(T) == 4 ? 2 : 4) void cache_weights(WeightsArgs a, int chunks, int items) {
  constexpr int NF = D * sizeof(T) / 64, NG = D / 64, H = KEY_TILES, CHUNK = 64 * H;
  constexpr bool CODES = BITS == 4 && sizeof(T) == 2;
  const BlockDims& m = a.m;
  const int chunk0 = blockIdx.x % items, hk = blockIdx.x / items % m.Hkv, b = blockIdx.x / items / m.Hkv;
  const BlockSeq s = block_seq(m, b);
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), n16 = lane & 15, quarter = lane >> 4, most = m.max_pages << m.lpage;
  const int rows = s.nq * m.G;

  // 16 rows: their operand, and of the lane's four what is taken off a score, the keys they see, sums of q
  RowFrag<T, D> q;
  float off[4];
  int lim[4];
  f32x4_t qsum[CODES ? NG : 1];
  const auto load_rows = [&](int row0) __attribute__((always_inline)) {
    const int row = row0 + n16, t = row / m.G;
    const T* const p = (const T*)a.q + (long long)(s.q0 + t) * a.qs.token + (long long)(hk * m.G + row % m.G) * a.qs.head;
#pragma unroll
    for (int f = 0; f < NF; ++f) q.p[f] = row < rows ? *(const u32x4_t*)(p + piece_of<T, BITS>(f, quarter) * Vec<T>::N) : u32x4_t{0, 0, 0, 0};
    const float lse = row < rows ? a.lse[(long long)(s.q0 + t) * m.Hq + hk * m.G + row % m.G] : -INFINITY;
    const float o = lse == -INFINITY ? INFINITY : lse * LOG2E;      // (a row without keys weighs none)
    const int l = row < rows ? (m.causal ? min(s.n, s.first + t + 1) : s.n) : 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) { off[j] = __shfl(o, 4 * quarter + j); lim[j] = __shfl(l, 4 * quarter + j); }
    if constexpr (CODES) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          u32x4_t& x = q.p[2 * g + c];
#pragma unroll
          for (int j = 0; j < 4; ++j) sum += __uint_as_float(x[j] << 16) + __uint_as_float(x[j] & 0xFFFF0000u);
          // dimensions 0..7 -> 0 4 1 5 2 6 3 7
          x = u32x4_t{(x[0] & 0xFFFFu) | x[2] << 16, x[0] >> 16 | (x[2] & 0xFFFF0000u), (x[1] & 0xFFFFu) | x[3] << 16, x[1] >> 16 | (x[3] & 0xFFFF0000u)};
        }
        sum = quarters_sum(sum);
#pragma unroll
        for (int j = 0; j < 4; ++j) qsum[g][j] = __shfl(sum, 4 * quarter + j);
      }
    }
  };

  // A turn's keys are loaded one turn ahead, their places in the pool two.
  struct Turn { RawKeys<T, BITS, D> k[H]; int end[H]; };      // end: keys from here on do not exist
  int place[H];
  const auto places = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int key = chunk * CHUNK + (wave * H + h) * 16;
      place[h] = chunk < chunks && key < s.n ? pool_page(m, b, key >> m.lpage) : -1;
    }
  };
  const auto fetch = [&](Turn& t, int chunk) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const int key = chunk * CHUNK + (wave * H + h) * 16, in = key & (m.page - 1), phys = uniform(place[h]);
      const bool there = phys >= 0 && key + n16 < s.n;
      t.end[h] = phys >= 0 ? s.n : 0;
      if constexpr (BITS == 0) {
        const T* const p = (const T*)a.k + max(phys, 0) * a.ks.page + (there ? in + n16 : 0) * a.ks.token + hk * a.ks.head;
#pragma unroll
        for (int f = 0; f < NF; ++f) t.k[h].f[f] = there ? *(const u32x4_t*)(p + (4 * f + quarter) * Vec<T>::N) : u32x4_t{0, 0, 0, 0};
      } else {
        const long long row = ((long long)max(phys, 0) * m.Hkv + hk) * m.page + in + n16;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          t.k[h].c[g] = there ? ((const uint2*)((const char*)a.k + row * (D / 2)))[quarter + 4 * g] : uint2{0, 0};
          t.k[h].pair[g] = there ? a.km[row * NG + g] : 0;
        }
      }
    }
  };
  Turn next;
  places(chunk0);
  fetch(next, chunk0);
  places(chunk0 + items);
  const bool once = rows <= 16;
  if (once) load_rows(0);
  for (int chunk = chunk0; chunk < chunks; chunk += items) {
    const int key0 = chunk * CHUNK + wave * H * 16;
    float w[H], before[H];
    RowFrag<T, D> k[H];
    float step[H][NG], low[H][NG];
    int end[H];
#pragma unroll
    for (int h = 0; h < H; ++h) {
      w[h] = 0.f;
      const int at = key0 + 16 * h + n16;
      before[h] = a.w && at < s.n ? a.w[((long long)b * m.Hkv + hk) * most + at] : 0.f;
      expand_keys<T, BITS, D>(k[h], next.k[h]);
      end[h] = next.end[h];
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        step[h][g] = CODES ? __uint_as_float(next.k[h].pair[BITS ? g : 0] << 16) : 0.f;
        low[h][g] = CODES ? __uint_as_float(next.k[h].pair[BITS ? g : 0] & 0xFFFF0000u) : 0.f;
      }
    }
    fetch(next, chunk + items);
    places(chunk + 2 * items);
    // causal: from the first query that sees key0
    const long long first = m.causal ? (long long)max(0, key0 - s.first) * m.G : 0;
    if (key0 < s.n)
      for (int row0 = (int)min(first, (long long)rows) & ~15; row0 < rows; row0 += 16) {
        if (!once) load_rows(row0);
#pragma unroll
        for (int h = 0; h < H; ++h) {
          f32x4_t sc;
          if constexpr (CODES) {
            sc = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              f32x4_t x = qsum[g] * -16.f;
              x = mma(T{}, q.p[2 * g], k[h].p[2 * g], x);
              x = mma(T{}, q.p[2 * g + 1], k[h].p[2 * g + 1], x);
#pragma unroll
              for (int j = 0; j < 4; ++j) sc[j] = fmaf(step[h][g], x[j], fmaf(low[h][g], qsum[g][j], sc[j]));
            }
          } else {
            sc = dots(q, k[h]);
          }
          const int at = key0 + 16 * h + n16;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float p = __builtin_amdgcn_exp2f(fmaf(sc[j], a.scale_log2e, -off[j]));
            w[h] += at < min(lim[j], end[h]) ? p : 0.f;
          }
        }
      }
#pragma unroll
    for (int h = 0; h < H; ++h) {
      const float sum = quarters_sum(w[h]);
      const int at = key0 + 16 * h + n16;
      if (quarter == 0 && at < most) a.out[((long long)b * m.Hkv + hk) * most + at] = at >= s.n ? 0.f : a.w ? fmaf(a.decay, before[h], sum) : sum;
    }
  }
}

// Many rows (bf16): 32 x 32 products.  A wave keeps the operands of KT * 32 keys in registers while 64 rows at a time go through LDS, staged once for
// all four waves by direct loads, one stage ahead (they stay there for further keys if they all fit).  Bound by vector arithmetic and matrix cores at
// once: for a wave's 64 weights an exponential (8 cycles of a SIMD), a multiply-add and an addition (4 each) beside 16 of the product at
// d = 128; of the cycles the matrix cores have 44 %, the vector units 64 %, at the 1.8 GHz that the power limit leaves.  Chunks of 2 x 1 024
// tokens, 32 / 8 heads, up to 16 384 keys: 1 048 us by 16 x 16 products without stages, 352 staged, 305 with a tile's products in turn with
// the weights of the one before (each in its first twenty calls; call after call the last one takes 273).
//
// 4 bits: a code c is a bfloat16 by itself.  Per group g of 64 dimensions x_g = c . q, and score = sum over g of step_g x_g + low_g sum_g q.
// The latter, scaled, less the row's log2(e) lse is one more product, of (low, low, low, .., -1, -1, -1) with three bfloat16 parts (24 bits) of every
// factor, which weights_sums has left: what remains is two multiplications, the exponential and an addition (64 tokens of 4 sequences up to 32 768:
// 214 us a step and lowest value a weight, 108 so, with a chunk's codes loaded a chunk ahead, 104 with its sums over the lanes in registers; call after
// call 93).

// 32 bytes a row and head: the sums of q over 64 dimensions, times scale log2(e), in three parts each, for the lanes below 32, and log2(e) lse
// in three parts for the others, which meet -1.
template <int D>
__global__ __launch_bounds__(256) void weights_sums(WeightsArgs a, u32x4_t* __restrict__ parts) {
  const BlockDims& m = a.m;
  const long long id = (long long)blockIdx.x * 64 + threadIdx.x / 4;      // 4 lanes a row and head
  if (id >= (long long)m.q_rows * m.Hq) return;                           // (whole quads)
  const int l = threadIdx.x & 3;
  const bf16raw* const p = (const bf16raw*)a.q + (id / m.Hq) * a.qs.token + (id % m.Hq) * a.qs.head + l * 16;
  uint32_t h[9] = {0, 0, 0, 0, 0, 0, 0, 0, 0};
  const auto cut = [&](float s, int at) __attribute__((always_inline)) {      // (cut, not rounded: what is left is exact)
#pragma unroll
    for (int x = 0; x < 3; ++x) { h[at + x] = __float_as_uint(s) >> 16; s -= __uint_as_float(h[at + x] << 16); }
  };
#pragma unroll
  for (int g = 0; g < D / 64; ++g) {
    float s = 0.f;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const u32x4_t w = *(const u32x4_t*)(p + g * 64 + x * 8);
#pragma unroll
      for (int j = 0; j < 4; ++j) s += __uint_as_float(w[j] << 16) + __uint_as_float(w[j] & 0xFFFF0000u);
    }
    s += __shfl_xor(s, 1);
    s += __shfl_xor(s, 2);
    cut(s * a.scale_log2e, 3 * g);
  }
  const float lse = a.lse[id];
  cut(fabsf(lse) == INFINITY ? 0x1p126f : lse * LOG2E, 6);      // (a row without keys weighs none)
  if (l == 0) parts[2 * id] = u32x4_t{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, 0};
  if (l == 1) parts[2 * id + 1] = u32x4_t{h[6] | h[7] << 16, h[8], 0, 0};
}

template <int CTRL> __device__ __forceinline__ float of_lane(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false)); }
// Of 2 n sums a lane keeps n, the upper ones where `bit` is set, and adds those of the lane CTRL names, whose bit is the other one.
template <int CTRL, int BIT, int N> __device__ __forceinline__ void halve(float* w, int lane) {
  const bool up = lane & BIT;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float give = up ? w[i] : w[i + N], mine = up ? w[i + N] : w[i];
    w[i] = mine + of_lane<CTRL>(give);
  }
}

constexpr int STAGE_ROWS = 64, STAGES = 4;      // of q in LDS: all rows of a share stay there if they fit
constexpr int key_tiles(int bits, int d) { return bits && d == 128 ? 1 : 2; }      // of 32 keys a wave (4 bits, d = 128: steps take the registers of the second)

template <int BITS, int D>
__global__ __launch_bounds__(256, 2) void cache_weights_wide(WeightsArgs a, int chunks, int items, int split) {
  constexpr int KT = key_tiles(BITS, D), KS = D / 16, CH = D / 8, ROWB = D * 2, NG = D / 64;
  constexpr int PT = STAGE_ROWS * CH / 256, STAGEB = STAGE_ROWS * ROWB;
  __shared__ __align__(16) char lds[STAGES * STAGEB];
  __shared__ __align__(16) u32x4_t sums_l[BITS ? STAGES : 1][2][BITS ? STAGE_ROWS : 1];      // (of both halves of the lanes)
  __shared__ __align__(16) float step_l[BITS ? 4 : 1][KT][NG][BITS ? 32 : 1];
  __shared__ float lse_l[BITS ? 1 : STAGES][STAGE_ROWS];
  const BlockDims& m = a.m;
  const HeadItem it = xcd_item(blockIdx.x, m.B * m.Hkv, items * a.nsplit, split);
  if (it.head < 0) return;
  const int share = it.item % a.nsplit, hk = it.head % m.Hkv, b = it.head / m.Hkv;
  const BlockSeq s = block_seq(m, b);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, hb = lane >> 5;
  const int most = m.max_pages << m.lpage;
  // the rows of this share, in stages
  const int all_rows = s.nq * m.G, from = (int)((long long)all_rows * share / a.nsplit), rows = (int)((long long)all_rows * (share + 1) / a.nsplit);
  const int stages = (rows - from + STAGE_ROWS - 1) / STAGE_ROWS;

  // Where this thread's pieces of a stage lie, in bytes from the token of the stage's first row (below 2^32: near() sees to it); if the
  // heads of a key do not divide 64 they change from stage to stage, without a division.
  const int ht = STAGE_ROWS / m.G, hr = STAGE_ROWS % m.G;
  const uint32_t token = (uint32_t)(a.qs.token * 2), head = (uint32_t)(a.qs.head * 2);
  uint32_t src[PT], lsrc = 0;                          // lsrc: of lse and of the sums, as an index
  int h[PT], lh = 0, stage_t = 0, stage_h = 0;         // heads; the stage's first row
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void_t*)lds, lse0 = (uint32_t)(uintptr_t)(lds_void_t*)&lse_l[0][0], sums0 = (uint32_t)(uintptr_t)(lds_void_t*)&sums_l[0][0];
  const uint32_t piece = ((tid % CH) ^ swz<D>(tid / CH)) * 16;      // (of all its pieces: the slots repeat every 16 rows)
  const auto start = [&](int stage) {
    const int r0 = from + stage * STAGE_ROWS;
    stage_t = uniform(r0 / m.G); stage_h = uniform(r0 % m.G);
#pragma unroll
    for (int x = 0; x < PT; ++x) {
      const int r = stage_h + (tid + x * 256) / CH;
      h[x] = r % m.G;
      src[x] = r / m.G * token + h[x] * head + piece;
    }
    lh = (stage_h + lane) % m.G;
    lsrc = (stage_h + lane) / m.G * m.Hq + lh;
  };
  const auto issue = [&](int stage) __attribute__((always_inline)) {      // (rows past the end: the stage's first, masked)
    const int r0 = from + stage * STAGE_ROWS, slot = stage % STAGES;
    const char* const q = uniform((const char*)a.q + ((long long)(s.q0 + stage_t) * a.qs.token + (long long)hk * m.G * a.qs.head) * 2);
    const long long l = (long long)(s.q0 + stage_t) * m.Hq + hk * m.G;
    const bool whole = r0 + STAGE_ROWS <= rows;
#pragma unroll
    for (int x = 0; x < PT; ++x) {
      const uint32_t off = whole || r0 + (tid + x * 256) / CH < rows ? src[x] : stage_h * head + piece;
      dma_b128(lds0 + slot * STAGEB + (wave * 64 + x * 256) * 16, off, q);
    }
    if (wave == 0) {
      const uint32_t off = whole || r0 + lane < rows ? lsrc : (uint32_t)stage_h;
      if constexpr (BITS == 0) {
        dma_b32(lse0 + slot * STAGE_ROWS * 4, off * 4, uniform((const char*)(a.lse + l)));
      } else {
        dma_b128(sums0 + slot * STAGE_ROWS * 32, off * 32, uniform((const char*)(a.sums + 2 * l)));
        dma_b128(sums0 + slot * STAGE_ROWS * 32 + STAGE_ROWS * 16, off * 32 + 16, uniform((const char*)(a.sums + 2 * l)));
      }
    }
    stage_t += ht;
    if (hr) {
      stage_h += hr;
      const bool next = stage_h >= m.G;                 // (the token of the first row moves on by one more)
      if (next) { stage_h -= m.G; ++stage_t; }
      const auto turn = [&](int& hx, uint32_t& at, uint32_t per_head, uint32_t per_token) __attribute__((always_inline)) {
        hx += hr;
        at += hr * per_head;
        if (hx >= m.G) { hx -= m.G; at += per_token - m.G * per_head; }
        if (next) at -= per_token;
      };
#pragma unroll
      for (int x = 0; x < PT; ++x) turn(h[x], src[x], head, token);
      turn(lh, lsrc, 1, m.Hq);
    }
  };

  // 4 bits: a chunk's codes and pairs are loaded one chunk ahead, its places in the pool two.
  struct Raw { uint32_t code[KT][KS], pair[KT][NG], named[KT]; };
  struct Place { int entry[KT]; };
  const auto place = [&](int chunk) __attribute__((always_inline)) {      // the table's entries of the lane's keys, as they are: nothing waits for them here
    Place p;
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      const int key = chunk * 128 * KT + wave * 32 * KT + 32 * x + c;
      p.entry[x] = -1;
      if (key < s.n) p.entry[x] = m.table[(long long)b * m.max_pages + (key >> m.lpage)];
    }
    return p;
  };
  const auto fetch = [&](Raw& r, int chunk, const Place& p) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < KT; ++x) {
      const int key = chunk * 128 * KT + wave * 32 * KT + 32 * x + c;
      const bool there = (unsigned)p.entry[x] < (unsigned)m.num_pages;
      const long long row = ((long long)p.entry[x] * m.Hkv + hk) * m.page + (key & (m.page - 1));
      r.named[x] = (uint32_t)__ballot(there);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) r.code[x][ks] = there ? ((const uint32_t*)a.k)[row * (D / 8) + ks * 2 + hb] : 0;
#pragma unroll
      for (int g = 0; g < NG; ++g) r.pair[x][g] = there ? a.km[row * NG + g] : 0;
    }
  };
  const int chunk0 = it.item / a.nsplit, mine = 8 * (c / 8) + 4 * hb + (c >> 1) % 4;      // the key of 32 that the lane is left with at the end
  Raw next;
  Place after;
  if constexpr (BITS == 4) { after = place(chunk0); fetch(next, chunk0, after); after = place(chunk0 + items); }

  int qrow[KS];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qrow[ks] = row_operand<D>(lane, ks);
  bool loaded = false;                                  // the rows are in LDS, from the first that a chunk so far has wanted on
  for (int chunk = chunk0; chunk < chunks; chunk += items) {
    const int first_key = chunk * 128 * KT, key0 = first_key + wave * 32 * KT;
    // the first stage with a row that sees a key of the workgroup
    const long long row0 = m.causal ? (long long)max(0, first_key - s.first) * m.G : 0;
    const int stage0 = first_key >= s.n || row0 >= rows ? stages : (int)max(0ll, row0 - from) / STAGE_ROWS;
    float w[KT][16], before[KT];
    uint32_t named[KT];                                 // keys that there are
#pragma unroll
    for (int x = 0; x < KT; ++x)
#pragma unroll
      for (int v = 0; v < 16; ++v) w[x][v] = 0.f;
#pragma unroll
    for (int x = 0; x < KT; ++x) { named[x] = 0; before[x] = 0.f; }
    if (stage0 < stages) {
      if (!loaded) { start(stage0); issue(stage0); }
      if (a.w && a.nsplit == 1) {                       // what the end adds to
#pragma unroll
        for (int x = 0; x < KT; ++x) if (mine + 32 * x < s.n - key0) before[x] = a.w[((long long)b * m.Hkv + hk) * most + key0 + 32 * x + mine];
      }
      bf16x8_t k[KT][KS], low[BITS ? KT : 1];
      float step[KT][NG][BITS ? 16 : 1];
      if constexpr (BITS == 0) {
#pragma unroll
        for (int x = 0; x < KT; ++x) {
          const int key = key0 + 32 * x + c, phys = key < s.n ? pool_page(m, b, key >> m.lpage) : -1;
          named[x] = (uint32_t)__ballot(phys >= 0);
          const bf16raw* const p = (const bf16raw*)a.k + (phys < 0 ? 0 : phys * a.ks.page + (key & (m.page - 1)) * a.ks.token + hk * a.ks.head);
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const u32x4_t u = phys < 0 ? u32x4_t{0, 0, 0, 0} : *(const u32x4_t*)(p + ks * 16 + hb * 8);
            k[x][ks] = *(const bf16x8_t*)&u;
          }
        }
      } else {
        compiler_fence();
#pragma unroll
        for (int x = 0; x < KT; ++x) {
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            union { uint32_t w[4]; bf16x8_t v; } u;
            const uint32_t even = next.code[x][ks] & 0x0F0F0F0Fu, odd = next.code[x][ks] >> 4 & 0x0F0F0F0Fu;
#pragma unroll
            for (int j = 0; j < 4; ++j) u.w[j] = __float_as_uint((float)(even >> (8 * j) & 255)) >> 16 | __float_as_uint((float)(odd >> (8 * j) & 255));
            k[x][ks] = u.v;
          }
          named[x] = next.named[x];
          const uint32_t l0 = next.pair[x][0] >> 16, l1 = NG == 2 ? next.pair[x][NG - 1] >> 16 : 0;
          union { uint32_t w[4]; bf16x8_t v; } u{{l0 | l0 << 16, l0 | l1 << 16, l1 | l1 << 16, 0}};
          if (hb) { u.w[0] = 0xBF80BF80u; u.w[1] = 0xBF80u; u.w[2] = 0; }
          low[x] = u.v;
#pragma unroll
          for (int g = 0; g < NG; ++g) step_l[wave][x][g][c] = __uint_as_float(next.pair[x][g] << 16) * a.scale_log2e;
        }
        compiler_fence();
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
          for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const f32x4_t z = *(const f32x4_t*)&step_l[wave][x][g][8 * y + 4 * hb];
#pragma unroll
              for (int j = 0; j < 4; ++j) step[x][g][4 * y + j] = z[j];
            }
        compiler_fence();
        if (chunk + items < chunks) { fetch(next, chunk + items, after); after = place(chunk + 2 * items); }
      }
      // Rows from which on all keys of the wave are seen.  (Keys that do not exist are left out at the end.)
      const int last = min(key0 + 32 * KT, s.n) - 1;
      const long long free_row = m.causal ? (long long)max(0, last - s.first) * m.G : 0;
      if (!loaded) { wait_vmcnt<0>(); lds_barrier(); }
      for (int stage = stage0; stage < stages; ++stage) {
        if (!loaded && stage + 1 < stages) issue(stage + 1);
        const int slot = stage % STAGES, r0 = from + stage * STAGE_ROWS;
        const char* const qt = lds + slot * STAGEB;
        const auto rows_of = [&](int half, bf16x8_t* q) __attribute__((always_inline)) {
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) q[ks] = *(const bf16x8_t*)(qt + qrow[ks] + half * 32 * ROWB);
        };
        const auto offset = [&](int half) __attribute__((always_inline)) {
          const float lse = lse_l[BITS ? 0 : slot][half * 32 + c];
          return lse == -INFINITY || r0 + half * 32 + c >= rows ? INFINITY : lse * LOG2E;      // (a row without keys, or behind the last, weighs none)
        };
        const auto sums = [&](int half) __attribute__((always_inline)) {
          u32x4_t u = sums_l[slot][BITS ? hb : 0][BITS ? half * 32 + c : 0];
          if (hb && r0 + half * 32 + c >= rows) u[0] = 0x7E80;      // (2^126, beside whatever else is there: nor does it here)
          return *(const bf16x8_t*)&u;
        };
        // exponents of 32 keys and 32 rows
        const auto scores = [&](int x, int half, const bf16x8_t* q, f32x16_t* y) __attribute__((always_inline)) {
          if constexpr (BITS == 0) {
            y[0] = zero16();
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) y[0] = mfma32(k[x][ks], q[ks], y[0]);
          } else {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              y[g] = zero16();
#pragma unroll
              for (int ks = 0; ks < 4; ++ks) y[g] = mfma32(k[x][4 * g + ks], q[4 * g + ks], y[g]);
            }
            y[NG] = mfma32(low[BITS ? x : 0], sums(half), zero16());
          }
        };
        const auto weight = [&](int x, const f32x16_t* y, float off, int v) __attribute__((always_inline)) {
          if constexpr (BITS == 0) return __builtin_amdgcn_exp2f(fmaf(y[0][v], a.scale_log2e, -off));
          float e = y[NG][v];
#pragma unroll
          for (int g = 0; g < NG; ++g) e = fmaf(step[x][g][v], y[g][v], e);
          return __builtin_amdgcn_exp2f(e);
        };
        constexpr int NY = BITS ? NG + 1 : 1, MT = KS + (BITS ? 1 : 0);
        if (r0 >= free_row) {
          // The products of a tile in turn with the weights of the one before, as written: left to itself the compiler puts all products
          // first, and a wave's matrix core waits for its exponentials.
          f32x16_t y[2][NY];
          bf16x8_t q[KS];
          rows_of(0, q);
          const float off[2] = {BITS ? 0.f : offset(0), BITS ? 0.f : offset(1)};
          scores(0, 0, q, y[0]);
#pragma unroll
          for (int i = 1; i <= 2 * KT; ++i) {
            const int x = i % KT, half = i / KT, px = (i - 1) % KT, ph = (i - 1) / KT;
            const bool more = i < 2 * KT;
            f32x16_t* const z = y[i & 1];
            if (KT == 1 && more) rows_of(half, q);
#pragma unroll
            for (int j = 0; j < MT; ++j) {
              if (more) {
                if (j == KS) z[NY - 1] = mfma32(low[BITS ? x : 0], sums(half), zero16());
                else if (BITS == 0) z[0] = mfma32(k[x][j], q[j], j ? z[0] : zero16());
                else z[j / 4] = mfma32(k[x][j], q[j], j % 4 ? z[j / 4] : zero16());
                if (x == KT - 1 && half == 0 && j < KS) q[j] = *(const bf16x8_t*)(qt + qrow[j] + 32 * ROWB);      // (KT 2: the second half's)
              }
#pragma unroll
              for (int v = 16 * max(0, j - 1) / (MT - 1); v < 16 * j / (MT - 1); ++v) w[px][v] += weight(px, y[(i - 1) & 1], off[ph], v);
              if (more) __builtin_amdgcn_sched_barrier(0);
            }
          }
        } else {
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            bf16x8_t q[KS];
            rows_of(half, q);
            const float off = BITS ? 0.f : offset(half);
            const int row = r0 + half * 32 + c;
            const int lim = row >= rows ? 0 : m.causal ? s.first + row / m.G + 1 - (key0 + 4 * hb) : 32 * KT;
#pragma unroll
            for (int x = 0; x < KT; ++x) {
              f32x16_t y[NY];
              scores(x, half, q, y);
#pragma unroll
              for (int v = 0; v < 16; ++v) {
                const float p = weight(x, y, off, v);
                w[x][v] += 32 * x + 8 * (v / 4) + v % 4 < lim ? p : 0.f;
              }
            }
          }
        }
        if (!loaded) { wait_vmcnt<0>(); lds_barrier(); }
      }
      loaded = stages <= STAGES;
    }
    // Over the 32 rows that the lanes hold: at every step a lane passes on half of its keys, and is left with one of the 16.  (Lanes 16, 8, then 7 and
    // 2 numbers apart by exclusive or, without a way through LDS.)
#pragma unroll
    for (int x = 0; x < KT; ++x) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(w[x][i]), __float_as_uint(w[x][i + 8]), false, false);
        w[x][i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
      }
      halve<0x128, 8, 4>(w[x], lane);
      halve<0x141, 4, 2>(w[x], lane);
      halve<0x4E, 2, 1>(w[x], lane);
      w[x][0] += of_lane<0xB1>(w[x][0]);
      const int at = key0 + 32 * x + mine;
      if ((c & 1) || at >= most) continue;
      const long long to = ((long long)b * m.Hkv + hk) * most + at;
      const float sum = named[x] >> mine & 1 ? w[x][0] : 0.f;
      if (a.nsplit > 1) a.part[(long long)share * m.B * m.Hkv * most + to] = sum;
      else a.out[to] = at >= s.n ? 0.f : a.w ? fmaf(a.decay, stage0 < stages ? before[x] : a.w[to], sum) : sum;
    }
  }
}

// The sums of shares of the rows, in order.
__global__ __launch_bounds__(256) void weights_join(WeightsArgs a) {
  const BlockDims& m = a.m;
  const int most = m.max_pages << m.lpage;
  const long long all = (long long)m.B * m.Hkv * most, to = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (to >= all) return;
  const int at = (int)(to % most), n = min(max(m.seq_lens[to / most / m.Hkv], 0), most);
  f32x4_t sum = *(const f32x4_t*)(a.part + to);
  for (int z = 1; z < a.nsplit; ++z) sum += *(const f32x4_t*)(a.part + z * all + to);
  const f32x4_t before = a.w && at < n ? *(const f32x4_t*)(a.w + to) : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < 4; ++j) sum[j] = at + j < n ? (a.w ? fmaf(a.decay, before[j], sum[j]) : sum[j]) : 0.f;
  *(f32x4_t*)(a.out + to) = sum;
}

// Whether 32 bits hold every offset (in bytes, from a stage's first token) of the kernel for many rows: the stage's first row may be any head of
// its token, so its 64 rows reach (G + 62) / G tokens further, and any of the G heads.
bool near(const KeyStride& qs, int G, int d) {
  if (qs.token >= (1 << 24) || qs.head >= (1 << 24)) return false;
  return 2 * ((long long)((G + STAGE_ROWS - 2) / G) * qs.token + (long long)(G - 1) * qs.head + d) <= 1ll << 32;
}
struct WeightsShape { bool wide; int chunks, items, nsplit; size_t sums, part; };      // items: workgroups that share a head's chunks of keys
WeightsShape weights_shape(int dtype, int bits, int d, const BlockDims& m, const KeyStride& qs) {
  WeightsShape s{};
  const long long rows = (long long)m.max_q * m.G, keys = (long long)m.max_pages << m.lpage;
  // (8 heads of keys, 8 sequences up to 16 384, d = 128, few against many: 32 rows 61 and 62 us, 40 rows 72 and 67, 64 rows 82 and 67; 4 bits: 32 rows 46 and
  // 63, 48 rows 56 and 64, 64 rows 69 and 67, 96 rows 92 and 81)
  s.wide = dtype == ADACLUSTER_BF16 && rows > (bits ? 48 : 32) && near(qs, m.G, d);
  s.nsplit = 1;
  if (!s.wide) return s;
  const int chunk = 128 * key_tiles(bits, d);
  s.chunks = (int)((keys + chunk - 1) / chunk);
  // Few keys for many rows: the rows are shared until the launch has the two workgroups a CU that it holds, 512 rows each at least.
  const long long wg = (long long)s.chunks * m.Hkv * m.B;
  long long n = 512 / wg;
  if (n > rows / 512) n = rows / 512;
  if (n > 1) s.nsplit = (int)n;
  // (one sequence of 2 048 tokens over as many keys, d = 128: 176 us by one share, 48 and 5 for their sum by eight)
  // Where the rows stay in LDS a workgroup takes several chunks of keys, four workgroups a CU in all (32 and 64 tokens of 8 sequences up to 16 384, 16
  // bits: 68 and 96 us; two a CU 74 and 93, three 72 and 107; of 2 sequences up to 32 768 46 and 59; 43 and 52, 49 and 65).
  s.items = s.chunks;
  if (rows <= STAGES * STAGE_ROWS) {
    const long long most = (1024 + (long long)m.Hkv * m.B - 1) / ((long long)m.Hkv * m.B);
    if (most < s.items) s.items = (int)most;
  }
  s.sums = bits ? align_up((size_t)m.q_rows * m.Hq * 32, 256) : 0;
  s.part = s.nsplit > 1 ? (size_t)s.nsplit * m.B * m.Hkv * keys * 4 : 0;
  return s;
}
}  // namespace

size_t cache_weights_bytes(int dtype, int bits, int d, const BlockDims& m, const KeyStride& qs) {
  const WeightsShape s = weights_shape(dtype, bits, d, m, qs);
  return s.sums + s.part;
}

int launch_cache_weights(hipStream_t s, int dtype, int bits, int d, WeightsArgs a, void* ws) {
  const WeightsShape sh = weights_shape(dtype, bits, d, a.m, a.qs);
  if (sh.wide) {
    const long long heads = (long long)a.m.Hkv * a.m.B, grid = xcd_grid(heads, (long long)sh.items * sh.nsplit);
    const long long pre = ((long long)a.m.q_rows * a.m.Hq + 63) / 64;      // of weights_sums (4 bits)
    if (!grid_fits(grid) || (bits && !grid_fits(pre))) return ADACLUSTER_E_UNSUPPORTED;
    a.sums = (const u32x4_t*)ws;
    a.part = (float*)((char*)ws + sh.sums);
    a.nsplit = sh.nsplit;
    const int split = xcd_split(heads);
    if (bits) {
      if (d == 64) weights_sums<64><<<(int)pre, 256, 0, s>>>(a, (u32x4_t*)ws); else weights_sums<128><<<(int)pre, 256, 0, s>>>(a, (u32x4_t*)ws);
      if (int rc = launched()) return rc;
      if (d == 64) cache_weights_wide<4, 64><<<(int)grid, 256, 0, s>>>(a, sh.chunks, sh.items, split);
      else cache_weights_wide<4, 128><<<(int)grid, 256, 0, s>>>(a, sh.chunks, sh.items, split);
    } else {
      if (d == 64) cache_weights_wide<0, 64><<<(int)grid, 256, 0, s>>>(a, sh.chunks, sh.items, split);
      else cache_weights_wide<0, 128><<<(int)grid, 256, 0, s>>>(a, sh.chunks, sh.items, split);
    }
    if (int rc = launched()) return rc;
    if (sh.nsplit > 1) weights_join<<<(int)((heads * ((long long)a.m.max_pages << a.m.lpage) / 4 + 255) / 256), 256, 0, s>>>(a);
    return launched();
  }
  // four workgroups a CU in all, which take a head's keys in turns (one token of 32 sequences up to 16 384: two a CU take 1.19 of the time, eight as long)
  const int chunk = 64 * KEY_TILES, chunks = (int)((((long long)a.m.max_pages << a.m.lpage) + chunk - 1) / chunk);
  const long long heads = (long long)a.m.Hkv * a.m.B, most = (1024 + heads - 1) / heads;
  const int items = (int)(most < chunks ? most : chunks);
  const long long wg = heads * items;
  if (!grid_fits(wg)) return ADACLUSTER_E_UNSUPPORTED;
#define CALL(T, D) if (bits == 4) cache_weights<T, 4, D><<<(int)wg, 256, 0, s>>>(a, chunks, items); else cache_weights<T, 0, D><<<(int)wg, 256, 0, s>>>(a, chunks, items)
  if (dtype == ADACLUSTER_BF16) { if (d == 64) { CALL(bf16raw, 64); } else { CALL(bf16raw, 128); } }
  else { if (d == 64) { CALL(float, 64); } else { CALL(float, 128); } }
#undef CALL
  return launched();
}

}  // namespace adac
