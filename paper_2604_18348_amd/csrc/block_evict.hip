// The tokens that a sequence keeps of its cache, by the weights of its keys, and their move to other pages.
#include "block.h"

namespace adac {

namespace {

// Order of weights as whole numbers: the two zeros the same, a NaN behind everything; 0 is left for what is not there, the largest for a
// token that stays whatever it weighs.
constexpr uint32_t KEY_NAN = 1, KEY_MUST = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t u = __float_as_uint(w + 0.f);
  return w != w ? KEY_NAN : u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
// ... and back
__device__ __forceinline__ float weight_of(uint32_t key) {
  return __uint_as_float(key == KEY_NAN ? 0x7FC00000u : key >> 31 ? key & 0x7FFFFFFFu : ~key);
}
// The sum over the lanes up to this one.
__device__ __forceinline__ uint32_t scan64(uint32_t v) {
  const auto add = [&](auto ctrl, auto rows) __attribute__((always_inline)) {
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
  };
  using std::integral_constant;
  add(integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});      // 1, 2, 4, 8 lanes below in a row of 16
  add(integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});
  add(integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});
  add(integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});
  add(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});      // the last of rows 0 and 2 to the next
  add(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});      // lane 31 to the upper half
  return v;
}

constexpr int DIGIT = 11, BINS = 1 << DIGIT, COPIES = 4, FOURS = 8;
constexpr int NT = 1024, SEGMENT = NT * 4 * FOURS;     // positions that a workgroup holds at a time

// A workgroup chooses for one head of a sequence: the weight at the border by a radix search (three digits of 11, 11 and 10 bits from the
// top), then the positions that stay are numbered: those above it, those at it as long as there is room, and the ones that stay whatever
// they weigh.  Weights are read once, into registers, up to 32 768 positions (else once a digit).  Bound by its chain of steps: loads,
// counts in LDS and barriers, one workgroup a head: 128 heads of 32 768 positions 27 us (56 with one
// count a bin, weights read anew for every digit and branches for the protected ones), of 8 192 13 (17 with four waves), of 1 100 10.5.
__global__ __launch_bounds__(NT) void evict_pick(EvictArgs a) {
  constexpr int WAVES = NT / 64, PER = BINS / NT, COUNTS = FOURS * WAVES;
  // Counts in four copies, a quarter of the lanes each (weights of one size meet in few bins), and a bin a lane for what is not counted:
  // no branch then.
  constexpr int COPY = BINS + 16;                       // (the copies of a bin lie in different banks)
  __shared__ __align__(16) uint32_t bins[COPIES * COPY + 64];
  __shared__ uint32_t sums[COUNTS];
  __shared__ uint32_t found[2];
  const BlockDims& m = a.m;
  const int hk = blockIdx.x % m.Hkv, b = blockIdx.x / m.Hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int most = m.max_pages << m.lpage, n = min(max(m.seq_lens[b], 0), most), keep = a.keep;
  const long long at = (long long)b * m.Hkv + hk;
  const float* const w = a.w + at * most;
  float* const out = a.new_w + at * most;
  int32_t* const kept = a.kept + at * keep;
  const int end = min(n, keep);
  // (stay whatever they weigh: positions below `first` and from `last` on)
  const int first = (int)min((long long)n, (long long)m.keep_first << m.lpage), last = max(first, n - a.recent);
  uint32_t key[FOURS][4];                              // of positions seg * SEGMENT + 4 (i NT + tid) ..
  int fours = 0;                                       // of them that hold any
  const auto load = [&](int seg) __attribute__((always_inline)) {
    f32x4_t v[FOURS];
    const int left = n - seg * SEGMENT;
    fours = min(FOURS, (left + 4 * NT - 1) / (4 * NT));
#pragma unroll
    for (int i = 0; i < FOURS; ++i) {
      const int p = 4 * (i * NT + tid);
      v[i] = p < left ? *(const f32x4_t*)(w + seg * SEGMENT + p) : f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int i = 0; i < FOURS; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int p = seg * SEGMENT + 4 * (i * NT + tid) + j;
        key[i][j] = p >= n ? 0 : p < first || p >= last ? KEY_MUST : order_of(v[i][j]);
      }
  };
  const int segments = (n + SEGMENT - 1) / SEGMENT;
  if (n) load(0);
  if (hk == 0 && tid == 0) a.new_lens[b] = end;
  for (int p = end + tid; p < keep; p += NT) kept[p] = -1;
  const int whole = min(most, (end + 3) & ~3);
  if (tid < whole - end) out[end + tid] = 0.f;
  for (long long p = whole + 4 * tid; p < most; p += 4 * NT) *(f32x4_t*)(out + p) = f32x4_t{0.f, 0.f, 0.f, 0.f};
  uint32_t border = 0, room = 0;                        // what is above the border stays, and the first `room` at it
  if (n > keep) {
    room = keep;
    uint32_t mask = 0;
    for (int x = tid; x < COPIES * COPY / 4; x += NT) ((u32x4_t*)bins)[x] = u32x4_t{0, 0, 0, 0};
    __syncthreads();
    for (int digit = 0; digit < 3; ++digit) {
      const int shift = digit == 0 ? 32 - DIGIT : digit == 1 ? 32 - 2 * DIGIT : 0;
      const uint32_t low = digit == 2 ? (1u << (32 - 2 * DIGIT)) - 1 : BINS - 1;
      for (int seg = 0; seg < segments; ++seg) {
        if (segments > 1) load(seg);
#pragma unroll
        for (int i = 0; i < FOURS; ++i) {
          if (i >= fours) break;
#pragma unroll
          for (int j = 0; j < 4; ++j)                   // (what is not there counts as the least)
            atomicAdd(&bins[(key[i][j] & mask) == border ? (lane & (COPIES - 1)) * COPY + (key[i][j] >> shift & low) : COPIES * COPY + lane], 1u);
        }
      }
      __syncthreads();
      // the digit at the border: from the largest down, PER bins a thread, which it clears for the next digit
      const int hi = BINS - 1 - PER * tid;
      uint32_t c[PER], mine = 0;
#pragma unroll
      for (int y = 0; y < PER; ++y) c[y] = 0;
#pragma unroll
      for (int x = 0; x < COPIES; ++x)
#pragma unroll
        for (int y = 0; y < PER; y += 2) {
          uint2* const bin = (uint2*)&bins[x * COPY + hi - y - 1];
          c[y] += bin->y; c[y + 1] += bin->x;
          *bin = uint2{0, 0};
        }
#pragma unroll
      for (int y = 0; y < PER; ++y) mine += c[y];
      const uint32_t run = scan64(mine);
      if (lane == 63) sums[wave] = run;
      __syncthreads();
      uint32_t before = run - mine;
#pragma unroll
      for (int x = 0; x < WAVES; ++x) if (x < wave) before += sums[x];
#pragma unroll
      for (int y = 0; y < PER; ++y) {
        if (before < room && before + c[y] >= room) { found[0] = hi - y; found[1] = room - before; }
        before += c[y];
      }
      __syncthreads();
      border |= found[0] << shift;
      room = found[1];
      mask |= low << shift;
    }
    if (segments > 1) load(0);
  }
  // Numbers, in the order of the positions: of every four by ballots inside a wave, of the waves by a sum over their counts; those above the
  // border in the lower half of a word, those at it in the upper (32 768 fit).
  const uint64_t below = (1ull << lane) - 1;
  uint32_t done = 0, ties = 0;
  for (int seg = 0; seg < segments; ++seg) {
    if (seg) load(seg);
    uint32_t rank[FOURS];
#pragma unroll
    for (int i = 0; i < FOURS; ++i) {
      uint32_t before = 0, all = 0;
      if (i < fours) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint64_t x = __ballot(key[i][j] > border), y = __ballot(key[i][j] == border);
          before += __popcll(x & below) + (__popcll(y & below) << 16);
          all += __popcll(x) + (__popcll(y) << 16);
        }
      }
      rank[i] = before;
      if (lane == 0) sums[i * WAVES + wave] = all;
    }
    __syncthreads();
    if (wave == 0) {
      constexpr int EACH = COUNTS / 64;
      uint32_t c[EACH], mine = 0;
#pragma unroll
      for (int y = 0; y < EACH; ++y) { c[y] = sums[EACH * lane + y]; mine += c[y]; }
      const uint32_t run = scan64(mine);
      uint32_t before = run - mine;
#pragma unroll
      for (int y = 0; y < EACH; ++y) { sums[EACH * lane + y] = before; before += c[y]; }
      if (lane == 63) found[0] = run;
    }
    __syncthreads();
    const uint32_t all = found[0], fits = min(all >> 16, room - min(ties, room));
#pragma unroll
    for (int i = 0; i < FOURS; ++i) {
      if (i >= fours) break;
      const uint32_t x = rank[i] + sums[i * WAVES + wave];
      uint32_t s = x & 0xFFFF, t = x >> 16;             // above the border and at it, before, in this segment
      const int p = seg * SEGMENT + 4 * (i * NT + tid);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool above = key[i][j] > border, tie = key[i][j] == border;
        if (above || (tie && t < fits)) {
          const uint32_t to = done + s + min(t, fits);
          kept[to] = p + j;
          out[to] = key[i][j] == KEY_MUST ? w[p + j] + 0.f : weight_of(key[i][j]);
        }
        s += above;
        t += tie;
      }
    }
    done += (all & 0xFFFF) + fits;
    ties += all >> 16;
    __syncthreads();
  }
}

// A workgroup fills one page of one head: rows as they are, 16 bytes a lane (4 bits: codes), and the page's box of them.  Bound by memory: rows of 256
// bytes from anywhere, read and written: 16 x 8 heads x 4 096 rows of d = 128 115 us, 4.7 TB/s (118 with four on their way a lane); 4 bits, 32 x 8
// heads x 2 001 rows of 64 bytes and 8 of steps, each out of a line of 128, 70 us with four on their way, 72 with one.
template <typename T, int BITS, int D>
__global__ __launch_bounds__(256) void evict_move(EvictArgs a, int pages) {
  constexpr int VEC = Vec<T>::N, LPR = D / VEC;         // lanes a row
  const int RPI = blockDim.x / LPR;                     // rows a turn
  const BlockDims& m = a.m;
  const int pg = blockIdx.x % pages, hk = blockIdx.x / pages % m.Hkv, b = blockIdx.x / pages / m.Hkv;
  const int most = m.max_pages << m.lpage, n = min(min(max(m.seq_lens[b], 0), most), a.keep);
  const int p0 = pg << m.lpage, p1 = min(n, p0 + m.page);
  if (p0 >= p1) return;
  const int to = a.new_table[(long long)b * m.max_pages + pg];
  if ((unsigned)to >= (unsigned)m.num_pages) return;
  const int tid = threadIdx.x, col = tid % LPR * VEC;
  const int32_t* const kept = a.kept + ((long long)b * m.Hkv + hk) * a.keep;
  const int last = kept[p1 - 1], here = m.table[(long long)b * m.max_pages + pg];
  const bool stays = m.seq_lens[b] <= a.keep;
  if (last == p1 - 1 && to == here && (p1 - p0 == m.page || stays)) return;      // a page that stays as it is, in its place
  float mx[VEC], mn[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) { mx[i] = -INFINITY; mn[i] = INFINITY; }
  constexpr int U = BITS == 4 ? 4 : 1;                  // rows on their way
  for (int q0 = p0 + tid / LPR; q0 < p1; q0 += U * RPI) {
    int src[U], from[U];
#pragma unroll
    for (int u = 0; u < U; ++u) src[u] = q0 + u * RPI < p1 ? kept[q0 + u * RPI] : -1;
#pragma unroll
    for (int u = 0; u < U; ++u) from[u] = src[u] >= 0 ? pool_page(m, b, src[u] >> m.lpage) : -1;
    if constexpr (BITS == 4) {
      uint32_t kc[U], vc[U], kp[U], vp[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        kc[u] = vc[u] = kp[u] = vp[u] = 0;
        if (from[u] < 0) continue;
        const long long x = ((long long)from[u] * m.Hkv + hk) * m.page + (src[u] & (m.page - 1));
        kp[u] = a.km[x * (D / 64) + col / 64]; vp[u] = a.vm[x * (D / 64) + col / 64];
        if constexpr (VEC == 8) { kc[u] = ((const uint32_t*)a.kp)[x * (D / 8) + col / 8]; vc[u] = ((const uint32_t*)a.vp)[x * (D / 8) + col / 8]; }
        else { kc[u] = ((const uint16_t*)a.kp)[x * (D / 4) + col / 4]; vc[u] = ((const uint16_t*)a.vp)[x * (D / 4) + col / 4]; }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (src[u] < 0) continue;
        const long long y = ((long long)to * m.Hkv + hk) * m.page + ((q0 + u * RPI) & (m.page - 1));
        if constexpr (VEC == 8) { ((uint32_t*)a.kp)[y * (D / 8) + col / 8] = kc[u]; ((uint32_t*)a.vp)[y * (D / 8) + col / 8] = vc[u]; }
        else { ((uint16_t*)a.kp)[y * (D / 4) + col / 4] = (uint16_t)kc[u]; ((uint16_t*)a.vp)[y * (D / 4) + col / 4] = (uint16_t)vc[u]; }
        if (col % 64 == 0) { a.km[y * (D / 64) + col / 64] = kp[u]; a.vm[y * (D / 64) + col / 64] = vp[u]; }
        const float step = __uint_as_float(kp[u] << 16), low = __uint_as_float(kp[u] & 0xFFFF0000u);
#pragma unroll
        for (int i = 0; i < VEC; ++i) { const float x = fmaf((float)(kc[u] >> (4 * i) & 15), step, low); mx[i] = fmaxf(mx[i], x); mn[i] = fminf(mn[i], x); }
      }
    } else {
      u32x4_t kw[U], vw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        kw[u] = vw[u] = u32x4_t{0, 0, 0, 0};
        if (from[u] < 0) continue;
        const int in = src[u] & (m.page - 1);
        kw[u] = *(const u32x4_t*)((const T*)a.kp + from[u] * a.ks.page + in * a.ks.token + hk * a.ks.head + col);
        vw[u] = *(const u32x4_t*)((const T*)a.vp + from[u] * a.vs.page + in * a.vs.token + hk * a.vs.head + col);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (src[u] < 0) continue;
        const int slot = (q0 + u * RPI) & (m.page - 1);
        *(u32x4_t*)((T*)a.kp + to * a.ks.page + slot * a.ks.token + hk * a.ks.head + col) = kw[u];
        *(u32x4_t*)((T*)a.vp + to * a.vs.page + slot * a.vs.token + hk * a.vs.head + col) = vw[u];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float x = sizeof(T) == 2 ? __uint_as_float(i & 1 ? kw[u][i / 2] & 0xFFFF0000u : kw[u][i / 2] << 16) : __uint_as_float(kw[u][i % 4]);
          mx[i] = fmaxf(mx[i], x); mn[i] = fminf(mn[i], x);
        }
      }
    }
  }
  __shared__ float s_mx[256 * VEC], s_mn[256 * VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) { s_mx[tid * VEC + i] = mx[i]; s_mn[tid * VEC + i] = mn[i]; }
  __syncthreads();
  T* const box = (T*)a.boxes + ((long long)to * m.Hkv + hk) * 2 * D;
  for (int c = tid; c < D; c += blockDim.x) {
    float x = s_mx[c], y = s_mn[c];
    for (int r = 1; r < RPI; ++r) { x = fmaxf(x, s_mx[r * D + c]); y = fminf(y, s_mn[r * D + c]); }
    if constexpr (sizeof(T) == 2) {
      const uint32_t z = pack_bf16x2(x, y);             // (codes: values that bfloat16 rounds, as adacluster_cache_read does)
      box[c] = (T)(z & 0xFFFFu); box[D + c] = (T)(z >> 16);
    } else { box[c] = x; box[D + c] = y; }
  }
}

}  // namespace

int launch_cache_evict(hipStream_t s, int dtype, int bits, int d, const EvictArgs& a) {
  const int all = (a.keep + a.m.page - 1) >> a.m.lpage, pages = all < a.m.max_pages ? all : a.m.max_pages;
  const long long wg = (long long)pages * a.m.Hkv * a.m.B;
  if (!grid_fits(wg) || !grid_fits(4ll * a.m.Hkv * a.m.B)) return ADACLUSTER_E_UNSUPPORTED;
  evict_pick<<<a.m.B * a.m.Hkv, NT, 0, s>>>(a);
  if (int rc = launched()) return rc;
  const int lanes = a.m.page * d / (dtype == ADACLUSTER_BF16 ? 8 : 4), nt = lanes < 256 ? lanes : 256;      // (128 for the smallest page)
#define CALL(T, D) if (bits == 4) evict_move<T, 4, D><<<(int)wg, nt, 0, s>>>(a, pages); else evict_move<T, 0, D><<<(int)wg, nt, 0, s>>>(a, pages)
  if (dtype == ADACLUSTER_BF16) { if (d == 64) { CALL(bf16raw, 64); } else { CALL(bf16raw, 128); } }
  else { if (d == 64) { CALL(float, 64); } else { CALL(float, 128); } }
#undef CALL
  return launched();
}

}  // namespace adac
