// Gradients of attention over listed pages of packed keys.  With P = softmax(scale Q K^T) over what a row sees,
//   dV = P^T dO,  dP = dO V^T,  dS = P (dP - rowsum(dO O)),  dQ = scale dS K,  dK = scale dS^T Q,
// dK and dV summed over the query heads that share the keys.  P is formed again from the scores and the row's logarithm of its sum.
// Two kernels, so that no sum is made with atomics: one goes over a block's list of keys for dQ, one over the blocks of queries that
// list a page for dK and dV (bit masks, set beforehand from the lists; the order of a sum is the order of the bits).
//
// In 16 bits P and dS are rounded to bfloat16 for their products, by half a step each: the other operands are bfloat16 too, and parts that
// kept more would double products that the matrix cores already spend a third of the time on.  Sums, P, dP and dS themselves are fp32.
#include "block_wide.h"
#include "launch.h"

namespace adac {

namespace {

// rowsum(dO O) of every query and head, 16 bytes a lane
template <typename T, int D>
__global__ __launch_bounds__(256) void grad_delta(BlockGradArgs a) {
  constexpr int VEC = Vec<T>::N, LPR = D / VEC, RPI = 256 / LPR;
  const long long x = (long long)blockIdx.x * RPI + threadIdx.x / LPR;
  if (x >= (long long)a.m.q_rows * a.m.Hq) return;
  const int t = (int)(x / a.m.Hq), h = (int)(x % a.m.Hq), col = threadIdx.x % LPR * VEC;
  const T* const o = (const T*)a.o + t * a.os.token + h * a.os.head + col;
  const T* const g = (const T*)a.d_o + t * a.dos.token + h * a.dos.head + col;
  float c = 0.f;
#pragma unroll
  for (int i = 0; i < VEC; ++i) c = fmaf(Elem<T>::load(o + i), Elem<T>::load(g + i), c);
#pragma unroll
  for (int w = 1; w < LPR; w <<= 1) c += __shfl_xor(c, w);
  if (col == 0) a.delta[x] = c;
}

__global__ __launch_bounds__(256) void grad_marks(BlockGradArgs a, long long entries) {
  const BlockDims& m = a.m;
  const long long x = (long long)blockIdx.x * 256 + threadIdx.x;
  if (x >= entries) return;
  const int e = (int)(x % m.topk);
  const long long rec = x / m.topk;
  const int hk = (int)(rec % m.Hkv), i = (int)(rec / m.Hkv % m.nb), b = (int)(rec / m.Hkv / m.nb);
  const BlockSeq s = block_seq(m, b);
  if (i * m.qblock >= s.nq) return;
  const int pg = list_page(a.sel + rec * m.topk, e, (s.n + m.page - 1) >> m.lpage);
  if (pg >= 0) atomicOr(&a.marks[(((long long)b * m.Hkv + hk) * m.max_pages + pg) * a.words + (i >> 5)], 1u << (i & 31));
}

// dQ: the walk of block_attn.  S^T = K Q^T and dP^T = V dO^T leave a lane one query and four keys, so dS^T is the operand of
// dQ^T = K^T dS^T as it stands; the keys' columns come out of LDS.
//
// In 16 bits rowsum(dO O) comes from a rounded O.  Its error e turns dS into dS - e P, whose rows no longer sum to 0, and a part of K
// that all keys share then shows in dQ.  The row sums of dS are that error, so sum P K is kept beside dQ and dQ - rowsum(dS) sum P K
// formed at the end, with the sums of dS as the product took it (against 64 bits, 17 776 keys, d=64: dQ 0.0047 off without, 0.0024 with
// it); the sums of the unrounded dS correct what goes on to grad_kv.
template <typename T, int D, int R>
__global__ __launch_bounds__(256) void grad_q(BlockGradArgs a, int rts) {
  constexpr int ND = D / 16;
  constexpr bool FIX = sizeof(T) == 2;
  constexpr int KBYTES = 32 * D * sizeof(T), JBYTES = (FIX ? 2 : 1) * 4 * 16 * D * 4 + 8 * 16 * 4;
  __shared__ __align__(16) char lds[4 * KBYTES > JBYTES ? 4 * KBYTES : JBYTES];
  const BlockDims& m = a.m;
  int id = blockIdx.x;
  const int rt = id % rts; id /= rts;
  const int i = id % m.nb; id /= m.nb;
  const int hk = id % m.Hkv, b = id / m.Hkv;
  const BlockSeq s = block_seq(m, b);
  const int t0 = i * m.qblock, rows = min(m.qblock, s.nq - t0) * m.G, base_row = rt * R * 16;
  if (t0 >= s.nq || base_row >= rows) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, quarter = lane >> 4;
  RowFrag<T, D> q[R], g[R];
  int lim[R];
  float lse[R], delta[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = base_row + r * 16 + n16, t = t0 + row / m.G, head = hk * m.G + row % m.G;
    const bool there = row < rows;
    lim[r] = there ? (m.causal ? min(s.n, s.first + t + 1) : s.n) : 0;
    load_frag(q[r], (const T*)a.q + (long long)(s.q0 + t) * a.qs.token + (long long)head * a.qs.head, quarter, there);
    load_frag(g[r], (const T*)a.d_o + (long long)(s.q0 + t) * a.dos.token + (long long)head * a.dos.head, quarter, there);
    const long long x = (long long)(s.q0 + t) * m.Hq + head;
    const float l = there ? a.lse[x] : -INFINITY;
    lse[r] = l == -INFINITY ? INFINITY : l * LOG2E;             // a row that sees nothing: all weights 0
    delta[r] = there ? a.delta[x] : 0.f;
  }
  const int last = min(base_row + R * 16, rows) - 1;
  const int maxlim = m.causal ? min(s.n, s.first + t0 + last / m.G + 1) : s.n;
  const int pages = maxlim > 0 ? (maxlim + m.page - 1) >> m.lpage : 0;
  const int32_t* const list = a.sel ? a.sel + (((long long)b * m.nb + i) * m.Hkv + hk) * m.topk : nullptr;
  const int lsub = m.lpage - 4, halves = (list ? m.topk : pages) << lsub, turns = (halves + 1) >> 1;
  f32x4_t acc[R][ND], pk[FIX ? R : 1][FIX ? ND : 1];
  float off[R], exact[R];                            // sums of dS, rounded and not
#pragma unroll
  for (int r = 0; r < R; ++r) {
    off[r] = exact[r] = 0.f;
#pragma unroll
    for (int x = 0; x < ND; ++x) {
      acc[r][x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      if constexpr (FIX) pk[r][x] = acc[r][x];
    }
  }
  char* const kl = lds + wave * KBYTES;
  for (int turn = wave; turn < turns; turn += 4) {
    int key0[2];
    RowFrag<T, D> k[2], v[2];
    bool any = false;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int half = 2 * turn + h, e = half >> lsub, sub = half & ((1 << lsub) - 1);
      int pg = half < halves ? list_page(list, e, pages) : -1;
      key0[h] = pg < 0 ? INT32_MAX - 64 : (pg << m.lpage) + sub * 16;
      if (key0[h] >= maxlim) pg = -1;
      any = any || pg >= 0;
      const bool there = pg >= 0 && key0[h] + n16 < s.n;
      load_frag(k[h], (const T*)a.k + row_at(m, s, a.ks, 0, pg, sub, hk) + n16 * a.ks.token, quarter, there);
      load_frag(v[h], (const T*)a.v + row_at(m, s, a.vs, 0, pg, sub, hk) + n16 * a.vs.token, quarter, there);
      compiler_fence();
      store_frag(kl, 16 * h + n16, quarter, k[h]);
    }
    compiler_fence();
    if (!any) continue;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      f32x4_t p[2], ds[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4_t sc = dots(k[h], q[r]), dp = dots(v[h], g[r]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool sees = key0[h] + 4 * quarter + j < lim[r];
          const float w = __builtin_amdgcn_exp2f(fmaf(sc[j], a.scale_log2e, -lse[r]));
          p[h][j] = sees ? w : 0.f;
          ds[h][j] = sees ? w * (dp[j] - delta[r]) : 0.f;
          if constexpr (FIX) { off[r] += __uint_as_float((uint32_t)f32_to_bf16(ds[h][j]) << 16); exact[r] += ds[h][j]; }
        }
      }
#pragma unroll
      for (int x = 0; x < ND; ++x) {
        acc[r][x] = mma_cols<D>(T{}, kl, 16 * x, lane, ds[0], ds[1], acc[r][x]);
        if constexpr (FIX) pk[r][x] = mma_cols<D>(T{}, kl, 16 * x, lane, p[0], p[1], pk[r][x]);
      }
    }
    compiler_fence();
  }
  float* const jo = (float*)lds;
  float* const jp = jo + 4 * 16 * D;
  float* const js = FIX ? jp + 4 * 16 * D : jp;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    __syncthreads();
#pragma unroll
    for (int x = 0; x < ND; ++x) {
      *(f32x4_t*)(jo + (wave * 16 + n16) * D + 16 * x + 4 * quarter) = acc[r][x];
      if constexpr (FIX) *(f32x4_t*)(jp + (wave * 16 + n16) * D + 16 * x + 4 * quarter) = pk[r][x];
    }
    if constexpr (FIX) {
      const float e = quarters_sum(off[r]), x = quarters_sum(exact[r]);
      if (quarter == 0) { js[wave * 16 + n16] = e; js[64 + wave * 16 + n16] = x; }
    }
    __syncthreads();
    const int jr = tid >> 4, row = base_row + r * 16 + jr, d0 = (tid & 15) * (D / 16);
    if (row >= rows) continue;
    float e = 0.f;
    if constexpr (FIX) {
      e = js[jr] + js[16 + jr] + js[32 + jr] + js[48 + jr];
      if (d0 == 0) a.delta[(long long)(s.q0 + t0 + row / m.G) * m.Hq + hk * m.G + row % m.G] += js[64 + jr] + js[80 + jr] + js[96 + jr] + js[112 + jr];      // (its only reader and writer here)
    }
    T* const out = (T*)a.dq + (long long)(s.q0 + t0 + row / m.G) * a.dqs.token + (long long)(hk * m.G + row % m.G) * a.dqs.head + d0;
#pragma unroll
    for (int x = 0; x < D / 16; x += 4) {
      f32x4_t o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        o += *(const f32x4_t*)(jo + (w * 16 + jr) * D + d0 + x);
        if constexpr (FIX) o -= e * *(const f32x4_t*)(jp + (w * 16 + jr) * D + d0 + x);
      }
      o *= a.scale;
      if constexpr (sizeof(T) == 2) *(uint2*)(out + x) = uint2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
      else *(f32x4_t*)(out + x) = o;
    }
  }
}

// A page that far more blocks list than others (the first one, say) would be the launch's critical path.  Where a launch has few
// workgroups, the blocks of such a page are dealt to up to `np` workgroups, each a run of the page's marks; their sums go to
// memory and grad_kv_add (grad_kv_join) adds them in order.
struct Share { int first, count, parts; };
__device__ __forceinline__ Share page_share(const BlockGradArgs& a, const uint32_t* marks, int blocks, int part) {
  if (a.np == 1) return {0, blocks, 1};
  int n = 0;
  for (int w = 0; w * 32 < blocks; ++w) n += __popc((uint32_t)uniform((int)marks[w]));      // (no mark lies past the last block)
  const int parts = min(a.np, max(1, (n + a.limit - 1) / a.limit));
  const int first = (int)((long long)n * part / parts);
  return {first, (int)((long long)n * (part + 1) / parts) - first, parts};
}
// dK and dV of KR * 16 keys of one head: the waves take tiles of 32 rows in turns.  S = Q K^T and dP = dO V^T leave a lane one key
// and four rows: P and dS are the operands of dV^T = dO^T P and dK^T = Q^T dS as they stand.
template <typename T, int D, int KR>
__global__ __launch_bounds__(256) void grad_kv(BlockGradArgs a) {
  constexpr int ND = D / 16;
  constexpr int TBYTES = 32 * D * sizeof(T), JBYTES = 4 * 16 * D * 4;
  __shared__ __align__(16) char lds[8 * TBYTES > JBYTES ? 8 * TBYTES : JBYTES];
  const BlockDims& m = a.m;
  // (heads side by side, first pages first, shares behind the first last, as in grad_kv_pair)
  const int part = uniform((int)(blockIdx.x / (unsigned)a.wg)), group = uniform((int)(blockIdx.x % (unsigned)a.wg));
  const int hk = group % m.Hkv, b = group / m.Hkv % m.B, kg = group / m.Hkv / m.B;
  const BlockSeq s = block_seq(m, b);
  const int key0 = kg * KR * 16;
  if (key0 >= s.n) return;
  const uint32_t* const marks = a.sel ? a.marks + (((long long)b * m.Hkv + hk) * m.max_pages + (key0 >> m.lpage)) * a.words : nullptr;
  const int blocks = (s.nq + m.qblock - 1) / m.qblock;
  const Share share = page_share(a, marks, blocks, part);
  if (part >= share.parts) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, quarter = lane >> 4;
  RowFrag<T, D> k[KR], v[KR];
  f32x4_t dk[KR][ND], dv[KR][ND];
#pragma unroll
  for (int r = 0; r < KR; ++r) {
    const int key = key0 + r * 16 + n16;
    load_frag(k[r], (const T*)a.k + (s.k0 + (long long)key) * a.ks.token + hk * a.ks.head, quarter, key < s.n);
    load_frag(v[r], (const T*)a.v + (s.k0 + (long long)key) * a.vs.token + hk * a.vs.head, quarter, key < s.n);
#pragma unroll
    for (int x = 0; x < ND; ++x) dk[r][x] = dv[r][x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  char* const ql = lds + wave * 2 * TBYTES;
  char* const gl = ql + TBYTES;
  int skip = share.first, left = share.count;
  int unit = 0;
  for (int w = 0; w * 32 < blocks; ++w) {
    uint32_t bits = left ? marks ? marks[w] : ~0u : 0;
    if (blocks - w * 32 < 32) bits &= (1u << (blocks - w * 32)) - 1;
    while (bits) {
      const int i = w * 32 + __builtin_ctz(bits), t0 = i * m.qblock, rows = min(m.qblock, s.nq - t0) * m.G;
      bits &= bits - 1;
      if (skip) { --skip; continue; }
      if (!left) break;
      --left;
      for (int base = 0; base < rows; base += 32) {
        const int last = t0 + (min(base + 32, rows) - 1) / m.G;
        if (m.causal && s.first + last < key0) continue;
        if ((unit++ & 3) != wave) continue;
        RowFrag<T, D> q[2], g[2];
        int lim[2][4];
        float lse[2][4], delta[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = base + 16 * h + n16, t = t0 + row / m.G, head = hk * m.G + row % m.G;
          load_frag(q[h], (const T*)a.q + (long long)(s.q0 + t) * a.qs.token + (long long)head * a.qs.head, quarter, row < rows);
          load_frag(g[h], (const T*)a.d_o + (long long)(s.q0 + t) * a.dos.token + (long long)head * a.dos.head, quarter, row < rows);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int row = base + 16 * h + 4 * quarter + j, t = t0 + row / m.G;
            const bool there = row < rows;
            const long long x = (long long)(s.q0 + t) * m.Hq + hk * m.G + row % m.G;
            const float l = there ? a.lse[x] : -INFINITY;
            lim[h][j] = there ? (m.causal ? min(s.n, s.first + t + 1) : s.n) : 0;
            lse[h][j] = l == -INFINITY ? INFINITY : l * LOG2E;
            delta[h][j] = there ? a.delta[x] : 0.f;
          }
          compiler_fence();
          store_frag(ql, 16 * h + n16, quarter, q[h]);
          store_frag(gl, 16 * h + n16, quarter, g[h]);
        }
        compiler_fence();
#pragma unroll
        for (int r = 0; r < KR; ++r) {
          f32x4_t p[2], ds[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const f32x4_t sc = dots(q[h], k[r]), dp = dots(g[h], v[r]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const bool sees = key0 + 16 * r + n16 < lim[h][j];
              const float w = __builtin_amdgcn_exp2f(fmaf(sc[j], a.scale_log2e, -lse[h][j]));
              p[h][j] = sees ? w : 0.f;
              ds[h][j] = sees ? w * (dp[j] - delta[h][j]) : 0.f;
            }
          }
#pragma unroll
          for (int x = 0; x < ND; ++x) {
            dv[r][x] = mma_cols<D>(T{}, gl, 16 * x, lane, p[0], p[1], dv[r][x]);
            dk[r][x] = mma_cols<D>(T{}, ql, 16 * x, lane, ds[0], ds[1], dk[r][x]);
          }
        }
        compiler_fence();
      }
    }
  }
  float* const jo = (float*)lds;
#pragma unroll
  for (int r = 0; r < KR; ++r)
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      __syncthreads();
#pragma unroll
      for (int x = 0; x < ND; ++x) *(f32x4_t*)(jo + (wave * 16 + n16) * D + 16 * x + 4 * quarter) = side ? dv[r][x] : dk[r][x];
      __syncthreads();
      const int jr = tid >> 4, key = key0 + r * 16 + jr, d0 = (tid & 15) * (D / 16);
      if (share.parts > 1) {
        float* const to = a.sums + ((((long long)group * a.np + part) * 2 + side) * (16 * KR) + r * 16 + jr) * D + d0;
#pragma unroll
        for (int x = 0; x < D / 16; x += 4) {
          f32x4_t o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < 4; ++w) o += *(const f32x4_t*)(jo + (w * 16 + jr) * D + d0 + x);
          *(f32x4_t*)(to + x) = o;
        }
        continue;
      }
      if (key >= s.n) continue;
      T* const out = (side ? (T*)a.dv + (s.k0 + (long long)key) * a.dvs.token + hk * a.dvs.head
                           : (T*)a.dk + (s.k0 + (long long)key) * a.dks.token + hk * a.dks.head) + d0;
#pragma unroll
      for (int x = 0; x < D / 16; x += 4) {
        f32x4_t o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) o += *(const f32x4_t*)(jo + (w * 16 + jr) * D + d0 + x);
        if (!side) o *= a.scale;
        if constexpr (sizeof(T) == 2) *(uint2*)(out + x) = uint2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
        else *(f32x4_t*)(out + x) = o;
      }
    }
}

// The sums of 16 KR keys whose blocks were dealt to several workgroups.
template <typename T, int D, int KR>
__global__ __launch_bounds__(256) void grad_kv_add(BlockGradArgs a) {
  const BlockDims& m = a.m;
  const int group = blockIdx.x, hk = group % m.Hkv, b = group / m.Hkv % m.B, key0 = group / m.Hkv / m.B * KR * 16;
  const BlockSeq s = block_seq(m, b);
  if (key0 >= s.n) return;
  const uint32_t* const marks = a.marks + (((long long)b * m.Hkv + hk) * m.max_pages + (key0 >> m.lpage)) * a.words;
  const Share share = page_share(a, marks, (s.nq + m.qblock - 1) / m.qblock, 0);
  if (share.parts < 2) return;
  for (int x = threadIdx.x; x < 2 * KR * 16 * (D / 4); x += 256) {
    const int d0 = x % (D / 4) * 4, row = x / (D / 4) % (KR * 16), side = x / (D / 4) / (KR * 16), key = key0 + row;
    if (key >= s.n) continue;
    f32x4_t o{0.f, 0.f, 0.f, 0.f};
    for (int part = 0; part < share.parts; ++part)
      o += *(const f32x4_t*)(a.sums + ((((long long)group * a.np + part) * 2 + side) * (16 * KR) + row) * D + d0);
    if (!side) o *= a.scale;
    T* const out = (side ? (T*)a.dv + (s.k0 + (long long)key) * a.dvs.token + hk * a.dvs.head
                         : (T*)a.dk + (s.k0 + (long long)key) * a.dks.token + hk * a.dks.head) + d0;
    if constexpr (sizeof(T) == 2) *(uint2*)out = uint2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
    else *(f32x4_t*)out = o;
  }
}

// Where a wave of the kernels for many rows leaves its 64 values a lane.
__device__ __forceinline__ float* share_slot(const BlockGradArgs& a, int group, int part, int wave, int lane) {
  return a.sums + (((long long)group * a.np + part) * 4 + wave) * 4096 + lane;
}
template <int DB> __device__ __forceinline__ void store_rows(bf16raw* out, const f32x16_t* x, float f) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int y = 0; y < 4; ++y)
      *(uint2*)(out + db * 32 + 8 * y) = uint2{pack_bf16x2(x[db][4 * y] * f, x[db][4 * y + 1] * f), pack_bf16x2(x[db][4 * y + 2] * f, x[db][4 * y + 3] * f)};
}

// dQ of blocks of many rows, bf16: grad_q on tiles of 64 keys that all waves share (the walk of block_attn_wide), 32 rows a wave.
// Three waves a SIMD cost 26 spilled registers (grad_kv_wide<4> 8), none of them reloaded between products.
__global__ __launch_bounds__(256, 3) void grad_q_wide(BlockGradArgs a, int rts, int split) {
  constexpr int D = 64, NW = 4, NT = NW * 64, KS = D / 16, DB = D / 32, CH = D / 8, ROWB = D * 2;
  constexpr int PT = TILE * CH / NT, TILEB = TILE * ROWB;
  __shared__ __align__(16) char lds[4 * TILEB];
  __shared__ int2 pages_l[LIST];
  __shared__ int32_t counts[NW];
  const BlockDims& m = a.m;
  const HeadItem it = xcd_item(blockIdx.x, m.B * m.Hkv, m.nb * rts, split);
  if (it.head < 0) return;
  const int rt = it.item % rts, i = it.item / rts, hk = it.head % m.Hkv, b = it.head / m.Hkv;
  const BlockSeq s = block_seq(m, b);
  const int t0 = i * m.qblock, rows = min(m.qblock, s.nq - t0) * m.G, base_row = rt * NT / 2;
  if (t0 >= s.nq || base_row >= rows) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, hb = lane >> 5;
  const int row = base_row + wave * 32 + c, tok = t0 + row / m.G, head = hk * m.G + row % m.G;
  const bool there = row < rows;
  const long long rec = (long long)(s.q0 + tok) * m.Hq + head;
  bf16x8_t qf[KS], gf[KS];
  {
    const bf16raw* const q = (const bf16raw*)a.q + (long long)(s.q0 + tok) * a.qs.token + (long long)head * a.qs.head + hb * 8;
    const bf16raw* const g = (const bf16raw*)a.d_o + (long long)(s.q0 + tok) * a.dos.token + (long long)head * a.dos.head + hb * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4_t z = {0, 0, 0, 0}, x = there ? *(const u32x4_t*)(q + ks * 16) : z, y = there ? *(const u32x4_t*)(g + ks * 16) : z;
      qf[ks] = *(const bf16x8_t*)&x;
      gf[ks] = *(const bf16x8_t*)&y;
    }
  }
  const int lim = there ? (m.causal ? min(s.n, s.first + tok + 1) : s.n) : INT32_MAX;
  const float l = there ? a.lse[rec] : -INFINITY, lse = l == -INFINITY ? INFINITY : l * LOG2E, delta = there ? a.delta[rec] : 0.f;
  const bool wave_has_rows = base_row + wave * 32 < rows;
  const int minlim = m.causal ? min(s.n, s.first + t0 + (base_row + wave * 32) / m.G + 1) : s.n;
  const int last = min(base_row + NT / 2, rows) - 1;
  const int maxlim = m.causal ? min(s.n, s.first + t0 + last / m.G + 1) : s.n;
  const int pages = maxlim > 0 ? (maxlim + m.page - 1) >> m.lpage : 0;
  const int32_t* const list = a.sel ? a.sel + (((long long)b * m.nb + i) * m.Hkv + hk) * m.topk : nullptr;
  const int entries = list ? m.topk : pages;
  f32x16_t dq[DB], pk[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dq[db] = pk[db] = zero16();
  float off = 0.f, exact[2] = {0.f, 0.f};            // sums of dS, rounded and not
  const float sc = a.scale_log2e;

  int lrow[PT], piece[PT];
#pragma unroll
  for (int x = 0; x < PT; ++x) {
    const int item = tid + x * NT;
    lrow[x] = item / CH;
    piece[x] = ((item % CH) ^ swz<D>(lrow[x])) * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void_t*)lds;
  const int lsub = m.lpage - 4, ktok = (int)(a.ks.token * 2), vtok = (int)(a.vs.token * 2);
  int ra[KS], ca[DB][2];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) ra[ks] = row_operand<D>(lane, ks);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 2; ++x) ca[db][x] = col_operand<D>(lane, db, x);

  for (int e0 = 0; e0 < entries; e0 += LIST) {
    const int n = fill_list<NT>(m, b, list, e0, 1, entries, pages, pages_l, counts);
    const int parts = n << lsub, tiles = (parts + 3) >> 2;
    if (!tiles) continue;
    auto issue = [&](int stage, int t) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < PT; ++x) {
        const int part = min(t * 4 + (((wave * 64 + x * NT) / CH) >> 4), parts - 1);
        const int pg = __builtin_amdgcn_readfirstlane(pages_l[part >> lsub].x);
        int sub = part & ((1 << lsub) - 1), have = s.n - ((pg << m.lpage) + sub * 16);
        if (have <= 0) { sub = 0; have = 1; }
        const int r = min(lrow[x] & 15, have - 1);
        const uint32_t dst = lds0 + stage * 2 * TILEB + (wave * 64 + x * NT) * 16;
        dma_b128(dst, (uint32_t)(r * ktok + piece[x]), uniform((const char*)a.k + row_at(m, s, a.ks, 0, pg, sub, hk) * 2));
        dma_b128(dst + TILEB, (uint32_t)(r * vtok + piece[x]), uniform((const char*)a.v + row_at(m, s, a.vs, 0, pg, sub, hk) * 2));
      }
    };
    issue(0, 0);
    wait_vmcnt<0>();
    lds_barrier();
    for (int t = 0; t < tiles; ++t) {
      if (t + 1 < tiles) issue((t + 1) & 1, t + 1);
      if (wave_has_rows) {
        const char* const kt = lds + (t & 1) * 2 * TILEB;
        const char* const vt = kt + TILEB;
#pragma unroll 1
        for (int kb = 0; kb < 2; ++kb) {
          f32x16_t sa = zero16(), dp = zero16();
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            sa = mfma32(*(const bf16x8_t*)(kt + kb * 32 * ROWB + ra[ks]), qf[ks], sa);
            dp = mfma32(*(const bf16x8_t*)(vt + kb * 32 * ROWB + ra[ks]), gf[ks], dp);
          }
          bool whole = true;
          int key0[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int part = t * 4 + kb * 2 + x, pg = __builtin_amdgcn_readfirstlane(pages_l[min(part, parts - 1) >> lsub].x);
            key0[x] = part < parts ? (pg << m.lpage) + (part & ((1 << lsub) - 1)) * 16 : INT32_MAX - 64;
            whole = whole && key0[x] + 16 <= minlim;
          }
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            sa[v] = __builtin_amdgcn_exp2f(fmaf(sa[v], sc, -lse));
            dp[v] = sa[v] * (dp[v] - delta);
          }
          if (!whole) {
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (key0[v >> 3] + 8 * ((v >> 2) & 1) + 4 * hb + (v & 3) >= lim) sa[v] = dp[v] = 0.f;
          }
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2) {
            const bf16x8_t pf = pack8(sa, s2), df = pack8(dp, s2);
            off = sum8(df, off);
#pragma unroll
            for (int v = 0; v < 8; ++v) exact[v & 1] += dp[8 * s2 + v];
            const char* const p = kt + (kb * 32 + 16 * s2) * ROWB;
#pragma unroll
            for (int db = 0; db < DB; ++db) {
              const bf16x8_t kc = join_tr(read_tr(p + ca[db][0]), read_tr(p + ca[db][1]));
              dq[db] = mfma32(kc, df, dq[db]);
              pk[db] = mfma32(kc, pf, pk[db]);
            }
          }
        }
      }
      wait_vmcnt<0>();
      lds_barrier();
    }
  }
  if (!there) return;
  const float e = off + __shfl_xor(off, 32), x = exact[0] + exact[1], fix = x + __shfl_xor(x, 32);
  bf16raw* const out = (bf16raw*)a.dq + (long long)(s.q0 + tok) * a.dqs.token + (long long)head * a.dqs.head + 4 * hb;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
#pragma unroll
    for (int v = 0; v < 16; ++v) dq[db][v] = (dq[db][v] - e * pk[db][v]) * a.scale;
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *(uint2*)(out + db * 32 + 8 * x) = uint2{pack_bf16x2(dq[db][4 * x], dq[db][4 * x + 1]), pack_bf16x2(dq[db][4 * x + 2], dq[db][4 * x + 3])};
  }
  if (hb == 0) a.delta[rec] = delta + fix;             // (its only reader and writer in this launch)
}

// dK and dV of 32 KG keys (a page, or a part of one), bf16, from blocks of many rows: KG waves of 32 keys side by side, and 4 / KG groups of
// them that share the rows of a tile.  A tile's rows of Q and dO are staged once for all waves and read both as rows (S, dP) and as
// columns (dK, dV); the next tile is on its way meanwhile.
template <int KG>
__global__ __launch_bounds__(256, 3) void grad_kv_wide(BlockGradArgs a, int split) {
  constexpr int D = 64, RG = 4 / KG, TR = 64 * RG, KS = D / 16, DB = D / 32, CH = D / 8, ROWB = D * 2;
  constexpr int PT = TR * CH / 256, TILEB = TR * ROWB;
  __shared__ __align__(16) char lds[4 * TILEB];
  __shared__ __align__(16) float row_lse[2][TR], row_delta[2][TR];
  __shared__ __align__(16) int row_lim[2][TR];
  const BlockDims& m = a.m;
  // The first pages come first, those of all heads side by side: they are seen by most.  A head stays on the same XCDs (as in xcd_item).
  // Shares behind the first come last.
  const int heads = m.B * m.Hkv, units = heads * split, per = (a.groups + split - 1) / split * units;
  const int part = uniform((int)(blockIdx.x / (unsigned)per)), at = uniform((int)(blockIdx.x % (unsigned)per)), unit = at % units;
  const int head = unit / split, kg = at / units * split + unit % split, group = kg * heads + head, hk = head % m.Hkv, b = head / m.Hkv;
  if (kg >= a.groups) return;
  const BlockSeq s = block_seq(m, b);
  if (kg * KG * 32 >= s.n) return;
  const uint32_t* const marks = a.sel ? a.marks + (((long long)b * m.Hkv + hk) * m.max_pages + (kg * KG * 32 >> m.lpage)) * a.words : nullptr;
  const int blocks = (s.nq + m.qblock - 1) / m.qblock;
  const Share share = page_share(a, marks, blocks, part);
  if (part >= share.parts) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, hb = lane >> 5;
  const int rg = wave / KG, key0 = kg * KG * 32 + (wave % KG) * 32, key = key0 + c;
  bf16x8_t kf[KS], vf[KS];
  {
    const bf16raw* const k = (const bf16raw*)a.k + (s.k0 + (long long)key) * a.ks.token + hk * a.ks.head + hb * 8;
    const bf16raw* const v = (const bf16raw*)a.v + (s.k0 + (long long)key) * a.vs.token + hk * a.vs.head + hb * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4_t z = {0, 0, 0, 0}, x = key < s.n ? *(const u32x4_t*)(k + ks * 16) : z, y = key < s.n ? *(const u32x4_t*)(v + ks * 16) : z;
      kf[ks] = *(const bf16x8_t*)&x;
      vf[ks] = *(const bf16x8_t*)&y;
    }
  }
  f32x16_t dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[db] = dv[db] = zero16();
  const float sc = a.scale_log2e, inv_g = 1.f / m.G;

  int lrow[PT], piece[PT];
#pragma unroll
  for (int x = 0; x < PT; ++x) {
    const int item = tid + x * 256;
    lrow[x] = item / CH;
    piece[x] = ((item % CH) ^ swz<D>(lrow[x])) * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void_t*)lds;
  const int qtok = (int)(a.qs.token * 2), qhead = (int)(a.qs.head * 2), gtok = (int)(a.dos.token * 2), ghead = (int)(a.dos.head * 2);
  int ra[KS], ca[DB][2];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) ra[ks] = row_operand<D>(lane, ks);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 2; ++x) ca[db][x] = col_operand<D>(lane, db, x);

  // tiles of the blocks that list the page and are not all before its keys: block `i`, rows from `base`
  int word = -1, i = 0, base = 0, rows = 0, skip = share.first, left = share.count;
  uint32_t bits = 0;
  auto advance = [&]() __attribute__((always_inline)) {      // false: no tile is left
    base += TR;
    for (;;) {
      for (; base < rows; base += TR)
        if (!m.causal || s.first + i * m.qblock + (min(base + TR, rows) - 1) / m.G >= kg * KG * 32) return true;
      while (!bits) {
        if (++word * 32 >= blocks) return false;
        bits = marks ? (uint32_t)uniform((int)marks[word]) : ~0u;
        if (blocks - word * 32 < 32) bits &= (1u << (blocks - word * 32)) - 1;
      }
      if (!left) return false;
      i = word * 32 + __builtin_ctz(bits);
      bits &= bits - 1;
      if (skip) { --skip; continue; }
      --left;
      base = 0;
      rows = min(m.qblock, s.nq - i * m.qblock) * m.G;
    }
  };
  float nl = 0.f, nd = 0.f;
  int nlim = 0;
  auto issue = [&](int stage) __attribute__((always_inline)) {
    const int t0 = i * m.qblock;
    const char* const q = uniform((const char*)a.q + ((long long)(s.q0 + t0) * a.qs.token + (long long)(hk * m.G) * a.qs.head) * 2);
    const char* const g = uniform((const char*)a.d_o + ((long long)(s.q0 + t0) * a.dos.token + (long long)(hk * m.G) * a.dos.head) * 2);
#pragma unroll
    for (int x = 0; x < PT; ++x) {
      const int r = min(base + lrow[x], rows - 1), t = (int)((r + 0.5f) * inv_g), h = r - t * m.G;
      const uint32_t dst = lds0 + stage * 2 * TILEB + (wave * 64 + x * 256) * 16;
      dma_b128(dst, (uint32_t)(t * qtok + h * qhead + piece[x]), q);
      dma_b128(dst + TILEB, (uint32_t)(t * gtok + h * ghead + piece[x]), g);
    }
    if (tid < TR) {
      const int r = base + tid, t = (int)((r + 0.5f) * inv_g);
      const bool there = r < rows;
      const long long x = (long long)(s.q0 + t0 + t) * m.Hq + hk * m.G + (r - t * m.G);
      const float l = there ? a.lse[x] : -INFINITY;
      nl = l == -INFINITY ? INFINITY : l * LOG2E;
      nd = there ? a.delta[x] : 0.f;
      nlim = there ? (m.causal ? min(s.n, s.first + t0 + t + 1) : s.n) : 0;
    }
  };
  auto land = [&](int stage) __attribute__((always_inline)) {
    if (tid < TR) { row_lse[stage][tid] = nl; row_delta[stage][tid] = nd; row_lim[stage][tid] = nlim; }
    wait_vmcnt<0>();
    lds_barrier();
  };
  bool more = advance();
  if (more) { issue(0); land(0); }
  int u = 0;
  while (more) {
    // the keys a row of the tile misses at most: none where its first row sees them all and all of its rows are there
    const int first_lim = m.causal ? min(s.n, s.first + i * m.qblock + base / m.G + 1) : s.n;
    const bool whole = key0 + 32 <= first_lim && base + TR <= rows;
    more = advance();
    if (more) issue(u ^ 1);
    const char* const qt = lds + u * 2 * TILEB;
    const char* const gt = qt + TILEB;
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
      const int r0 = (rg * 2 + half) * 32;
      f32x16_t sa = zero16(), dp = zero16();
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        sa = mfma32(*(const bf16x8_t*)(qt + r0 * ROWB + ra[ks]), kf[ks], sa);
        dp = mfma32(*(const bf16x8_t*)(gt + r0 * ROWB + ra[ks]), vf[ks], dp);
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const f32x4_t l4 = *(const f32x4_t*)&row_lse[u][r0 + 8 * x + 4 * hb], d4 = *(const f32x4_t*)&row_delta[u][r0 + 8 * x + 4 * hb];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sa[4 * x + j] = __builtin_amdgcn_exp2f(fmaf(sa[4 * x + j], sc, -l4[j]));
          dp[4 * x + j] = sa[4 * x + j] * (dp[4 * x + j] - d4[j]);
        }
      }
      if (!whole) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (key >= row_lim[u][r0 + 8 * x + 4 * hb + j]) sa[4 * x + j] = dp[4 * x + j] = 0.f;
      }
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const bf16x8_t pf = pack8(sa, s2), df = pack8(dp, s2);
        const char* const qp = qt + (r0 + 16 * s2) * ROWB;
        const char* const gp = gt + (r0 + 16 * s2) * ROWB;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          dv[db] = mfma32(join_tr(read_tr(gp + ca[db][0]), read_tr(gp + ca[db][1])), pf, dv[db]);
          dk[db] = mfma32(join_tr(read_tr(qp + ca[db][0]), read_tr(qp + ca[db][1])), df, dk[db]);
        }
      }
    }
    if (more) land(u ^ 1);
    u ^= 1;
  }
  // the groups' sums joined through LDS, in order
  if constexpr (RG > 1) {
    float* const part = (float*)lds;
#pragma unroll
    for (int side = 0; side < 2; ++side)
      for (int g = 1; g < RG; ++g) {
        __syncthreads();
        if (rg == g) {
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) part[(((wave % KG) * DB + db) * 16 + v) * 64 + lane] = side ? dv[db][v] : dk[db][v];
        }
        __syncthreads();
        if (rg == 0) {
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const float x = part[(((wave % KG) * DB + db) * 16 + v) * 64 + lane];
              if (side) dv[db][v] += x; else dk[db][v] += x;
            }
        }
      }
    if (rg) return;
  }
  if (share.parts > 1) {
    float* const to = share_slot(a, group, part, wave, lane);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) { to[(db * 16 + v) * 64] = dk[db][v]; to[((DB + db) * 16 + v) * 64] = dv[db][v]; }
    return;
  }
  if (key >= s.n) return;
  store_rows<DB>((bf16raw*)a.dk + (s.k0 + (long long)key) * a.dks.token + hk * a.dks.head + 4 * hb, dk, a.scale);
  store_rows<DB>((bf16raw*)a.dv + (s.k0 + (long long)key) * a.dvs.token + hk * a.dvs.head + 4 * hb, dv, 1.f);
}

// The same at d = 128, where a wave of 32 rows would hold 346 registers and a SIMD one wave.  Two waves share 32 rows: each forms the weights
// and dS of 32 of a tile's 64 keys, passes the one that it does not need itself through LDS as the operand it is, and sums one of the two
// products, dS K or P K, over all 64.  Two waves a SIMD then, of two workgroups with barriers of their own.  3 sequences up to 8 192 tokens, 16 / 4 heads: 770 us, 1 033
// by the kernel for d = 64.
__global__ __launch_bounds__(256, 2) void grad_q_pair(BlockGradArgs a, int rts, int split) {
  constexpr int D = 128, NW = 4, NT = NW * 64, KS = D / 16, DB = D / 32, CH = D / 8, ROWB = D * 2;
  constexpr int PT = TILE * CH / NT, TILEB = TILE * ROWB;
  __shared__ __align__(16) char lds[4 * TILEB];
  __shared__ __align__(16) u32x4_t pass[2][2][2][64];         // [rows][from][sixteen] of a lane's operands
  __shared__ float2 offs[2][2][32];
  __shared__ int2 pages_l[LIST];
  __shared__ int32_t counts[NW];
  const BlockDims& m = a.m;
  const HeadItem it = xcd_item(blockIdx.x, m.B * m.Hkv, m.nb * rts, split);
  if (it.head < 0) return;
  const int rt = it.item % rts, i = it.item / rts, hk = it.head % m.Hkv, b = it.head / m.Hkv;
  const BlockSeq s = block_seq(m, b);
  const int t0 = i * m.qblock, rows = min(m.qblock, s.nq - t0) * m.G, base_row = rt * 64;
  if (t0 >= s.nq || base_row >= rows) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, hb = lane >> 5, rg = wave & 1, half = wave >> 1;
  const int row = base_row + rg * 32 + c, tok = t0 + row / m.G, head = hk * m.G + row % m.G;
  const bool there = row < rows;
  const long long rec = (long long)(s.q0 + tok) * m.Hq + head;
  bf16x8_t qf[KS], gf[KS];
  {
    const bf16raw* const q = (const bf16raw*)a.q + (long long)(s.q0 + tok) * a.qs.token + (long long)head * a.qs.head + hb * 8;
    const bf16raw* const g = (const bf16raw*)a.d_o + (long long)(s.q0 + tok) * a.dos.token + (long long)head * a.dos.head + hb * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4_t z = {0, 0, 0, 0}, x = there ? *(const u32x4_t*)(q + ks * 16) : z, y = there ? *(const u32x4_t*)(g + ks * 16) : z;
      qf[ks] = *(const bf16x8_t*)&x;
      gf[ks] = *(const bf16x8_t*)&y;
    }
  }
  const int lim = there ? (m.causal ? min(s.n, s.first + tok + 1) : s.n) : INT32_MAX;
  const float l = there ? a.lse[rec] : -INFINITY, lse = l == -INFINITY ? INFINITY : l * LOG2E, delta = there ? a.delta[rec] : 0.f;
  const bool wave_has_rows = base_row + rg * 32 < rows;
  const int minlim = m.causal ? min(s.n, s.first + t0 + (base_row + rg * 32) / m.G + 1) : s.n;
  const int last = min(base_row + 64, rows) - 1;
  const int maxlim = m.causal ? min(s.n, s.first + t0 + last / m.G + 1) : s.n;
  const int pages = maxlim > 0 ? (maxlim + m.page - 1) >> m.lpage : 0;
  const int32_t* const list = a.sel ? a.sel + (((long long)b * m.nb + i) * m.Hkv + hk) * m.topk : nullptr;
  const int entries = list ? m.topk : pages;
  f32x16_t acc[DB];                                 // of dS K in the first wave of a pair, of P K in the second
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = zero16();
  float off = 0.f, exact[2] = {0.f, 0.f};            // sums of dS, rounded and not
  const float sc = a.scale_log2e;

  int lrow[PT], piece[PT];
#pragma unroll
  for (int x = 0; x < PT; ++x) {
    const int item = tid + x * NT;
    lrow[x] = item / CH;
    piece[x] = ((item % CH) ^ swz<D>(lrow[x])) * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void_t*)lds;
  const int lsub = m.lpage - 4, ktok = (int)(a.ks.token * 2), vtok = (int)(a.vs.token * 2);
  int ra[KS], ca[DB][2];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) ra[ks] = row_operand<D>(lane, ks);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 2; ++x) ca[db][x] = col_operand<D>(lane, db, x);

  for (int e0 = 0; e0 < entries; e0 += LIST) {
    const int n = fill_list<NT>(m, b, list, e0, 1, entries, pages, pages_l, counts);
    const int parts = n << lsub, tiles = (parts + 3) >> 2;
    if (!tiles) continue;
    auto issue = [&](int stage, int t) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < PT; ++x) {
        const int part = min(t * 4 + (((wave * 64 + x * NT) / CH) >> 4), parts - 1);
        const int pg = __builtin_amdgcn_readfirstlane(pages_l[part >> lsub].x);
        int sub = part & ((1 << lsub) - 1), have = s.n - ((pg << m.lpage) + sub * 16);
        if (have <= 0) { sub = 0; have = 1; }
        const int r = min(lrow[x] & 15, have - 1);
        const uint32_t dst = lds0 + stage * 2 * TILEB + (wave * 64 + x * NT) * 16;
        dma_b128(dst, (uint32_t)(r * ktok + piece[x]), uniform((const char*)a.k + row_at(m, s, a.ks, 0, pg, sub, hk) * 2));
        dma_b128(dst + TILEB, (uint32_t)(r * vtok + piece[x]), uniform((const char*)a.v + row_at(m, s, a.vs, 0, pg, sub, hk) * 2));
      }
    };
    issue(0, 0);
    wait_vmcnt<0>();
    lds_barrier();
    for (int t = 0; t < tiles; ++t) {
      if (t + 1 < tiles) issue((t + 1) & 1, t + 1);
      const char* const kt = lds + (t & 1) * 2 * TILEB;
      const char* const vt = kt + TILEB;
      bf16x8_t own[2];
      if (wave_has_rows) {
        f32x16_t sa = zero16(), dp = zero16();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          sa = mfma32(*(const bf16x8_t*)(kt + half * 32 * ROWB + ra[ks]), qf[ks], sa);
          dp = mfma32(*(const bf16x8_t*)(vt + half * 32 * ROWB + ra[ks]), gf[ks], dp);
        }
        bool whole = true;
        int key0[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int part = t * 4 + half * 2 + x, pg = __builtin_amdgcn_readfirstlane(pages_l[min(part, parts - 1) >> lsub].x);
          key0[x] = part < parts ? (pg << m.lpage) + (part & ((1 << lsub) - 1)) * 16 : INT32_MAX - 64;
          whole = whole && key0[x] + 16 <= minlim;
        }
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          sa[v] = __builtin_amdgcn_exp2f(fmaf(sa[v], sc, -lse));
          dp[v] = sa[v] * (dp[v] - delta);
        }
        if (!whole) {
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (key0[v >> 3] + 8 * ((v >> 2) & 1) + 4 * hb + (v & 3) >= lim) sa[v] = dp[v] = 0.f;
        }
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          const bf16x8_t pf = pack8(sa, s2), df = pack8(dp, s2);
          off = sum8(df, off);
#pragma unroll
          for (int v = 0; v < 8; ++v) exact[v & 1] += dp[8 * s2 + v];
          own[s2] = half ? pf : df;
          *(bf16x8_t*)&pass[rg][half][s2][lane] = half ? df : pf;
        }
      }
      lds_barrier();
      if (wave_has_rows) {
#pragma unroll
        for (int x = 0; x < 2; ++x)                   // its own half of the keys, then the other
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2) {
            const bf16x8_t w = x == 0 ? own[s2] : *(const bf16x8_t*)&pass[rg][half ^ 1][s2][lane];
            const char* const p = kt + ((half ^ x) * 32 + 16 * s2) * ROWB;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = mfma32(join_tr(read_tr(p + ca[db][0]), read_tr(p + ca[db][1])), w, acc[db]);
          }
      }
      wait_vmcnt<0>();
      lds_barrier();
    }
  }
  off += __shfl_xor(off, 32);
  float fix = exact[0] + exact[1];
  fix += __shfl_xor(fix, 32);
  if (hb == 0) offs[rg][half][c] = float2{off, fix};
  float* const pk = (float*)lds + rg * 64 * 64;      // P K to the first wave of a pair: [value][lane]
  if (half) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) pk[(db * 16 + v) * 64 + lane] = acc[db][v];
  }
  __syncthreads();
  if (half || !there) return;
  const float e = offs[rg][0][c].x + offs[rg][1][c].x;
  bf16raw* const out = (bf16raw*)a.dq + (long long)(s.q0 + tok) * a.dqs.token + (long long)head * a.dqs.head + 4 * hb;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
#pragma unroll
    for (int v = 0; v < 16; ++v) acc[db][v] = (acc[db][v] - e * pk[(db * 16 + v) * 64 + lane]) * a.scale;
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *(uint2*)(out + db * 32 + 8 * x) = uint2{pack_bf16x2(acc[db][4 * x], acc[db][4 * x + 1]), pack_bf16x2(acc[db][4 * x + 2], acc[db][4 * x + 3])};
  }
  if (hb == 0) a.delta[rec] = delta + offs[rg][0][c].y + offs[rg][1][c].y;             // (its only reader and writer in this launch)
}

// The same at d = 128, by pairs of waves as in grad_q_pair: each forms weights and dS of 32 of a tile's 64 rows, and sums one of dV and dK
// over all of them.  64 keys a workgroup: 1 050 us, 1 335 by the kernel for d = 64.
__global__ __launch_bounds__(256, 2) void grad_kv_pair(BlockGradArgs a, int split) {
  constexpr int D = 128, KG = 2, TR = 64, KS = D / 16, DB = D / 32, CH = D / 8, ROWB = D * 2;
  constexpr int PT = TR * CH / 256, TILEB = TR * ROWB;
  __shared__ __align__(16) char lds[4 * TILEB];
  __shared__ __align__(16) u32x4_t pass[2][2][2][64];         // [keys][from][sixteen] of a lane's operands
  __shared__ __align__(16) float row_lse[2][TR], row_delta[2][TR];
  __shared__ __align__(16) int row_lim[2][TR];
  const BlockDims& m = a.m;
  // The first pages come first, those of all heads side by side: they are seen by most.  A head stays on the same XCDs (as in xcd_item).
  // Shares behind the first come last.
  const int heads = m.B * m.Hkv, units = heads * split, per = (a.groups + split - 1) / split * units;
  const int part = uniform((int)(blockIdx.x / (unsigned)per)), at = uniform((int)(blockIdx.x % (unsigned)per)), unit = at % units;
  const int head = unit / split, kg = at / units * split + unit % split, group = kg * heads + head, hk = head % m.Hkv, b = head / m.Hkv;
  if (kg >= a.groups) return;
  const BlockSeq s = block_seq(m, b);
  if (kg * KG * 32 >= s.n) return;
  const uint32_t* const marks = a.sel ? a.marks + (((long long)b * m.Hkv + hk) * m.max_pages + (kg * KG * 32 >> m.lpage)) * a.words : nullptr;
  const int blocks = (s.nq + m.qblock - 1) / m.qblock;
  const Share share = page_share(a, marks, blocks, part);
  if (part >= share.parts) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, hb = lane >> 5;
  const int kw = wave & 1, half = wave >> 1, key0 = kg * KG * 32 + kw * 32, key = key0 + c;
  bf16x8_t kf[KS], vf[KS];
  {
    const bf16raw* const k = (const bf16raw*)a.k + (s.k0 + (long long)key) * a.ks.token + hk * a.ks.head + hb * 8;
    const bf16raw* const v = (const bf16raw*)a.v + (s.k0 + (long long)key) * a.vs.token + hk * a.vs.head + hb * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4_t z = {0, 0, 0, 0}, x = key < s.n ? *(const u32x4_t*)(k + ks * 16) : z, y = key < s.n ? *(const u32x4_t*)(v + ks * 16) : z;
      kf[ks] = *(const bf16x8_t*)&x;
      vf[ks] = *(const bf16x8_t*)&y;
    }
  }
  f32x16_t acc[DB];                                 // of dV in the first wave of a pair, of dK in the second
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = zero16();
  const float sc = a.scale_log2e, inv_g = 1.f / m.G;

  int lrow[PT], piece[PT];
#pragma unroll
  for (int x = 0; x < PT; ++x) {
    const int item = tid + x * 256;
    lrow[x] = item / CH;
    piece[x] = ((item % CH) ^ swz<D>(lrow[x])) * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void_t*)lds;
  const int qtok = (int)(a.qs.token * 2), qhead = (int)(a.qs.head * 2), gtok = (int)(a.dos.token * 2), ghead = (int)(a.dos.head * 2);
  int ra[KS], ca[DB][2];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) ra[ks] = row_operand<D>(lane, ks);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 2; ++x) ca[db][x] = col_operand<D>(lane, db, x);

  // tiles of the blocks that list the page and are not all before its keys: block `i`, rows from `base`
  int word = -1, i = 0, base = 0, rows = 0, skip = share.first, left = share.count;
  uint32_t bits = 0;
  auto advance = [&]() __attribute__((always_inline)) {      // false: no tile is left
    base += TR;
    for (;;) {
      for (; base < rows; base += TR)
        if (!m.causal || s.first + i * m.qblock + (min(base + TR, rows) - 1) / m.G >= kg * KG * 32) return true;
      while (!bits) {
        if (++word * 32 >= blocks) return false;
        bits = marks ? (uint32_t)uniform((int)marks[word]) : ~0u;
        if (blocks - word * 32 < 32) bits &= (1u << (blocks - word * 32)) - 1;
      }
      if (!left) return false;
      i = word * 32 + __builtin_ctz(bits);
      bits &= bits - 1;
      if (skip) { --skip; continue; }
      --left;
      base = 0;
      rows = min(m.qblock, s.nq - i * m.qblock) * m.G;
    }
  };
  float nl = 0.f, nd = 0.f;
  int nlim = 0;
  auto issue = [&](int stage) __attribute__((always_inline)) {
    const int t0 = i * m.qblock;
    const char* const q = uniform((const char*)a.q + ((long long)(s.q0 + t0) * a.qs.token + (long long)(hk * m.G) * a.qs.head) * 2);
    const char* const g = uniform((const char*)a.d_o + ((long long)(s.q0 + t0) * a.dos.token + (long long)(hk * m.G) * a.dos.head) * 2);
#pragma unroll
    for (int x = 0; x < PT; ++x) {
      const int r = min(base + lrow[x], rows - 1), t = (int)((r + 0.5f) * inv_g), h = r - t * m.G;
      const uint32_t dst = lds0 + stage * 2 * TILEB + (wave * 64 + x * 256) * 16;
      dma_b128(dst, (uint32_t)(t * qtok + h * qhead + piece[x]), q);
      dma_b128(dst + TILEB, (uint32_t)(t * gtok + h * ghead + piece[x]), g);
    }
    if (tid < TR) {
      const int r = base + tid, t = (int)((r + 0.5f) * inv_g);
      const bool there = r < rows;
      const long long x = (long long)(s.q0 + t0 + t) * m.Hq + hk * m.G + (r - t * m.G);
      const float l = there ? a.lse[x] : -INFINITY;
      nl = l == -INFINITY ? INFINITY : l * LOG2E;
      nd = there ? a.delta[x] : 0.f;
      nlim = there ? (m.causal ? min(s.n, s.first + t0 + t + 1) : s.n) : 0;
    }
  };
  auto land = [&](int stage) __attribute__((always_inline)) {
    if (tid < TR) { row_lse[stage][tid] = nl; row_delta[stage][tid] = nd; row_lim[stage][tid] = nlim; }
    wait_vmcnt<0>();
    lds_barrier();
  };
  bool more = advance();
  if (more) { issue(0); land(0); }
  int u = 0;
  while (more) {
    // the keys a row of the tile misses at most: none where its first row sees them all and all of its rows are there
    const int first_lim = m.causal ? min(s.n, s.first + i * m.qblock + base / m.G + 1) : s.n;
    const bool whole = key0 + 32 <= first_lim && base + TR <= rows;
    more = advance();
    if (more) issue(u ^ 1);
    const char* const qt = lds + u * 2 * TILEB;
    const char* const gt = qt + TILEB;
    bf16x8_t own[2];
    {
      const int r0 = half * 32;
      f32x16_t sa = zero16(), dp = zero16();
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        sa = mfma32(*(const bf16x8_t*)(qt + r0 * ROWB + ra[ks]), kf[ks], sa);
        dp = mfma32(*(const bf16x8_t*)(gt + r0 * ROWB + ra[ks]), vf[ks], dp);
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const f32x4_t l4 = *(const f32x4_t*)&row_lse[u][r0 + 8 * x + 4 * hb], d4 = *(const f32x4_t*)&row_delta[u][r0 + 8 * x + 4 * hb];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sa[4 * x + j] = __builtin_amdgcn_exp2f(fmaf(sa[4 * x + j], sc, -l4[j]));
          dp[4 * x + j] = sa[4 * x + j] * (dp[4 * x + j] - d4[j]);
        }
      }
      if (!whole) {
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (key >= row_lim[u][r0 + 8 * x + 4 * hb + j]) sa[4 * x + j] = dp[4 * x + j] = 0.f;
      }
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const bf16x8_t pf = pack8(sa, s2), df = pack8(dp, s2);
        own[s2] = half ? df : pf;
        *(bf16x8_t*)&pass[kw][half][s2][lane] = half ? pf : df;
      }
    }
    lds_barrier();
    const char* const ct = half ? qt : gt;
#pragma unroll
    for (int x = 0; x < 2; ++x)                       // its own half of the rows, then the other
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        const bf16x8_t w = x == 0 ? own[s2] : *(const bf16x8_t*)&pass[kw][half ^ 1][s2][lane];
        const char* const p = ct + ((half ^ x) * 32 + 16 * s2) * ROWB;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = mfma32(join_tr(read_tr(p + ca[db][0]), read_tr(p + ca[db][1])), w, acc[db]);
      }
    if (more) land(u ^ 1);
    u ^= 1;
  }
  if (share.parts > 1) {
    float* const to = share_slot(a, group, part, wave, lane);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) to[(db * 16 + v) * 64] = acc[db][v];
    return;
  }
  if (key >= s.n) return;
  store_rows<DB>((half ? (bf16raw*)a.dk + (s.k0 + (long long)key) * a.dks.token + hk * a.dks.head
                       : (bf16raw*)a.dv + (s.k0 + (long long)key) * a.dvs.token + hk * a.dvs.head) + 4 * hb, acc, half ? a.scale : 1.f);
}

// The sums of pages whose blocks were dealt to several workgroups.  A wave's lane holds what it held there: d = 64 both gradients of a key
// (wave: 32 keys, or with two of them the first two waves), d = 128 one of them (waves 0, 1: dV; 2, 3: dK).
template <int D, int KG>
__global__ __launch_bounds__(256) void grad_kv_join(BlockGradArgs a) {
  constexpr int DB = D / 32;
  const BlockDims& m = a.m;
  const int group = blockIdx.x, hk = group % m.Hkv, b = group / m.Hkv % m.B, kg = group / m.Hkv / m.B;
  const BlockSeq s = block_seq(m, b);
  if (kg * KG * 32 >= s.n) return;
  const uint32_t* const marks = a.marks + (((long long)b * m.Hkv + hk) * m.max_pages + (kg * KG * 32 >> m.lpage)) * a.words;
  const Share share = page_share(a, marks, (s.nq + m.qblock - 1) / m.qblock, 0);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (share.parts < 2 || (D == 64 && wave >= KG)) return;
  f32x16_t x[4];                                     // 64 values
#pragma unroll
  for (int y = 0; y < 4; ++y) x[y] = zero16();
  for (int part = 0; part < share.parts; ++part) {
    const float* const from = share_slot(a, group, part, wave, lane);
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int v = 0; v < 16; ++v) x[y][v] += from[(y * 16 + v) * 64];
  }
  const int key = kg * KG * 32 + (D == 64 ? wave : wave & 1) * 32 + (lane & 31), hb = lane >> 5;
  if (key >= s.n) return;
  bf16raw* const ok = (bf16raw*)a.dk + (s.k0 + (long long)key) * a.dks.token + hk * a.dks.head + 4 * hb;
  bf16raw* const ov = (bf16raw*)a.dv + (s.k0 + (long long)key) * a.dvs.token + hk * a.dvs.head + 4 * hb;
  if constexpr (D == 64) { store_rows<DB>(ok, x, a.scale); store_rows<DB>(ov, x + DB, 1.f); }
  else store_rows<DB>(wave >> 1 ? ok : ov, x, wave >> 1 ? a.scale : 1.f);
}

// The kernels for many rows: bf16, blocks of more than 32 rows at d = 128 (one sequence of 4 096, blocks of 40 rows: a pass
// 573 us, 769 by those for few rows), of at least 48 at d = 64 (40 rows: 574 us, 438);
// dK and dV over pages of 64 keys or more ...
bool rows_wide(const BlockDims& m, int dtype, int d) { return dtype == ADACLUSTER_BF16 && m.qblock * m.G >= (d == 128 ? 33 : 48) && m.qblock * m.G <= (1 << 20); }
// ... with offsets inside a block or a sixteenth that 32 bits hold.
bool wide_takes(const BlockGradArgs& a, int dtype, int d) {
  const BlockDims& m = a.m;
  const auto block = [&](const KeyStride& st) { return m.qblock * st.token + m.G * st.head < (1 << 30); };
  return rows_wide(m, dtype, d) && a.ks.token < (1 << 25) && a.vs.token < (1 << 25) && block(a.qs) && block(a.dos);
}

// Workgroups that a page's blocks go to at most, where there are lists and a launch has fewer than 4 096 workgroups (eight rounds of two a CU,
// and 268 MB of sums at most); and the blocks from which on: a quarter more than a page has on average.  A training pass of one
// sequence of 8 192 tokens, lists of 32 pages: 4 / 1 heads, d = 128 1 226 -> 541 us, 16 / 4 heads 1 575 -> 1 031, 8 / 2 heads, d = 64 734 -> 392;
// three sequences, 1 536 workgroups: 3 % of the launch.
struct Deal { int keys, groups, np, limit; long long wg; size_t bytes; };
Deal deal_of(const BlockDims& m, int dtype, int d, bool wide, bool listed) {
  Deal x;
  if (wide) x.keys = d == 64 && m.page >= 128 ? 128 : 64;
  // 32 keys a workgroup (its registers allow that but for fp32 at d = 128) where that leaves two workgroups a CU (fp32, one head of 4 096
  // keys: 128 workgroups 216 us, 256 of 16 keys 154, and with the first pages dealt out 78)
  else x.keys = m.page == 16 || (dtype == ADACLUSTER_F32 && d == 128) || (long long)(m.max_pages << m.lpage) / 32 * m.Hkv * m.B < 512 ? 16 : 32;
  x.groups = (m.max_pages << m.lpage) / x.keys;
  x.wg = (long long)x.groups * m.Hkv * m.B;
  x.np = listed && x.wg < 4096 ? (int)(x.wg < 512 ? 8 : 4096 / x.wg) : 1;
  const long long mean = (long long)m.nb * m.topk / m.max_pages;
  x.limit = (int)(mean + mean / 4 > 4 ? mean + mean / 4 : 4);
  x.bytes = x.np > 1 ? (size_t)x.wg * x.np * (wide ? 4 * 4096 : 2 * x.keys * d) * sizeof(float) : 0;
  return x;
}

template <int D>
int go_wide_q(hipStream_t s, const BlockGradArgs& a) {
  const BlockDims& m = a.m;
  const int rows = m.qblock * m.G, per = D == 128 ? 64 : 128, rts = (rows + per - 1) / per;
  const long long heads = (long long)m.Hkv * m.B, grid = xcd_grid(heads, (long long)rts * m.nb);
  const int split = xcd_split(heads);
  if (!grid_fits(grid)) return ADACLUSTER_E_UNSUPPORTED;
  if constexpr (D == 128) grad_q_pair<<<(int)grid, 256, 0, s>>>(a, rts, split); else grad_q_wide<<<(int)grid, 256, 0, s>>>(a, rts, split);
  return launched();
}

template <int D>
int go_wide_kv(hipStream_t s, const BlockGradArgs& a, const Deal& x) {
  const BlockDims& m = a.m;
  const long long heads = (long long)m.Hkv * m.B, wk = xcd_grid(heads, x.groups) * x.np;
  const int split = xcd_split(heads);
  if (!grid_fits(wk)) return ADACLUSTER_E_UNSUPPORTED;
  if constexpr (D == 128) grad_kv_pair<<<(int)wk, 256, 0, s>>>(a, split);
  else if (x.keys == 128) grad_kv_wide<4><<<(int)wk, 256, 0, s>>>(a, split);
  else grad_kv_wide<2><<<(int)wk, 256, 0, s>>>(a, split);
  if (x.np > 1) {
    if (int rc = launched()) return rc;
    if constexpr (D == 128) grad_kv_join<128, 2><<<(int)x.wg, 256, 0, s>>>(a);
    else if (x.keys == 128) grad_kv_join<64, 4><<<(int)x.wg, 256, 0, s>>>(a);
    else grad_kv_join<64, 2><<<(int)x.wg, 256, 0, s>>>(a);
  }
  return launched();
}

template <typename T, int D>
int go(hipStream_t s, const BlockGradArgs& a, const Deal& x, bool wide) {
  const BlockDims& m = a.m;
  constexpr int RPI = 256 / (D / Vec<T>::N);
  const long long deltas = ((long long)m.q_rows * m.Hq + RPI - 1) / RPI;
  const int rows = m.qblock * m.G, R = rows <= 16 ? 1 : 2, rts = (rows + 16 * R - 1) / (16 * R);
  const long long wq = (long long)rts * m.nb * m.Hkv * m.B, wk = x.wg * x.np;
  const long long entries = a.sel ? (long long)m.B * m.nb * m.Hkv * m.topk : 0;
  if (!grid_fits(deltas) || !grid_fits(wq) || !grid_fits(wk) || !grid_fits(entries / 256 + 1)) return ADACLUSTER_E_UNSUPPORTED;
  if (a.sel) {
    if (int rc = launch_fill_i32(s, (int32_t*)a.marks, (size_t)m.B * m.Hkv * m.max_pages * a.words, 0)) return rc;
    grad_marks<<<(int)((entries + 255) / 256), 256, 0, s>>>(a, entries);
    if (int rc = launched()) return rc;
  }
  grad_delta<T, D><<<(int)deltas, 256, 0, s>>>(a);
  if (int rc = launched()) return rc;
  if constexpr (sizeof(T) == 2) {
    if (wide) {
      if (int rc = go_wide_q<D>(s, a)) return rc;
      if (m.page >= 64) return go_wide_kv<D>(s, a, x);
    }
  }
  if (!wide) {
    if (R == 1) grad_q<T, D, 1><<<(int)wq, 256, 0, s>>>(a, rts); else grad_q<T, D, 2><<<(int)wq, 256, 0, s>>>(a, rts);
    if (int rc = launched()) return rc;
  }
  if (x.keys == 16) grad_kv<T, D, 1><<<(int)wk, 256, 0, s>>>(a);
  else if constexpr (sizeof(T) == 2 || D == 64) grad_kv<T, D, 2><<<(int)wk, 256, 0, s>>>(a);
  if (x.np > 1) {
    if (int rc = launched()) return rc;
    if (x.keys == 16) grad_kv_add<T, D, 1><<<(int)x.wg, 256, 0, s>>>(a);
    else if constexpr (sizeof(T) == 2 || D == 64) grad_kv_add<T, D, 2><<<(int)x.wg, 256, 0, s>>>(a);
  }
  return launched();
}

size_t marks_bytes(const BlockDims& m) { return align_up((size_t)m.B * m.Hkv * m.max_pages * ((m.nb + 31) / 32) * 4, 256); }
size_t delta_bytes(const BlockDims& m) { return align_up((size_t)m.q_rows * m.Hq * 4, 256); }

}  // namespace

size_t block_grad_bytes(const BlockDims& m, int dtype, int d, bool listed) {
  const size_t few = deal_of(m, dtype, d, false, listed).bytes, many = rows_wide(m, dtype, d) && m.page >= 64 ? deal_of(m, dtype, d, true, listed).bytes : 0;
  return delta_bytes(m) + (listed ? marks_bytes(m) : 0) + (few > many ? few : many);      // (which kernels run hangs on the strides too)
}

int launch_block_attn_backward(hipStream_t s, int dtype, int d, BlockGradArgs a, void* ws) {
  const bool wide = wide_takes(a, dtype, d);
  const Deal x = deal_of(a.m, dtype, d, wide && a.m.page >= 64, a.sel != nullptr);
  a.delta = (float*)ws;
  a.marks = (uint32_t*)((char*)ws + delta_bytes(a.m));
  a.sums = (float*)((char*)a.marks + marks_bytes(a.m));
  a.words = (a.m.nb + 31) / 32;
  a.np = x.np;
  a.limit = x.limit;
  a.groups = x.groups;
  a.wg = (int)x.wg;
  if (dtype == ADACLUSTER_BF16) return d == 64 ? go<bf16raw, 64>(s, a, x, wide) : go<bf16raw, 128>(s, a, x, wide);
  return d == 64 ? go<float, 64>(s, a, x, wide) : go<float, 128>(s, a, x, wide);
}

}  // namespace adac
