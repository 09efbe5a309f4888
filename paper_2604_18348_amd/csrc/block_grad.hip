// Gradients of attention over listed pages of packed keys.  With P = softmax(scale Q K^T) over what a row sees,
//   dV = P^T dO,  dP = dO V^T,  dS = P (dP - rowsum(dO O)),  dQ = scale dS K,  dK = scale dS^T Q,
// dK and dV summed over the query heads that share the keys.  P is formed again from the scores and the row's logarithm of its sum.
// Two kernels, so that no sum is made with atomics: one goes over a block's list of keys for dQ, one over the blocks of queries that
// list a page for dK and dV (bit masks, set beforehand from the lists; the order of a sum is the order of the bits).
#include "block.h"
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
// formed at the end (against 64 bits, 17 776 keys, d=64: dQ 0.0047 off without, 0.0025 with it); the corrected sums go on to grad_kv.
template <typename T, int D, int R>
__global__ __launch_bounds__(256) void grad_q(BlockGradArgs a, int rts) {
  constexpr int NF = D * sizeof(T) / 64, ND = D / 16;
  constexpr bool FIX = sizeof(T) == 2;
  constexpr int KBYTES = 32 * D * sizeof(T), JBYTES = (FIX ? 2 : 1) * 4 * 16 * D * 4 + 4 * 16 * 4;
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
  float off[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    off[r] = 0.f;
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
        f32x4_t sc{0.f, 0.f, 0.f, 0.f}, dp{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int f = 0; f < NF; ++f) { sc = mma(T{}, k[h].p[f], q[r].p[f], sc); dp = mma(T{}, v[h].p[f], g[r].p[f], dp); }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool sees = key0[h] + 4 * quarter + j < lim[r];
          const float w = __builtin_amdgcn_exp2f(fmaf(sc[j], a.scale_log2e, -lse[r]));
          p[h][j] = sees ? w : 0.f;
          ds[h][j] = sees ? w * (dp[j] - delta[r]) : 0.f;
          if constexpr (FIX) off[r] += ds[h][j];
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
    if constexpr (FIX) { const float e = quarters_sum(off[r]); if (quarter == 0) js[wave * 16 + n16] = e; }
    __syncthreads();
    const int jr = tid >> 4, row = base_row + r * 16 + jr, d0 = (tid & 15) * (D / 16);
    if (row >= rows) continue;
    float e = 0.f;
    if constexpr (FIX) {
      e = js[jr] + js[16 + jr] + js[32 + jr] + js[48 + jr];
      if (d0 == 0) a.delta[(long long)(s.q0 + t0 + row / m.G) * m.Hq + hk * m.G + row % m.G] += e;      // (its only reader and writer here)
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

// dK and dV of KR * 16 keys of one head: the waves take tiles of 32 rows in turns.  S = Q K^T and dP = dO V^T leave a lane one key
// and four rows: P and dS are the operands of dV^T = dO^T P and dK^T = Q^T dS as they stand.
template <typename T, int D, int KR>
__global__ __launch_bounds__(256) void grad_kv(BlockGradArgs a, int groups) {
  constexpr int NF = D * sizeof(T) / 64, ND = D / 16;
  constexpr int TBYTES = 32 * D * sizeof(T), JBYTES = 4 * 16 * D * 4;
  __shared__ __align__(16) char lds[8 * TBYTES > JBYTES ? 8 * TBYTES : JBYTES];
  const BlockDims& m = a.m;
  int id = blockIdx.x;
  const int kg = id % groups; id /= groups;
  const int hk = id % m.Hkv, b = id / m.Hkv;
  const BlockSeq s = block_seq(m, b);
  const int key0 = kg * KR * 16;
  if (key0 >= s.n) return;
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
  const uint32_t* const marks = a.sel ? a.marks + (((long long)b * m.Hkv + hk) * m.max_pages + (key0 >> m.lpage)) * a.words : nullptr;
  const int blocks = (s.nq + m.qblock - 1) / m.qblock;
  int unit = 0;
  for (int w = 0; w * 32 < blocks; ++w) {
    uint32_t bits = marks ? marks[w] : ~0u;
    if (blocks - w * 32 < 32) bits &= (1u << (blocks - w * 32)) - 1;
    while (bits) {
      const int i = w * 32 + __builtin_ctz(bits), t0 = i * m.qblock, rows = min(m.qblock, s.nq - t0) * m.G;
      bits &= bits - 1;
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
            f32x4_t sc{0.f, 0.f, 0.f, 0.f}, dp{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int f = 0; f < NF; ++f) { sc = mma(T{}, q[h].p[f], k[r].p[f], sc); dp = mma(T{}, g[h].p[f], v[r].p[f], dp); }
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

template <typename T, int D>
int go(hipStream_t s, const BlockGradArgs& a) {
  const BlockDims& m = a.m;
  constexpr int RPI = 256 / (D / Vec<T>::N);
  const long long deltas = ((long long)m.q_rows * m.Hq + RPI - 1) / RPI;
  const int rows = m.qblock * m.G, R = rows <= 16 ? 1 : 2, rts = (rows + 16 * R - 1) / (16 * R);
  const int KR = m.page == 16 || (sizeof(T) == 4 && D == 128) ? 1 : 2, groups = (m.max_pages << m.lpage) / (16 * KR);
  const long long wq = (long long)rts * m.nb * m.Hkv * m.B, wk = (long long)groups * m.Hkv * m.B;
  const long long entries = a.sel ? (long long)m.B * m.nb * m.Hkv * m.topk : 0;
  if (!grid_fits(deltas) || !grid_fits(wq) || !grid_fits(wk) || !grid_fits(entries / 256 + 1)) return ADACLUSTER_E_UNSUPPORTED;
  if (a.sel) {
    if (int rc = launch_fill_i32(s, (int32_t*)a.marks, (size_t)m.B * m.Hkv * m.max_pages * a.words, 0)) return rc;
    grad_marks<<<(int)((entries + 255) / 256), 256, 0, s>>>(a, entries);
    if (int rc = launched()) return rc;
  }
  grad_delta<T, D><<<(int)deltas, 256, 0, s>>>(a);
  if (int rc = launched()) return rc;
  if (R == 1) grad_q<T, D, 1><<<(int)wq, 256, 0, s>>>(a, rts); else grad_q<T, D, 2><<<(int)wq, 256, 0, s>>>(a, rts);
  if (int rc = launched()) return rc;
  if (KR == 1) grad_kv<T, D, 1><<<(int)wk, 256, 0, s>>>(a, groups);
  else if constexpr (sizeof(T) == 2 || D == 64) grad_kv<T, D, 2><<<(int)wk, 256, 0, s>>>(a, groups);
  return launched();
}

size_t delta_bytes(const BlockDims& m) { return align_up((size_t)m.q_rows * m.Hq * 4, 256); }

}  // namespace

size_t block_grad_bytes(const BlockDims& m, bool listed) {
  return delta_bytes(m) + (listed ? (size_t)m.B * m.Hkv * m.max_pages * ((m.nb + 31) / 32) * 4 : 0);
}

int launch_block_attn_backward(hipStream_t s, int dtype, int d, BlockGradArgs a, void* ws) {
  a.delta = (float*)ws;
  a.marks = (uint32_t*)((char*)ws + delta_bytes(a.m));
  a.words = (a.m.nb + 31) / 32;
  if (dtype == ADACLUSTER_BF16) return d == 64 ? go<bf16raw, 64>(s, a) : go<bf16raw, 128>(s, a);
  return d == 64 ? go<float, 64>(s, a) : go<float, 128>(s, a);
}

}  // namespace adac
