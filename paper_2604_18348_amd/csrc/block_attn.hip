// Attention of blocks of queries over listed pages of keys, packed or in a paged cache, in 16 and 32 bits or from 4-bit codes.
#include "block_few.h"

namespace adac {

namespace {

template <typename T, int BITS, int D, int R>
__global__ __launch_bounds__(256, (few_waves<T, BITS, D, R>())) void block_attn(BlockAttnArgs a, int rts) {
  __shared__ FewLds<T, BITS, D> sh;
  few_rows<T, BITS, D, R, false>(a, rts, blockIdx.x, sh);
}

// Joins the nsplit partial results of a row: a wave's 16 lanes a row.
template <typename T, int D>
__global__ __launch_bounds__(256) void block_attn_join(BlockAttnArgs a, int rts, int R) {
  const BlockDims& m = a.m;
  const int item = blockIdx.x / R, r = blockIdx.x % R;
  int id = item;
  const int rt = id % rts; id /= rts;
  const int i = id % m.nb; id /= m.nb;
  const int hk = id % m.Hkv, b = id / m.Hkv;
  const BlockSeq s = block_seq(m, b);
  const int t0 = i * m.qblock, rows = min(m.qblock, s.nq - t0) * m.G;
  const int jr = threadIdx.x >> 4, row = (rt * R + r) * 16 + jr, d0 = (threadIdx.x & 15) * (D / 16);
  if (t0 >= s.nq || row >= rows) return;
  const long long rec = (long long)item * a.nsplit * (16 * R) + r * 16 + jr;
  float top = -INFINITY, all = 0.f, o[D / 16];
  for (int z = 0; z < a.nsplit; ++z) top = fmaxf(top, a.part_ml[(rec + (long long)z * 16 * R) * 2]);
  const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int x = 0; x < D / 16; ++x) o[x] = 0.f;
  for (int z = 0; z < a.nsplit; ++z) {
    const long long at = rec + (long long)z * 16 * R;
    const float f = __builtin_amdgcn_exp2f(a.part_ml[at * 2] - ref);
    all += f * a.part_ml[at * 2 + 1];
#pragma unroll
    for (int x = 0; x < D / 16; x += 4) {
      const f32x4_t v = *(const f32x4_t*)(a.part_o + at * D + d0 + x);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[x + j] = fmaf(f, v[j], o[x + j]);
    }
  }
  const int t = t0 + row / m.G, head = hk * m.G + row % m.G;
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

struct Shape { int R, rts, nsplit; long long items; };
Shape shape_of(const BlockDims& m, bool listed) {
  Shape s;
  // 32 rows a wave at most: more registers than a wave has beside what is on its way (64 rows: 16 x 8 rows over 32 768 keys, d = 128 146 us,
  // now 107; 4-bit chunks of 512 tokens over 48 pages 339, now 295).
  const int rows = m.qblock * m.G;
  s.R = rows <= 16 ? 1 : 2;
  s.rts = (rows + 16 * s.R - 1) / (16 * s.R);
  s.items = (long long)s.rts * m.nb * m.Hkv * m.B;
  // Few rows: the list is split until the launch has four workgroups a CU, each wave with two turns of 32 keys at least.
  const long long turns = ((long long)(listed ? m.topk : m.max_pages) << (m.lpage - 4)) / 2;
  long long n = (1024 + s.items - 1) / s.items;
  if (n > turns / 8) n = turns / 8;
  s.nsplit = (int)(n < 1 ? 1 : n);
  return s;
}

template <typename T, int BITS, int D>
void go(hipStream_t s, const BlockAttnArgs& a, const Shape& sh) {
  const int wg = (int)(sh.items * sh.nsplit);
  if (sh.R == 1) block_attn<T, BITS, D, 1><<<wg, 256, 0, s>>>(a, sh.rts);
  else block_attn<T, BITS, D, 2><<<wg, 256, 0, s>>>(a, sh.rts);
  if (sh.nsplit > 1) block_attn_join<T, D><<<(int)(sh.items * sh.R), 256, 0, s>>>(a, sh.rts, sh.R);
}

}  // namespace

size_t block_attn_bytes(const BlockDims& m, int d, bool listed) {
  const Shape s = shape_of(m, listed);
  if (s.nsplit == 1) return 0;
  const size_t rows = (size_t)s.items * s.nsplit * 16 * s.R;
  return align_up(rows * d * 4, 256) + align_up(rows * 8, 256);
}

int launch_block_attn(hipStream_t s, int dtype, int bits, int d, BlockAttnArgs a, void* ws) {
  if (block_wide_takes(a, dtype, bits)) return launch_block_attn_wide(s, d, a);
  const Shape sh = shape_of(a.m, a.sel != nullptr);
  if (!grid_fits(sh.items * (sh.nsplit > sh.R ? sh.nsplit : sh.R))) return ADACLUSTER_E_UNSUPPORTED;
  a.nsplit = sh.nsplit;
  a.part_o = (float*)ws;
  a.part_ml = (float*)((char*)ws + align_up((size_t)sh.items * sh.nsplit * 16 * sh.R * d * 4, 256));
  if (dtype == ADACLUSTER_BF16) {
    if (bits == 4) { if (d == 64) go<bf16raw, 4, 64>(s, a, sh); else go<bf16raw, 4, 128>(s, a, sh); }
    else { if (d == 64) go<bf16raw, 0, 64>(s, a, sh); else go<bf16raw, 0, 128>(s, a, sh); }
  } else {
    if (bits == 4) { if (d == 64) go<float, 4, 64>(s, a, sh); else go<float, 4, 128>(s, a, sh); }
    else { if (d == 64) go<float, 0, 64>(s, a, sh); else go<float, 0, 128>(s, a, sh); }
  }
  return launched();
}

}  // namespace adac
