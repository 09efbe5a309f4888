// Attention of blocks of many rows over listed pages, bf16: the walk of block_attn with tiles of 32 keys staged once for all waves.
#include "block_wide.h"

namespace adac {

namespace {

// NW waves of 32 rows each.  A tile's keys and values go global -> LDS directly, 16 bytes a lane, one tile ahead of the products.  Rows past
// a sequence's end are read from the last row there is in their sixteenth (or the page's first) and masked: nothing behind the end is
// touched.  Bound by what lies between the products (exponentials, roundings, LDS reads), so waves a SIMD count: tiles of 32 keys and three
// waves (two with NW = 2) against 64 keys and two, or one: 3 sequences up to 8 192 tokens, 32 pages of 64, 16 / 4 heads, d = 128 385 us
// (489), 17 776 tokens, 30 heads, d = 64 730 (744), chunks of 2 x 1 024 tokens, NW = 2, d = 128 193 (303).
template <int D, int NW>
__global__ __launch_bounds__(NW * 64, NW == 4 ? 3 : 2) void block_attn_wide(BlockAttnArgs a, int rts, int split) {
  constexpr int NT = NW * 64, KS = D / 16, DB = D / 32, CH = D / 8, ROWB = D * 2;
  constexpr int TK = 32, PARTS = TK / 16;      // keys a tile: one product's rows
  constexpr int PT = TK * CH / NT, TILEB = TK * ROWB;
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
  bf16x8_t qf[KS];
  {
    const bf16raw* const p = (const bf16raw*)a.q + (long long)(s.q0 + tok) * a.qs.token + (long long)head * a.qs.head + hb * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4_t w = there ? *(const u32x4_t*)(p + ks * 16) : u32x4_t{0, 0, 0, 0};
      qf[ks] = *(const bf16x8_t*)&w;
    }
  }
  const int lim = there ? (m.causal ? min(s.n, s.first + tok + 1) : s.n) : INT32_MAX;      // (a row that is not there needs no mask)
  const int wave_first = base_row + wave * 32;
  const bool wave_has_rows = wave_first < rows;
  const int minlim = m.causal ? min(s.n, s.first + t0 + wave_first / m.G + 1) : s.n;       // keys below: seen by all rows of the wave
  const int last = min(base_row + NT / 2, rows) - 1;
  const int maxlim = m.causal ? min(s.n, s.first + t0 + last / m.G + 1) : s.n;
  const int pages = maxlim > 0 ? (maxlim + m.page - 1) >> m.lpage : 0;
  const int32_t* const list = a.sel ? a.sel + (((long long)b * m.nb + i) * m.Hkv + hk) * m.topk : nullptr;
  const int entries = list ? m.topk : pages;

  f32x16_t oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = zero16();
  // The weights are taken relative to a reference that moves only when a tile's sum leaves its range (see below); from where it
  // starts, tiles a row sees nothing of leave sum and accumulator at zero.
  const float sc = a.scale_log2e;
  float mref = softmax_start(sc), lrun = 0.f;

  int lrow[PT], piece[PT];                         // this thread's pieces of a tile
#pragma unroll
  for (int x = 0; x < PT; ++x) {
    const int item = tid + x * NT;
    lrow[x] = item / CH;
    piece[x] = ((item % CH) ^ swz<D>(lrow[x])) * 16;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void_t*)lds;
  const int lsub = m.lpage - 4, ktok = (int)(a.ks.token * 2), vtok = (int)(a.vs.token * 2);
  int kaddr[KS], vaddr[DB][2];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kaddr[ks] = row_operand<D>(lane, ks);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 2; ++x) vaddr[db][x] = col_operand<D>(lane, db, x);

  for (int e0 = 0; e0 < entries; e0 += LIST) {
    const int n = fill_list<NT>(m, b, list, e0, 1, entries, pages, pages_l, counts);
    const int parts = n << lsub, tiles = (parts + PARTS - 1) / PARTS;
    if (!tiles) continue;
    auto issue = [&](int stage, int t) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < PT; ++x) {                // a wave's request lies inside one sixteenth of a page
        const int part = min(t * PARTS + (((wave * 64 + x * NT) / CH) >> 4), parts - 1);
        const int2 pp = pages_l[part >> lsub];
        const int pg = uniform(pp.x), phys = uniform(pp.y);
        int sub = part & ((1 << lsub) - 1), have = s.n - ((pg << m.lpage) + sub * 16);      // rows of it that exist
        if (have <= 0) { sub = 0; have = 1; }
        const int r = min(lrow[x] & 15, have - 1);
        const uint32_t dst = lds0 + stage * 2 * TILEB + (wave * 64 + x * NT) * 16;
        dma_b128(dst, (uint32_t)(r * ktok + piece[x]), uniform((const char*)a.k + row_at(m, s, a.ks, phys, pg, sub, hk) * 2));
        dma_b128(dst + TILEB, (uint32_t)(r * vtok + piece[x]), uniform((const char*)a.v + row_at(m, s, a.vs, phys, pg, sub, hk) * 2));
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
        f32x16_t sacc = zero16();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) sacc = mfma32(*(const bf16x8_t*)(kt + kaddr[ks]), qf[ks], sacc);
        int key0[PARTS];
        bool whole = true;
#pragma unroll
        for (int x = 0; x < PARTS; ++x) {
          const int part = t * PARTS + x, pg = uniform(pages_l[min(part, parts - 1) >> lsub].x);
          key0[x] = part < parts ? (pg << m.lpage) + (part & ((1 << lsub) - 1)) * 16 : INT32_MAX - 64;
          whole = whole && key0[x] + 16 <= minlim;
        }
        if (!whole) {
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (key0[v >> 3] + 8 * ((v >> 2) & 1) + 4 * hb + (v & 3) >= lim) sacc[v] = -INFINITY;
        }
        // p = 2^((s - reference) scale): any reference gives the same result as long as nothing overflows.  The row sum of the tile
        // tells (on the first tile with a score above -inf it is infinite): only then is the tile's maximum taken, the reference
        // moved up to it and the accumulator scaled.
        bf16x8_t pf[2];
        float rsum;
        auto weights = [&]() __attribute__((always_inline)) {
          const float off = mref * sc;
          float part[2];
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2) {
            union { uint32_t w[4]; bf16x8_t v; } u;
            part[s2] = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float p0 = __builtin_amdgcn_exp2f(fmaf(sacc[8 * s2 + 2 * j], sc, -off)), p1 = __builtin_amdgcn_exp2f(fmaf(sacc[8 * s2 + 2 * j + 1], sc, -off));
              u.w[j] = pack_bf16x2(p0, p1);
              part[s2] += p0;                       // (not the rounded ones: the sum's logarithm is an output)
              part[s2] += p1;
            }
            pf[s2] = u.v;
          }
          rsum = part[0] + part[1];
        };
        weights();
        if (__any(!(rsum <= 65536.f))) {
          float top = sacc[0];
#pragma unroll
          for (int v = 0; v < 16; ++v) top = fmaxf(top, sacc[v]);
          top = fmaxf(top, __shfl_xor(top, 32));
          const float next = fmaxf(mref, top), alpha = __builtin_amdgcn_exp2f((mref - next) * sc);
          mref = next;
          lrun *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
          weights();
        }
        lrun += rsum;
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          const char* const p = vt + 16 * s2 * ROWB;
#pragma unroll
          for (int db = 0; db < DB; ++db) oacc[db] = mfma32(join_tr(read_tr(p + vaddr[db][0]), read_tr(p + vaddr[db][1])), pf[s2], oacc[db]);
        }
      }
      wait_vmcnt<0>();
      lds_barrier();
    }
    lds_barrier();                                  // before the list is filled again
  }

  if (!there) return;
  const float all = lrun + __shfl_xor(lrun, 32), inv = all == 0.f ? 0.f : 1.f / all;
  bf16raw* const out = (bf16raw*)a.o + (long long)(s.q0 + tok) * a.os.token + (long long)head * a.os.head + 4 * hb;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *(uint2*)(out + db * 32 + 8 * x) = uint2{pack_bf16x2(oacc[db][4 * x] * inv, oacc[db][4 * x + 1] * inv), pack_bf16x2(oacc[db][4 * x + 2] * inv, oacc[db][4 * x + 3] * inv)};
  if (hb == 0 && a.lse) a.lse[(long long)(s.q0 + tok) * m.Hq + head] = all == 0.f ? -INFINITY : fmaf(mref, sc, __builtin_amdgcn_logf(all)) * LN2;
}

}  // namespace

// Whether the kernel for many rows takes a call: bf16 keys, more than 32 rows a block (blocks of 40 rows, d = 128 146 us, 204 by block_attn)
// and a workgroup a CU (below, the list has to be split), offsets inside a sixteenth that 32 bits hold.
bool block_wide_takes(const BlockAttnArgs& a, int dtype, int bits) {
  const int rows = a.m.qblock * a.m.G;
  if (dtype != ADACLUSTER_BF16 || bits || rows < 33) return false;
  const int rt = rows <= 64 ? 64 : 128;
  const long long items = (long long)((rows + rt - 1) / rt) * a.m.nb * a.m.Hkv * a.m.B;
  return items >= 256 && a.ks.token < (1 << 25) && a.vs.token < (1 << 25);
}

int launch_block_attn_wide(hipStream_t s, int d, const BlockAttnArgs& a) {
  const int rows = a.m.qblock * a.m.G, rt = rows <= 64 ? 64 : 128, rts = (rows + rt - 1) / rt;
  const long long heads = (long long)a.m.Hkv * a.m.B, grid = xcd_grid(heads, (long long)rts * a.m.nb);
  if (!grid_fits(grid)) return ADACLUSTER_E_UNSUPPORTED;
  const int split = xcd_split(heads);
  if (rt == 64) {
    if (d == 64) block_attn_wide<64, 2><<<(int)grid, 128, 0, s>>>(a, rts, split);
    else block_attn_wide<128, 2><<<(int)grid, 128, 0, s>>>(a, rts, split);
  } else {
    if (d == 64) block_attn_wide<64, 4><<<(int)grid, 256, 0, s>>>(a, rts, split);
    else block_attn_wide<128, 4><<<(int)grid, 256, 0, s>>>(a, rts, split);
  }
  return launched();
}

}  // namespace adac
