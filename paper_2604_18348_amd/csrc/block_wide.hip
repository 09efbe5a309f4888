// Attention of blocks of many rows over listed pages, bf16: the walk of block_attn with tiles of 32 keys staged once for all waves.
#include "block_wide.h"

namespace adac {

namespace {

// NW waves of 32 rows each.  A tile's keys and values go global -> LDS directly, 16 bytes a lane, one tile ahead of the products.  Rows past
// a sequence's end are read from the last row there is in their sixteenth (or the page's first) and masked: nothing behind the end is
// touched.  Bound by what lies between the products (exponentials, roundings, LDS reads), so waves a SIMD count: tiles of 32 keys and three
// waves (two with NW = 2) against 64 keys and two, or one: 3 sequences up to 8 192 tokens, 32 pages of 64, 16 / 4 heads, d = 128 385 us
// (489), 17 776 tokens, 30 heads, d = 64 730 (744), chunks of 2 x 1 024 tokens, NW = 2, d = 128 193 (303).
template <int D, int NW, Rows ROWS = Rows::OWN>
__global__ __launch_bounds__(NW * 64, NW == 4 ? 3 : 2) void block_attn_wide(BlockAttnArgs a, int rts, int split) {
  constexpr int NT = NW * 64, KS = D / 16, DB = D / 32, CH = D / 8, ROWB = D * 2;
  constexpr int TK = 32, PARTS = TK / 16;      // keys a tile: one product's rows
  constexpr int PT = TK * CH / NT, TILEB = TK * ROWB;
  constexpr int STAGES = ROWS == Rows::OWN ? 2 : 3;
  __shared__ __align__(16) char lds[STAGES * 2 * TILEB];
  __shared__ int2 pages_l[LIST];
  __shared__ int32_t counts[NW];
  const BlockDims& m = a.m;
  // (GROUP: rts tiles; a share of the keys is walked by all tiles side by side)
  const HeadItem it = ROWS == Rows::OWN ? xcd_item(blockIdx.x, m.B * m.Hkv, m.nb * rts, split) : xcd_item(blockIdx.x, m.Hkv, rts * a.nsplit, split);
  if (it.head < 0) return;
  const int rt = it.item % rts, i = it.item / rts, hk = it.head % m.Hkv;
  int b = it.head / m.Hkv, t0 = 0, rows, base_row, from = 0, to = INT32_MAX;
  BlockSeq s;
  Group group;
  if constexpr (ROWS == Rows::GROUP) {
    const int g = last_group(a.gr.groups, [&](int x) { return first_tile(m, group_at(m, a.gr, x).q0, x, NT / 2) <= rt; });
    if (g < 0) return;
    group = group_at(m, a.gr, g);
    b = group.b0;
    base_row = (rt - first_tile(m, group.q0, g, NT / 2)) * (NT / 2);
    rows = (group.q1 - group.q0) * m.G;
    s = BlockSeq{group.q0, group.q1 - group.q0, 0, group.pages << m.lpage, 0};
    const int shares = splits_of(m, group.pages, a.nsplit, NT / 2);
    if (base_row < 0 || base_row >= rows || i >= shares) return;      // (below 0: groups that do not ascend)
    from = (int)((long long)group.pages * i / shares);
    to = (int)((long long)group.pages * (i + 1) / shares);
  } else {
    s = block_seq(m, b);
    t0 = i * m.qblock; rows = min(m.qblock, s.nq - t0) * m.G; base_row = rt * NT / 2;
    if (t0 >= s.nq || base_row >= rows) return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, hb = lane >> 5;

  const int row = base_row + wave * 32 + c, tok = t0 + row / m.G, head = hk * m.G + row % m.G;
  const int group_lim = ROWS == Rows::GROUP && row < rows ? row_limit(m, group, s.q0 + tok) : -1;
  const bool there = ROWS == Rows::GROUP ? group_lim >= 0 : row < rows;
  bf16x8_t qf[KS];
  {
    const bf16raw* const p = (const bf16raw*)a.q + (long long)(s.q0 + tok) * a.qs.token + (long long)head * a.qs.head + hb * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4_t w = there ? *(const u32x4_t*)(p + ks * 16) : u32x4_t{0, 0, 0, 0};
      qf[ks] = *(const bf16x8_t*)&w;
    }
  }
  const int lim = there ? (ROWS == Rows::GROUP ? group_lim : m.causal ? min(s.n, s.first + tok + 1) : s.n) : INT32_MAX;      // (a row that is not there needs no mask)
  const int wave_first = base_row + wave * 32;
  const bool wave_has_rows = wave_first < rows;
  int minlim = m.causal ? min(s.n, s.first + t0 + wave_first / m.G + 1) : s.n;       // keys below: seen by all rows of the wave
  const int last = min(base_row + NT / 2, rows) - 1;
  int maxlim = m.causal ? min(s.n, s.first + t0 + last / m.G + 1) : s.n;
  if constexpr (ROWS == Rows::GROUP) {
    int low = lim;
#pragma unroll
    for (int x = 1; x < 32; x *= 2) low = min(low, __shfl_xor(low, x));
    minlim = uniform(low); maxlim = s.n;
  }
  const int pages = maxlim > 0 ? (maxlim + m.page - 1) >> m.lpage : 0;
  const int32_t* const list = ROWS == Rows::OWN && a.sel ? a.sel + (((long long)b * m.nb + i) * m.Hkv + hk) * m.topk : nullptr;
  const int entries = list ? m.topk : min(pages, to);

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

  for (int e0 = from; e0 < entries; e0 += LIST) {
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
    if constexpr (STAGES == 2) {
      wait_vmcnt<0>();
      lds_barrier();
    } else if (tiles > 1) {
      issue(1, 1);
    }
    int stage = 0;
    for (int t = 0; t < tiles; ++t) {
      if constexpr (STAGES == 2) {
        if (t + 1 < tiles) issue((t + 1) & 1, t + 1);
        stage = t & 1;
      } else {                                      // two tiles on their way: the prefix of one group waits for memory, not for products
        if (t + 1 < tiles) wait_vmcnt<2 * PT>();
        else wait_vmcnt<0>();
        lds_barrier();
        if (t) stage = stage == 2 ? 0 : stage + 1;
        if (t + 2 < tiles) issue(stage == 0 ? 2 : stage - 1, t + 2);
      }
      if (wave_has_rows) {
        const char* const kt = lds + stage * 2 * TILEB;
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
      if constexpr (STAGES == 2) {
        wait_vmcnt<0>();
        lds_barrier();
      }
    }
    lds_barrier();                                  // before the list is filled again
  }

  if (!there) return;
  const float all = lrun + __shfl_xor(lrun, 32), inv = all == 0.f ? 0.f : 1.f / all;
  if constexpr (ROWS == Rows::GROUP) {
    const long long rec = (((long long)rt * m.Hkv + hk) * a.nsplit + i) * (NT / 2) + wave * 32 + c;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        *(f32x4_t*)(a.part_o + rec * D + db * 32 + 8 * x + 4 * hb) = f32x4_t{oacc[db][4 * x], oacc[db][4 * x + 1], oacc[db][4 * x + 2], oacc[db][4 * x + 3]};
    if (hb == 0) { a.part_ml[rec * 2] = mref * sc; a.part_ml[rec * 2 + 1] = all; }
    return;
  }
  bf16raw* const out = (bf16raw*)a.o + (long long)(s.q0 + tok) * a.os.token + (long long)head * a.os.head + 4 * hb;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 4; ++x)
      *(uint2*)(out + db * 32 + 8 * x) = uint2{pack_bf16x2(oacc[db][4 * x] * inv, oacc[db][4 * x + 1] * inv), pack_bf16x2(oacc[db][4 * x + 2] * inv, oacc[db][4 * x + 3] * inv)};
  if (hb == 0 && a.lse) a.lse[(long long)(s.q0 + tok) * m.Hq + head] = all == 0.f ? -INFINITY : fmaf(mref, sc, __builtin_amdgcn_logf(all)) * LN2;
}

// The same walk over 4-bit pages for the rows of a group.  A tile's codes come one tile ahead into registers and go to LDS as bfloat16: those
// of keys by themselves, those of values less 8.  Per group g of 64 dimensions
//   scores   sum of step_g (c . q) + low_g sum q, scaled: the latter one more product, of (low, low, low) with three bfloat16 parts of sum q;
//   values   weights times step_g, rounded to bfloat16, times c - 8 (a rounding weighs codes about their middle), and the sum of weights
//            times low_g + 8 step_g, unrounded.
// Steps are applied to 16 keys a lane, which reads them from LDS: with them LDS is what bounds it (24 of 48 wide reads a tile).
template <int D, int NW>
__global__ __launch_bounds__(NW * 64, 2) void block_attn_wide_codes(BlockAttnArgs a, int tiles, int split) {
  constexpr int NT = NW * 64, KS = D / 16, DB = D / 32, NG = D / 64, ROWB = D * 2, WORDS = D / 8;      // words of eight codes a row
  constexpr int TK = 32, PT = TK * WORDS / NT, TILEB = TK * ROWB;
  __shared__ __align__(16) char lds[4 * TILEB];
  __shared__ __align__(16) float kstep_l[2][NG][TK], vstep_l[2][NG][TK], vlow_l[2][NG][TK];
  __shared__ uint32_t klow_l[2][TK][NG];
  __shared__ int2 pages_l[LIST];
  __shared__ int32_t counts[NW];
  const BlockDims& m = a.m;
  const HeadItem it = xcd_item(blockIdx.x, m.Hkv, tiles * a.nsplit, split);
  if (it.head < 0) return;
  const int rt = it.item % tiles, share = it.item / tiles, hk = it.head;
  const int g = last_group(a.gr.groups, [&](int x) { return first_tile(m, group_at(m, a.gr, x).q0, x, NT / 2) <= rt; });
  if (g < 0) return;
  const Group group = group_at(m, a.gr, g);
  const int b = group.b0, base_row = (rt - first_tile(m, group.q0, g, NT / 2)) * (NT / 2), rows = (group.q1 - group.q0) * m.G;
  const int shares = splits_of(m, group.pages, a.nsplit, NT / 2);
  if (base_row < 0 || base_row >= rows || share >= shares) return;      // (below 0: groups that do not ascend)
  const int from = (int)((long long)group.pages * share / shares), to = (int)((long long)group.pages * (share + 1) / shares);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, hb = lane >> 5;

  const int row = base_row + wave * 32 + c, tok = row / m.G, head = hk * m.G + row % m.G;
  const int group_lim = row < rows ? row_limit(m, group, group.q0 + tok) : -1;
  const bool there = group_lim >= 0;
  const int lim = there ? group_lim : INT32_MAX;
  const float sc = a.scale_log2e;
  bf16x8_t qf[KS], qsum;
  {
    const bf16raw* const p = (const bf16raw*)a.q + (long long)(group.q0 + tok) * a.qs.token + (long long)head * a.qs.head + hb * 8;
    float s[NG];
#pragma unroll
    for (int x = 0; x < NG; ++x) s[x] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const u32x4_t w = there ? *(const u32x4_t*)(p + ks * 16) : u32x4_t{0, 0, 0, 0};
      qf[ks] = *(const bf16x8_t*)&w;
#pragma unroll
      for (int j = 0; j < 4; ++j) s[ks / 4] += __uint_as_float(w[j] << 16) + __uint_as_float(w[j] & 0xFFFF0000u);
    }
    uint32_t h[6] = {0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int x = 0; x < NG; ++x) {
      float v = (s[x] + __shfl_xor(s[x], 32)) * sc;
#pragma unroll
      for (int y = 0; y < 3; ++y) { h[3 * x + y] = __float_as_uint(v) >> 16; v -= __uint_as_float(h[3 * x + y] << 16); }      // (cut: what is left is exact)
    }
    union { uint32_t w[4]; bf16x8_t v; } u{{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, 0}};
    if (hb) u.w[0] = u.w[1] = u.w[2] = 0;
    qsum = u.v;
  }
  const bool wave_has_rows = base_row + wave * 32 < rows;
  int minlim = lim;
#pragma unroll
  for (int x = 1; x < 32; x *= 2) minlim = min(minlim, __shfl_xor(minlim, x));
  minlim = uniform(minlim);

  f32x16_t oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) oacc[db] = zero16();
  // The weights are taken relative to a reference (scaled here) that moves only when a tile's sum leaves its range, as above.
  float mref = -3.4028e38f, lrun = 0.f, corr[NG];
#pragma unroll
  for (int x = 0; x < NG; ++x) corr[x] = 0.f;

  int kaddr[KS], vaddr[DB][2];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) kaddr[ks] = row_operand<D>(lane, ks);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 2; ++x) vaddr[db][x] = col_operand<D>(lane, db, x);

  const int lsub = m.lpage - 4;
  for (int e0 = from; e0 < to; e0 += LIST) {
    const int n = fill_list<NT>(m, b, nullptr, e0, 1, to, to, pages_l, counts);
    const int parts = n << lsub, count = (parts + 1) / 2;
    if (!count) continue;
    uint32_t kc[PT], vc[PT], pair[(2 * TK * NG + NT - 1) / NT];
    const auto fetch = [&](int t) __attribute__((always_inline)) {      // (past the end: the last sixteenth again, masked)
#pragma unroll
      for (int x = 0; x < PT; ++x) {
        const int item = tid + x * NT, r = item / WORDS, part = min(t * 2 + (r >> 4), parts - 1);
        const int2 pp = pages_l[part >> lsub];
        const long long at = ((((long long)pp.y * m.Hkv + hk) << m.lpage) + (part & ((1 << lsub) - 1)) * 16 + (r & 15)) * WORDS + item % WORDS;
        kc[x] = ((const uint32_t*)a.k)[at];
        vc[x] = ((const uint32_t*)a.v)[at];
      }
#pragma unroll
      for (int x = 0; x < (2 * TK * NG + NT - 1) / NT; ++x) {          // a pair of a key or value and group a thread
        const int item = tid + x * NT, r = item / NG % TK, part = min(t * 2 + (r >> 4), parts - 1);
        if (item >= 2 * TK * NG) break;
        const int2 pp = pages_l[part >> lsub];
        const long long at = (((((long long)pp.y * m.Hkv + hk) << m.lpage) + (part & ((1 << lsub) - 1)) * 16 + (r & 15)) * NG) + item % NG;
        pair[x] = (item < TK * NG ? a.km : a.vm)[at];
      }
    };
    const auto expand = [&](int stage) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < PT; ++x) {
        const int item = tid + x * NT, r = item / WORDS, at = r * ROWB + ((item % WORDS) ^ swz<D>(r)) * 16;
        u32x4_t k, v;
        const uint32_t even = kc[x] & 0x0F0F0F0Fu, odd = kc[x] >> 4 & 0x0F0F0F0Fu, mid = vc[x] ^ 0x88888888u;      // (a code less 8: four bits with a sign)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          k[j] = __float_as_uint((float)(even >> (8 * j) & 255)) >> 16 | __float_as_uint((float)(odd >> (8 * j) & 255));
          v[j] = __float_as_uint((float)((int)(mid << (28 - 8 * j)) >> 28)) >> 16 | __float_as_uint((float)((int)(mid << (24 - 8 * j)) >> 28));
        }
        *(u32x4_t*)(lds + stage * 2 * TILEB + at) = k;
        *(u32x4_t*)(lds + stage * 2 * TILEB + TILEB + at) = v;
      }
#pragma unroll
      for (int x = 0; x < (2 * TK * NG + NT - 1) / NT; ++x) {
        const int item = tid + x * NT, r = item / NG % TK, gr = item % NG;
        if (item >= 2 * TK * NG) break;
        const float step = __uint_as_float(pair[x] << 16), low = __uint_as_float(pair[x] & 0xFFFF0000u);
        if (item < TK * NG) { kstep_l[stage][gr][r] = step * sc; klow_l[stage][r][gr] = pair[x] >> 16; }
        else { vstep_l[stage][gr][r] = step; vlow_l[stage][gr][r] = fmaf(8.f, step, low); }
      }
    };
    fetch(0);
    expand(0);
    __syncthreads();
    for (int t = 0; t < count; ++t) {
      const int stage = t & 1;
      if (t + 1 < count) fetch(t + 1);
      if (wave_has_rows) {
        const char* const kt = lds + stage * 2 * TILEB;
        const char* const vt = kt + TILEB;
        f32x16_t sacc;
        {
          const uint32_t l0 = klow_l[stage][c][0], l1 = NG == 2 ? klow_l[stage][c][NG - 1] : 0;
          union { uint32_t w[4]; bf16x8_t v; } u{{l0 | l0 << 16, l0 | l1 << 16, l1 | l1 << 16, 0}};
          sacc = mfma32(u.v, qsum, zero16());
          f32x16_t y[NG];
#pragma unroll
          for (int x = 0; x < NG; ++x) {
            y[x] = zero16();
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) y[x] = mfma32(*(const bf16x8_t*)(kt + kaddr[4 * x + ks]), qf[4 * x + ks], y[x]);
          }
#pragma unroll
          for (int x = 0; x < NG; ++x)
#pragma unroll
            for (int z = 0; z < 4; ++z) {
              const f32x4_t step = *(const f32x4_t*)&kstep_l[stage][x][8 * z + 4 * hb];
#pragma unroll
              for (int j = 0; j < 4; ++j) sacc[4 * z + j] = fmaf(step[j], y[x][4 * z + j], sacc[4 * z + j]);
            }
        }
        int key0[2];
        bool whole = true;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int part = t * 2 + x, pg = uniform(pages_l[min(part, parts - 1) >> lsub].x);
          key0[x] = part < parts ? (pg << m.lpage) + (part & ((1 << lsub) - 1)) * 16 : INT32_MAX - 64;
          whole = whole && key0[x] + 16 <= minlim;
        }
        if (!whole) {
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (key0[v >> 3] + 8 * ((v >> 2) & 1) + 4 * hb + (v & 3) >= lim) sacc[v] = -INFINITY;
        }
        float p[16], rsum;
        const auto weights = [&]() __attribute__((always_inline)) {
          float part[2] = {0.f, 0.f};
#pragma unroll
          for (int v = 0; v < 16; ++v) { p[v] = __builtin_amdgcn_exp2f(sacc[v] - mref); part[v >> 3] += p[v]; }
          rsum = part[0] + part[1];
        };
        weights();
        if (__any(!(rsum <= 65536.f))) {
          float top = sacc[0];
#pragma unroll
          for (int v = 0; v < 16; ++v) top = fmaxf(top, sacc[v]);
          top = fmaxf(top, __shfl_xor(top, 32));
          const float next = fmaxf(mref, top), alpha = __builtin_amdgcn_exp2f(mref - next);
          mref = next;
          lrun *= alpha;
#pragma unroll
          for (int x = 0; x < NG; ++x) corr[x] *= alpha;
#pragma unroll
          for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
          weights();
        }
        lrun += rsum;
#pragma unroll
        for (int x = 0; x < NG; ++x) {
          bf16x8_t pf[2];
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2) {
            union { uint32_t w[4]; bf16x8_t v; } u;
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const int at = 16 * s2 + 8 * z + 4 * hb, v0 = 8 * s2 + 4 * z;
              const f32x4_t step = *(const f32x4_t*)&vstep_l[stage][x][at], low = *(const f32x4_t*)&vlow_l[stage][x][at];
#pragma unroll
              for (int j = 0; j < 2; ++j) u.w[2 * z + j] = pack_bf16x2(p[v0 + 2 * j] * step[2 * j], p[v0 + 2 * j + 1] * step[2 * j + 1]);
#pragma unroll
              for (int j = 0; j < 4; ++j) corr[x] = fmaf(p[v0 + j], low[j], corr[x]);
            }
            pf[s2] = u.v;
          }
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2) {
            const char* const q = vt + 16 * s2 * ROWB;
#pragma unroll
            for (int db = 2 * x; db < 2 * x + 2; ++db) oacc[db] = mfma32(join_tr(read_tr(q + vaddr[db][0]), read_tr(q + vaddr[db][1])), pf[s2], oacc[db]);
          }
        }
      }
      if (t + 1 < count) expand(stage ^ 1);
      __syncthreads();
    }
  }

  if (!there) return;
  const float all = lrun + __shfl_xor(lrun, 32);
#pragma unroll
  for (int x = 0; x < NG; ++x) corr[x] += __shfl_xor(corr[x], 32);
  const long long rec = (((long long)rt * m.Hkv + hk) * a.nsplit + share) * (NT / 2) + wave * 32 + c;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      f32x4_t o;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = oacc[db][4 * x + j] + corr[db / 2];
      *(f32x4_t*)(a.part_o + rec * D + db * 32 + 8 * x + 4 * hb) = o;
    }
  if (hb == 0) { a.part_ml[rec * 2] = mref; a.part_ml[rec * 2 + 1] = all; }
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

void launch_block_attn_wide_part(hipStream_t s, int bits, int d, int TR, int tiles, const BlockAttnArgs& a) {
  const int grid = (int)xcd_grid(a.m.Hkv, (long long)tiles * a.nsplit), split = xcd_split(a.m.Hkv);
  if (bits) {
    if (TR == 64) {
      if (d == 64) block_attn_wide_codes<64, 2><<<grid, 128, 0, s>>>(a, tiles, split);
      else block_attn_wide_codes<128, 2><<<grid, 128, 0, s>>>(a, tiles, split);
    } else {
      if (d == 64) block_attn_wide_codes<64, 4><<<grid, 256, 0, s>>>(a, tiles, split);
      else block_attn_wide_codes<128, 4><<<grid, 256, 0, s>>>(a, tiles, split);
    }
    return;
  }
  if (TR == 64) {
    if (d == 64) block_attn_wide<64, 2, Rows::GROUP><<<grid, 128, 0, s>>>(a, tiles, split);
    else block_attn_wide<128, 2, Rows::GROUP><<<grid, 128, 0, s>>>(a, tiles, split);
  } else {
    if (d == 64) block_attn_wide<64, 4, Rows::GROUP><<<grid, 256, 0, s>>>(a, tiles, split);
    else block_attn_wide<128, 4, Rows::GROUP><<<grid, 256, 0, s>>>(a, tiles, split);
  }
}

}  // namespace adac
