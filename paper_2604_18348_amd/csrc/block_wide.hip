// Attention of blocks of many rows over listed pages, bf16: the walk of block_attn with tiles of 32 keys staged once for all waves.
#include "block_wide.h"

namespace adac {

namespace {

template <int D, int NW>
__global__ __launch_bounds__(NW * 64, NW == 4 ? 3 : 2) void block_attn_wide(BlockAttnArgs a, int rts, int split) {
  __shared__ WideLds<D, NW, false> sh;
  wide_rows<D, NW, false, false>(a, rts, split, sh);
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
