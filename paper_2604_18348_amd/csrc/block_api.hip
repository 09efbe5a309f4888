// C ABI of attention over pages of keys: argument checks and the order of the launches.  Everything that lies in device memory
// (lengths, page tables, lists) is checked where it is read, by the kernels.
#include "block.h"
#include "launch.h"

#include <math.h>

using namespace adac;

namespace {

bool shifted(int v, int* l) { for (*l = 4; *l <= 7; ++*l) if (v == 1 << *l) return true; return false; }

// dims common to all calls
int check(const adacluster_block_params* p, BlockDims* m) {
  if (!p) return fail(ADACLUSTER_E_BADARG, "params is NULL");
  if (p->B < 1 || p->B > 65535) return fail(ADACLUSTER_E_BADSHAPE, "B must be in [1,65535] (B=%d)", p->B);
  if (p->Hkv < 1 || p->Hkv > 4096 || p->Hq < 1 || p->Hq > 65535 || p->Hq % p->Hkv)
    return fail(ADACLUSTER_E_BADSHAPE, "Hq must be a multiple of Hkv (Hq=%d Hkv=%d)", p->Hq, p->Hkv);
  if (p->d != 64 && p->d != 128) return fail(ADACLUSTER_E_BADSHAPE, "d must be 64 or 128 (d=%d)", p->d);
  if (p->dtype != ADACLUSTER_F32 && p->dtype != ADACLUSTER_BF16) return fail(ADACLUSTER_E_BADDTYPE, "unknown dtype %d", p->dtype);
  if (p->bits != 0 && p->bits != 4) return fail(ADACLUSTER_E_BADDTYPE, "bits must be 0 (as dtype) or 4 (bits=%d)", p->bits);
  if (!shifted(p->page, &m->lpage)) return fail(ADACLUSTER_E_BADSHAPE, "page must be 16, 32, 64 or 128 (page=%d)", p->page);
  if (p->num_pages < 0) return fail(ADACLUSTER_E_BADSHAPE, "num_pages must be >= 0");
  if (p->max_pages < 1 || (long long)p->max_pages * p->page > (1 << 29)) return fail(ADACLUSTER_E_BADSHAPE, "max_pages must be >= 1, and max_pages * page <= 2^29 (max_pages=%d)", p->max_pages);
  if (p->max_q < 1 || p->max_q > (1 << 29)) return fail(ADACLUSTER_E_BADSHAPE, "max_q must be in [1,2^29] (max_q=%d)", p->max_q);
  if (p->qblock < 1 || p->qblock > 1024) return fail(ADACLUSTER_E_BADSHAPE, "qblock must be in [1,1024] (qblock=%d)", p->qblock);
  if (p->causal != 0 && p->causal != 1) return fail(ADACLUSTER_E_BADARG, "causal must be 0 or 1");
  if (p->topk < 0 || p->topk > (1 << 24)) return fail(ADACLUSTER_E_BADARG, "topk must be in [0,2^24] (topk=%d)", p->topk);
  if (p->keep_first < 0) return fail(ADACLUSTER_E_BADARG, "keep_first must be >= 0");
  if (p->q_rows < 1 || p->k_rows < 0) return fail(ADACLUSTER_E_BADSHAPE, "q_rows must be >= 1 and k_rows >= 0");
  if (!(p->softmax_scale < 0x1p100f)) return fail(ADACLUSTER_E_BADARG, "softmax_scale must be below 2^100");
  if (((long long)p->max_q + p->qblock - 1) / p->qblock * p->Hkv > (1ll << 31) / p->B)
    return fail(ADACLUSTER_E_BADSHAPE, "more than 2^31 blocks of queries (B * Hkv * max_q / qblock)");
  m->B = p->B; m->Hq = p->Hq; m->Hkv = p->Hkv; m->G = p->Hq / p->Hkv;
  m->page = p->page; m->num_pages = p->num_pages; m->max_pages = p->max_pages;
  m->max_q = p->max_q; m->qblock = p->qblock; m->nb = (p->max_q + p->qblock - 1) / p->qblock;
  m->causal = p->causal; m->topk = p->topk; m->keep_first = p->keep_first;
  m->q_rows = p->q_rows; m->k_rows = p->k_rows;
  m->cu_q = m->cu_k = m->seq_lens = m->table = nullptr;
  return 0;
}

int check_list(const BlockDims& m) {
  if (m.topk < 1) return fail(ADACLUSTER_E_BADARG, "topk must be >= 1 for lists of pages");
  const int own = m.causal ? (m.qblock - 1 + m.page - 1) / m.page + 1 : 0;
  if ((long long)m.keep_first + own > m.topk)
    return fail(ADACLUSTER_E_BADARG, "topk must hold the first pages and those of the block's own positions: %d + %d > %d", m.keep_first, own, m.topk);
  return 0;
}

// where the keys are: a paged cache or packed rows
int check_keys(BlockDims* m, const int32_t* cu_k, const int32_t* seq_lens, const int32_t* table) {
  if (m->num_pages) {
    if (!seq_lens || !table) return fail(ADACLUSTER_E_BADARG, "a paged cache needs seq_lens and page_table");
  } else {
    if (!cu_k) return fail(ADACLUSTER_E_BADARG, "packed keys need cu_k (num_pages is 0)");
    if (m->k_rows < 1) return fail(ADACLUSTER_E_BADSHAPE, "packed keys need k_rows >= 1");
  }
  m->cu_k = cu_k; m->seq_lens = seq_lens; m->table = table;
  return 0;
}

bool apart(const void* a, size_t na, const void* b, size_t nb) { return (uintptr_t)a + na <= (uintptr_t)b || (uintptr_t)b + nb <= (uintptr_t)a; }

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// 16-byte rows: the base and every stride that is used
int check_rows(const char* name, const void* p, int dtype, const KeyStride& s) {
  if (!p) return fail(ADACLUSTER_E_BADARG, "%s is NULL", name);
  const int n = dtype == ADACLUSTER_BF16 ? 8 : 4;
  if (!aligned(p, 16) || s.page % n || s.token % n || s.head % n)
    return fail(ADACLUSTER_E_BADARG, "%s: rows must start at multiples of 16 bytes (base and strides)", name);
  if (s.page < 0 || s.token < 0 || s.head < 0) return fail(ADACLUSTER_E_BADARG, "%s: strides must not be negative", name);
  return 0;
}

KeyStride two(const int64_t* s) { return {0, s[0], s[1]}; }
KeyStride three(const BlockDims& m, const int64_t* s) { return {m.num_pages ? s[0] : 0, s[1], s[2]}; }

int check_pool(const adacluster_block_params* p, const void* k, const void* v, const uint32_t* km, const uint32_t* vm, const KeyStride& ks, const KeyStride& vs) {
  if (p->bits == 4) {
    if (!p->num_pages) return fail(ADACLUSTER_E_UNSUPPORTED, "4-bit keys are those of a paged cache (num_pages > 0)");
    if (!k || !v || !km || !vm) return fail(ADACLUSTER_E_BADARG, "a 4-bit cache has codes and (step, lowest) pairs for keys and values: one is NULL");
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(km, 16) || !aligned(vm, 16)) return fail(ADACLUSTER_E_BADARG, "a 4-bit cache starts at multiples of 16 bytes");
    return 0;
  }
  if (int rc = check_rows("k", k, p->dtype, ks)) return rc;
  return check_rows("v", v, p->dtype, vs);
}

int check_ws(void* ws, size_t have, size_t need) {
  if (!need) return 0;
  if (!ws) return fail(ADACLUSTER_E_WORKSPACE, "workspace is NULL");
  if (!aligned(ws, 256)) return fail(ADACLUSTER_E_WORKSPACE, "workspace must be 256-byte aligned");
  if (have < need) return fail(ADACLUSTER_E_WORKSPACE, "workspace too small: %zu < %zu bytes", have, need);
  return 0;
}

int done(int rc) {
  if (rc == ADACLUSTER_E_INTERNAL) return fail(rc, "HIP launch failed: %s", hipGetErrorString(hipGetLastError()));
  if (rc == ADACLUSTER_E_UNSUPPORTED) return fail(rc, "the call needs more workgroups than a launch may have: fewer sequences, queries or pages a call");
  return rc;
}

// Without lists nothing hangs on the blocks: as many queries as fill a workgroup's 128 rows (2 x 512 tokens over 16 384 keys, 32 / 8 heads:
// 603 us, in blocks of 16 queries 769; 8 heads, d = 64 103, 221).
BlockDims unlisted(BlockDims m) {
  m.qblock = m.G >= 128 ? 1 : 128 / m.G;
  if (m.qblock > m.max_q) m.qblock = m.max_q;
  m.nb = (m.max_q + m.qblock - 1) / m.qblock;
  return m;
}

double scale_of(const adacluster_block_params* p) { return p->softmax_scale > 0.f ? p->softmax_scale : 1.0 / sqrt((double)p->d); }
float log2_scale(const adacluster_block_params* p) { return (float)(scale_of(p) * 1.4426950408889634); }      // (rounded once: logits of 20 feel it)

// rows of a head of keys: their numbers, and those of the rows past the last that its tile or stage goes on with, are 32 bits
constexpr long long MOST_ROWS = (1ll << 31) - 1024;

// what the shape of a call of prefix_attn follows from
int prefix_args(const adacluster_block_params* p, int32_t groups, PrefixArgs* a) {
  if (int rc = check(p, &a->m)) return rc;
  if (!p->num_pages) return fail(ADACLUSTER_E_BADARG, "prefix_attn: num_pages must be >= 1 (a paged cache)");
  if (groups < 0 || groups > p->B) return fail(ADACLUSTER_E_BADSHAPE, "groups must be in [0,B] (groups=%d)", groups);
  if ((long long)p->q_rows * a->m.G > MOST_ROWS) return fail(ADACLUSTER_E_UNSUPPORTED, "prefix_attn: q_rows * Hq / Hkv must be at most 2^31 - 1024");
  a->m = unlisted(a->m);
  a->gr.groups = groups;
  a->qs = two(p->q_stride); a->os = two(p->o_stride); a->ks = three(a->m, p->k_stride); a->vs = three(a->m, p->v_stride);
  return 0;
}

}  // namespace

extern "C" {

int adacluster_block_workspace_bytes(const adacluster_block_params* p, int32_t call, size_t* bytes) {
  BlockDims m;
  if (int rc = check(p, &m)) return rc;
  if (!bytes) return fail(ADACLUSTER_E_BADARG, "bytes is NULL");
  if (call == ADACLUSTER_BLOCK_SELECT) *bytes = block_select_bytes(m, p->dtype);
  else if (call == ADACLUSTER_BLOCK_ATTN) {
    const size_t x = block_attn_bytes(m, p->d, true), y = block_attn_bytes(unlisted(m), p->d, false);
    *bytes = p->topk > 0 && x > y ? x : y;
  } else if (call == ADACLUSTER_BLOCK_BACKWARD) {
    const size_t x = block_grad_bytes(m, p->dtype, p->d, true), y = block_grad_bytes(unlisted(m), p->dtype, p->d, false);
    *bytes = p->topk > 0 && x > y ? x : y;
  }
  else return fail(ADACLUSTER_E_BADARG, "unknown call %d", call);
  return 0;
}

int adacluster_cache_append(const adacluster_block_params* p, const void* k, const void* v, const int32_t* cu_new, const int32_t* seq_lens,
                            const int32_t* page_table, void* k_pool, void* v_pool, uint32_t* k_meta, uint32_t* v_meta, void* boxes, void* stream) {
  CacheArgs a{};
  if (int rc = check(p, &a.m)) return rc;
  if (!p->num_pages) return fail(ADACLUSTER_E_BADARG, "cache_append: num_pages must be >= 1");
  if (!cu_new || !boxes) return fail(ADACLUSTER_E_BADARG, "cache_append: NULL tensor pointer");
  if (int rc = check_keys(&a.m, nullptr, seq_lens, page_table)) return rc;
  a.m.cu_q = cu_new;
  a.new_k = two(p->new_k_stride); a.new_v = two(p->new_v_stride); a.ks = three(a.m, p->k_stride); a.vs = three(a.m, p->v_stride);
  if (int rc = check_rows("new keys", k, p->dtype, a.new_k)) return rc;
  if (int rc = check_rows("new values", v, p->dtype, a.new_v)) return rc;
  if (int rc = check_pool(p, k_pool, v_pool, k_meta, v_meta, a.ks, a.vs)) return rc;
  a.k = k; a.v = v; a.kp = k_pool; a.vp = v_pool; a.km = k_meta; a.vm = v_meta; a.boxes = boxes;
  return done(launch_cache_append((hipStream_t)stream, p->dtype, p->bits, p->d, a));
}

int adacluster_cache_read(const adacluster_block_params* p, const int32_t* cu_new, const int32_t* first, const int32_t* page_table,
                          const void* k_pool, const void* v_pool, const uint32_t* k_meta, const uint32_t* v_meta, void* k, void* v, void* stream) {
  CacheArgs a{};
  if (int rc = check(p, &a.m)) return rc;
  if (!p->num_pages) return fail(ADACLUSTER_E_BADARG, "cache_read: num_pages must be >= 1");
  if (!cu_new) return fail(ADACLUSTER_E_BADARG, "cache_read: NULL tensor pointer");
  if (int rc = check_keys(&a.m, nullptr, first, page_table)) return rc;
  a.m.cu_q = cu_new;
  a.ks = three(a.m, p->k_stride); a.vs = three(a.m, p->v_stride);
  const KeyStride whole{0, 0, 0};
  if (int rc = check_rows("k", k, p->dtype, whole)) return rc;
  if (int rc = check_rows("v", v, p->dtype, whole)) return rc;
  if (int rc = check_pool(p, k_pool, v_pool, k_meta, v_meta, a.ks, a.vs)) return rc;
  a.kp = (void*)k_pool; a.vp = (void*)v_pool; a.km = (uint32_t*)k_meta; a.vm = (uint32_t*)v_meta; a.ko = k; a.vo = v;
  return done(launch_cache_read((hipStream_t)stream, p->dtype, p->bits, p->d, a));
}

int adacluster_block_boxes(const adacluster_block_params* p, const void* k, const int32_t* cu_k, void* boxes, void* stream) {
  BlockDims m;
  if (int rc = check(p, &m)) return rc;
  if (p->num_pages) return fail(ADACLUSTER_E_BADARG, "block_boxes: packed keys only (num_pages must be 0; adacluster_cache_append keeps the boxes of a cache)");
  if (!boxes) return fail(ADACLUSTER_E_BADARG, "block_boxes: NULL tensor pointer");
  if (int rc = check_keys(&m, cu_k, nullptr, nullptr)) return rc;
  const KeyStride ks = three(m, p->k_stride);
  if (int rc = check_rows("k", k, p->dtype, ks)) return rc;
  return done(launch_block_boxes((hipStream_t)stream, p->dtype, p->d, m, k, ks, boxes));
}

int adacluster_block_select(const adacluster_block_params* p, const void* q, const int32_t* cu_q, const int32_t* cu_k, const int32_t* seq_lens,
                            const int32_t* page_table, const void* boxes, int32_t* sel_idx, int32_t* sel_cnt, void* ws, size_t ws_bytes, void* stream) {
  BlockDims m;
  if (int rc = check(p, &m)) return rc;
  if (int rc = check_list(m)) return rc;
  if (!cu_q || !boxes || !sel_idx || !sel_cnt) return fail(ADACLUSTER_E_BADARG, "block_select: NULL tensor pointer");
  if (!aligned(boxes, 16)) return fail(ADACLUSTER_E_BADARG, "block_select: boxes must start at a multiple of 16 bytes");
  if (int rc = check_keys(&m, cu_k, seq_lens, page_table)) return rc;
  m.cu_q = cu_q;
  const KeyStride qs = two(p->q_stride);
  if (int rc = check_rows("q", q, p->dtype, qs)) return rc;
  if (int rc = check_ws(ws, ws_bytes, block_select_bytes(m, p->dtype))) return rc;
  return done(launch_block_select((hipStream_t)stream, p->dtype, p->d, m, q, qs, boxes, sel_idx, sel_cnt, ws));
}

int adacluster_block_attn(const adacluster_block_params* p, const void* q, const int32_t* cu_q, const void* k, const void* v, const uint32_t* k_meta,
                          const uint32_t* v_meta, const int32_t* cu_k, const int32_t* seq_lens, const int32_t* page_table, const int32_t* sel_idx,
                          void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  BlockAttnArgs a{};
  if (int rc = check(p, &a.m)) return rc;
  if (sel_idx && p->topk < 1) return fail(ADACLUSTER_E_BADARG, "topk must be >= 1 for lists of pages");
  if (!cu_q) return fail(ADACLUSTER_E_BADARG, "block_attn: NULL tensor pointer");
  if (int rc = check_keys(&a.m, cu_k, seq_lens, page_table)) return rc;
  a.m.cu_q = cu_q;
  if (!sel_idx) a.m = unlisted(a.m);
  a.qs = two(p->q_stride); a.os = two(p->o_stride); a.ks = three(a.m, p->k_stride); a.vs = three(a.m, p->v_stride);
  if (int rc = check_rows("q", q, p->dtype, a.qs)) return rc;
  if (int rc = check_rows("o", o, p->dtype, a.os)) return rc;
  if (int rc = check_pool(p, k, v, k_meta, v_meta, a.ks, a.vs)) return rc;
  if (int rc = check_ws(ws, ws_bytes, block_attn_bytes(a.m, p->d, sel_idx != nullptr))) return rc;
  a.q = q; a.k = k; a.v = v; a.km = k_meta; a.vm = v_meta; a.sel = sel_idx; a.o = o; a.lse = lse;
  a.scale_log2e = log2_scale(p);
  return done(launch_block_attn((hipStream_t)stream, p->dtype, p->bits, p->d, a, ws));
}

int adacluster_block_attn_backward(const adacluster_block_params* p, const void* q, const void* k, const void* v, const void* o, const float* lse,
                                   const void* d_o, const int32_t* cu_q, const int32_t* cu_k, const int32_t* sel_idx, void* dq, void* dk, void* dv,
                                   void* ws, size_t ws_bytes, void* stream) {
  BlockGradArgs a{};
  if (int rc = check(p, &a.m)) return rc;
  if (p->num_pages || p->bits) return fail(ADACLUSTER_E_UNSUPPORTED, "block_attn_backward: packed keys in dtype only (num_pages and bits must be 0)");
  if (sel_idx && p->topk < 1) return fail(ADACLUSTER_E_BADARG, "topk must be >= 1 for lists of pages");
  if (!cu_q || !lse) return fail(ADACLUSTER_E_BADARG, "block_attn_backward: NULL tensor pointer");
  if (int rc = check_keys(&a.m, cu_k, nullptr, nullptr)) return rc;
  a.m.cu_q = cu_q;
  if (!sel_idx) a.m = unlisted(a.m);
  a.qs = two(p->q_stride); a.os = two(p->o_stride); a.dos = two(p->do_stride); a.dqs = two(p->dq_stride);
  a.ks = three(a.m, p->k_stride); a.vs = three(a.m, p->v_stride); a.dks = two(p->dk_stride); a.dvs = two(p->dv_stride);
  const struct { const char* name; const void* p; const KeyStride* s; } rows[] = {{"q", q, &a.qs}, {"k", k, &a.ks}, {"v", v, &a.vs}, {"o", o, &a.os},
      {"d_o", d_o, &a.dos}, {"dq", dq, &a.dqs}, {"dk", dk, &a.dks}, {"dv", dv, &a.dvs}};
  for (const auto& r : rows) if (int rc = check_rows(r.name, r.p, p->dtype, *r.s)) return rc;
  if (int rc = check_ws(ws, ws_bytes, block_grad_bytes(a.m, p->dtype, p->d, sel_idx != nullptr))) return rc;
  a.q = q; a.k = k; a.v = v; a.o = o; a.lse = lse; a.d_o = d_o; a.sel = sel_idx; a.dq = dq; a.dk = dk; a.dv = dv;
  a.scale = (float)scale_of(p);
  a.scale_log2e = log2_scale(p);
  return done(launch_block_attn_backward((hipStream_t)stream, p->dtype, p->d, a, ws));
}

int adacluster_prefix_workspace_bytes(const adacluster_block_params* p, int32_t groups, size_t* bytes) {
  PrefixArgs a{};
  if (int rc = prefix_args(p, groups, &a)) return rc;
  if (!bytes) return fail(ADACLUSTER_E_BADARG, "bytes is NULL");
  *bytes = prefix_attn_bytes(p->dtype, p->bits, p->d, a);
  return 0;
}

int adacluster_prefix_attn(const adacluster_block_params* p, int32_t groups, const void* q, const int32_t* cu_q, const void* k_pool, const void* v_pool,
                           const uint32_t* k_meta, const uint32_t* v_meta, const int32_t* seq_lens, const int32_t* page_table, const int32_t* cu_group,
                           const int32_t* prefix_lens, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  PrefixArgs a{};
  if (int rc = prefix_args(p, groups, &a)) return rc;
  if (!cu_q || (groups && (!cu_group || !prefix_lens))) return fail(ADACLUSTER_E_BADARG, "prefix_attn: NULL tensor pointer");
  if (int rc = check_keys(&a.m, nullptr, seq_lens, page_table)) return rc;
  a.m.cu_q = cu_q;
  if (int rc = check_rows("q", q, p->dtype, a.qs)) return rc;
  if (int rc = check_rows("o", o, p->dtype, a.os)) return rc;
  if (int rc = check_pool(p, k_pool, v_pool, k_meta, v_meta, a.ks, a.vs)) return rc;
  if (int rc = check_ws(ws, ws_bytes, prefix_attn_bytes(p->dtype, p->bits, p->d, a))) return rc;
  a.q = q; a.k = k_pool; a.v = v_pool; a.km = k_meta; a.vm = v_meta; a.o = o; a.lse = lse;
  a.gr.cu_group = cu_group; a.gr.prefix = prefix_lens;
  a.scale_log2e = log2_scale(p);
  return done(launch_prefix_attn((hipStream_t)stream, p->dtype, p->bits, p->d, a, ws));
}

int adacluster_weights_workspace_bytes(const adacluster_block_params* p, size_t* bytes) {
  BlockDims m;
  if (int rc = check(p, &m)) return rc;
  if (!p->num_pages) return fail(ADACLUSTER_E_BADARG, "cache_weights: num_pages must be >= 1");
  if (!bytes) return fail(ADACLUSTER_E_BADARG, "bytes is NULL");
  *bytes = cache_weights_bytes(p->dtype, p->bits, p->d, m, two(p->q_stride));
  return 0;
}

int adacluster_cache_weights(const adacluster_block_params* p, const void* q, const int32_t* cu_q, const float* lse, const void* k_pool,
                             const uint32_t* k_meta, const int32_t* seq_lens, const int32_t* page_table, const float* weights, float decay,
                             float* new_weights, void* ws, size_t ws_bytes, void* stream) {
  WeightsArgs a{};
  if (int rc = check(p, &a.m)) return rc;
  if (!p->num_pages) return fail(ADACLUSTER_E_BADARG, "cache_weights: num_pages must be >= 1");
  if (!(decay >= 0.f && decay <= 1.f)) return fail(ADACLUSTER_E_BADARG, "cache_weights: decay must be in [0,1]");
  if (!cu_q || !lse || !new_weights) return fail(ADACLUSTER_E_BADARG, "cache_weights: NULL tensor pointer");
  if (!aligned(weights, 16) || !aligned(new_weights, 16)) return fail(ADACLUSTER_E_BADARG, "cache_weights: weights must start at multiples of 16 bytes");
  const size_t all = (size_t)p->B * p->Hkv * p->max_pages * p->page * sizeof(float);
  if (weights && decay > 0.f && weights != new_weights && !apart(weights, all, new_weights, all)) return fail(ADACLUSTER_E_BADARG, "cache_weights: new_weights must be weights or lie apart from them");
  if (int rc = check_keys(&a.m, nullptr, seq_lens, page_table)) return rc;
  a.m.cu_q = cu_q;
  a.qs = two(p->q_stride); a.ks = three(a.m, p->k_stride);
  if (int rc = check_rows("q", q, p->dtype, a.qs)) return rc;
  if (int rc = check_pool(p, k_pool, k_pool, k_meta, k_meta, a.ks, a.ks)) return rc;
  if ((long long)p->max_q * a.m.G > MOST_ROWS) return fail(ADACLUSTER_E_UNSUPPORTED, "cache_weights: max_q * Hq / Hkv must be at most 2^31 - 1024");
  if (int rc = check_ws(ws, ws_bytes, cache_weights_bytes(p->dtype, p->bits, p->d, a.m, a.qs))) return rc;
  a.q = q; a.k = k_pool; a.km = k_meta; a.lse = lse; a.w = decay == 0.f ? nullptr : weights; a.out = new_weights;
  a.scale_log2e = log2_scale(p); a.decay = decay;
  return done(launch_cache_weights((hipStream_t)stream, p->dtype, p->bits, p->d, a, ws));
}

int adacluster_cache_evict(const adacluster_block_params* p, const int32_t* seq_lens, const int32_t* page_table, const float* weights, int32_t keep,
                           int32_t recent, const int32_t* new_table, int32_t* kept, int32_t* new_lens, float* new_weights, void* k_pool, void* v_pool,
                           uint32_t* k_meta, uint32_t* v_meta, void* boxes, void* stream) {
  EvictArgs a{};
  if (int rc = check(p, &a.m)) return rc;
  if (!p->num_pages) return fail(ADACLUSTER_E_BADARG, "cache_evict: num_pages must be >= 1");
  if (keep < 1 || keep > (1 << 29) || recent < 0) return fail(ADACLUSTER_E_BADARG, "cache_evict: keep must be in [1,2^29] and recent >= 0 (keep=%d recent=%d)", keep, recent);
  if ((long long)p->keep_first * p->page + recent > keep)
    return fail(ADACLUSTER_E_BADARG, "cache_evict: keep must hold the first pages and the last tokens: %d * %d + %d > %d", p->keep_first, p->page, recent, keep);
  if (!weights || !new_table || !kept || !new_lens || !new_weights || !boxes) return fail(ADACLUSTER_E_BADARG, "cache_evict: NULL tensor pointer");
  if (!aligned(weights, 16) || !aligned(new_weights, 16)) return fail(ADACLUSTER_E_BADARG, "cache_evict: weights must start at multiples of 16 bytes");
  const size_t all = (size_t)p->B * p->Hkv * p->max_pages * p->page * sizeof(float);
  if (!apart(weights, all, new_weights, all)) return fail(ADACLUSTER_E_BADARG, "cache_evict: new_weights must not overlap weights");
  if (int rc = check_keys(&a.m, nullptr, seq_lens, page_table)) return rc;
  a.ks = three(a.m, p->k_stride); a.vs = three(a.m, p->v_stride);
  if (int rc = check_pool(p, k_pool, v_pool, k_meta, v_meta, a.ks, a.vs)) return rc;
  // (the workgroup of a sequence's first head writes new_lens while those of the others read seq_lens, and the move reads it again)
  if (!apart(seq_lens, p->B * sizeof(int32_t), new_lens, p->B * sizeof(int32_t))) return fail(ADACLUSTER_E_BADARG, "cache_evict: new_lens must not overlap seq_lens");
  a.w = weights; a.new_table = new_table; a.keep = keep; a.recent = recent; a.kept = kept; a.new_lens = new_lens; a.new_w = new_weights;
  a.kp = k_pool; a.vp = v_pool; a.km = k_meta; a.vm = v_meta; a.boxes = boxes;
  return done(launch_cache_evict((hipStream_t)stream, p->dtype, p->bits, p->d, a));
}

}  // extern "C"
