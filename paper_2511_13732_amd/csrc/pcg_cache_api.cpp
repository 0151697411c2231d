// C ABI of the operators around a step's forward pass (see include/pcg.h): argument checks, then one launcher each.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "pcg_attend.h"
#include "pcg_cache.h"
#include "pcg_kernels.h"

namespace {

using namespace pcg;

constexpr int64_t kInt31 = (int64_t) 1 << 31;
constexpr int64_t kFar = (int64_t) 1 << 40;       // rows and strides: products of two stay below 2^63 with room

bool aligned(const void *p, size_t n) { return (uintptr_t) p % n == 0; }

bool good_dtype(pcg_dtype dt) { return dt == PCG_F32 || dt == PCG_BF16; }

int32_t elem_bytes(pcg_dtype dt) { return dt == PCG_BF16 ? 2 : 4; }

// A stride of rows that are read 16 bytes at a time.  (Of a single row any stride will do.)
bool stride16(int64_t s, pcg_dtype dt, bool single) {
  return single || (s > 0 && s < kFar / 256 && s * elem_bytes(dt) % 16 == 0);
}

int check_heads(int32_t heads, int32_t kv_heads, int32_t head_dim) {
  if (kv_heads < 1 || heads < kv_heads || heads % kv_heads || heads > 65536) return PCG_ERR_BAD_SHAPE;
  if (head_dim < 8 || head_dim > 128 || head_dim % 8) return PCG_ERR_BAD_SHAPE;
  return PCG_OK;
}

int check_cache(const pcg_kv_cache *c) {
  if (!c || !c->k || !c->v) return PCG_ERR_NULL_ARG;
  if (!good_dtype(c->dt)) return PCG_ERR_BAD_DTYPE;
  if (c->num_pages < 1 || c->page_size < 1 || (int64_t) c->num_pages * c->page_size >= kInt31) return PCG_ERR_BAD_SHAPE;
  if (int rc = check_heads(c->kv_heads, c->kv_heads, c->head_dim)) return rc;
  if (!stride16(c->page_stride, c->dt, c->num_pages == 1) || !stride16(c->slot_stride, c->dt, c->page_size == 1) ||
      !stride16(c->head_stride, c->dt, c->kv_heads == 1))
    return PCG_ERR_BAD_STRIDE;
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return PCG_ERR_MISALIGNED;
  return PCG_OK;
}

int check_cache4(const pcg_kv4_cache *c) {
  if (!c || !c->k || !c->v || !c->scales) return PCG_ERR_NULL_ARG;
  if (c->num_pages < 1 || c->page_size < 1 || (int64_t) c->num_pages * c->page_size >= kInt31) return PCG_ERR_BAD_SHAPE;
  if (int rc = check_heads(c->kv_heads, c->kv_heads, c->head_dim)) return rc;
  auto bytes = [](int64_t s, bool single) { return single || (s > 0 && s < kFar / 256 && s % 16 == 0); };
  auto pairs = [](int64_t s, bool single) { return single || (s > 0 && s < kFar / 256); };
  if (!bytes(c->page_stride, c->num_pages == 1) || !bytes(c->slot_stride, c->page_size == 1) || !bytes(c->head_stride, c->kv_heads == 1) ||
      !pairs(c->scale_page_stride, c->num_pages == 1) || !pairs(c->scale_slot_stride, c->page_size == 1) ||
      !pairs(c->scale_head_stride, c->kv_heads == 1))
    return PCG_ERR_BAD_STRIDE;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->scales, 4)) return PCG_ERR_MISALIGNED;
  return PCG_OK;
}

// What both ways of new rows into a cache check of them, and the part of the arguments that comes from it.
int check_append(AppendArgs &a, pcg_dtype dt, int32_t kv_heads, int32_t head_dim, const pcg_rotation *rotation, const int32_t *positions,
                 const void *q, int64_t q_tok, int64_t q_head, int32_t heads, void *q_out, int64_t o_tok, int64_t o_head, const void *k_new,
                 int64_t k_tok, int64_t k_head, const void *v_new, int64_t v_tok, int64_t v_head, int64_t T, const int32_t *slots) {
  if (T < 0 || T >= kInt31) return PCG_ERR_BAD_SHAPE;
  if (q && (heads < 1 || heads > 65536)) return PCG_ERR_BAD_SHAPE;
  // a grid's threads are counted in 32 bits
  if (T * append_threads(q ? heads : 0, kv_heads, head_dim) >= kInt31) return PCG_ERR_BAD_SHAPE;
  std::memset(&a, 0, sizeof a);
  if (rotation) {
    const pcg_rotation &r = *rotation;
    if (r.dim < 2 || r.dim > head_dim || r.dim % 2 || r.positions < 1) return PCG_ERR_BAD_SHAPE;
    if (!r.table || (T && !positions)) return PCG_ERR_NULL_ARG;
    if (r.positions > 1 && (r.stride < r.dim || r.stride >= kFar / 256)) return PCG_ERR_BAD_STRIDE;
    if (!aligned(r.table, 4) || !aligned(positions, 4)) return PCG_ERR_MISALIGNED;
    a.table = r.table;
    a.table_stride = r.positions > 1 ? r.stride : 0;
    a.rot = r.dim;
    a.places = r.positions;
    a.interleaved = r.interleaved != 0;
    a.positions = positions;
  } else if (q) {
    return PCG_ERR_NULL_ARG;           // nothing happens to queries then
  }
  if (T == 0) return PCG_OK;
  if (!k_new || !v_new || !slots || (q && !q_out)) return PCG_ERR_NULL_ARG;
  if (!stride16(k_tok, dt, T == 1) || !stride16(v_tok, dt, T == 1) || !stride16(k_head, dt, kv_heads == 1) ||
      !stride16(v_head, dt, kv_heads == 1))
    return PCG_ERR_BAD_STRIDE;
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(slots, 4)) return PCG_ERR_MISALIGNED;
  if (q) {
    if (!stride16(q_tok, dt, T == 1) || !stride16(q_head, dt, heads == 1) || !stride16(o_tok, dt, T == 1) || !stride16(o_head, dt, heads == 1))
      return PCG_ERR_BAD_STRIDE;
    if (!aligned(q, 16) || !aligned(q_out, 16)) return PCG_ERR_MISALIGNED;
  }
  a.q = q;
  a.q_out = q_out;
  a.k_new = k_new;
  a.v_new = v_new;
  a.slots = slots;
  a.T = T;
  a.q_tok = q_tok;
  a.q_head = q_head;
  a.o_tok = o_tok;
  a.o_head = o_head;
  a.k_tok = k_tok;
  a.k_head = k_head;
  a.v_tok = v_tok;
  a.v_head = v_head;
  a.heads = q ? heads : 0;
  a.kv_heads = kv_heads;
  a.D = head_dim;
  return PCG_OK;
}

uint32_t magic(int32_t d) { return d > 1 ? (uint32_t) (((uint64_t) 1 << 32) / (uint32_t) d) : UINT32_MAX; }

int finish(hipError_t e) { return e == hipSuccess ? PCG_OK : record_hip_error(e); }

// What both attention calls check of their queries, and the part of the arguments that comes from it.
int check_queries(AttendArgs &a, const void *q, int64_t q_tok, int64_t q_head, pcg_dtype dt, int32_t heads, int32_t kv_heads,
                  int32_t head_dim, int64_t T, const int32_t *q_start, int32_t B, int64_t longest, float scale,
                  int32_t window, void *out, int64_t o_tok, int64_t o_head) {
  if (int rc = check_heads(heads, kv_heads, head_dim)) return rc;
  if (B < 0 || T < 0 || longest < 0 || longest >= kInt31 || window < 0) return PCG_ERR_BAD_SHAPE;
  // a grid's threads are counted in 32 bits: 256 for every 64 rows of a shared head, and for what a request leaves over
  if (T >= kInt31 || T * heads >= (int64_t) 1 << 28 || (int64_t) B * kv_heads >= (int64_t) 1 << 22) return PCG_ERR_BAD_SHAPE;
  const float c = (float) (1.4426950408889634074 * (double) scale);
  if (!(std::isfinite(c) && c > 0.0f)) return PCG_ERR_BAD_SCALE;
  std::memset(&a, 0, sizeof a);
  if (B == 0 || T == 0) return PCG_OK;
  if (!q || !out || !q_start) return PCG_ERR_NULL_ARG;
  if (!stride16(q_tok, dt, T == 1) || !stride16(q_head, dt, heads == 1) || !stride16(o_tok, dt, T == 1) ||
      !stride16(o_head, dt, heads == 1))
    return PCG_ERR_BAD_STRIDE;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(q_start, 4)) return PCG_ERR_MISALIGNED;
  a.q = q;
  a.out = out;
  a.q_tok = q_tok;
  a.q_head = q_head;
  a.o_tok = o_tok;
  a.o_head = o_head;
  a.q_start = q_start;
  a.B = B;
  a.T = (int32_t) T;
  a.G = heads / kv_heads;
  a.heads_kv = kv_heads;
  a.D = head_dim;
  a.window = window;
  a.magic_G = magic(a.G);
  a.page_size = 1;
  a.magic_page = magic(1);
  a.c = c;
  return PCG_OK;
}

// What the attention calls over a cache check of their page table and workspace.
int check_table(int32_t page_size, int64_t T, const int32_t *block_table, int64_t table_stride, int32_t max_blocks, const int32_t *lens,
                int32_t B, const void *workspace, size_t workspace_bytes, size_t needed) {
  // positions are counted in 32 bits, up to a tile behind the last
  if (max_blocks < 1 || (int64_t) max_blocks * page_size + T >= kInt31 - 256) return PCG_ERR_BAD_SHAPE;
  if (B > 1 && (table_stride < max_blocks || table_stride >= kFar)) return PCG_ERR_BAD_STRIDE;
  if (B == 0 || T == 0) return PCG_OK;
  if (!block_table || !lens || !workspace) return PCG_ERR_NULL_ARG;
  if (!aligned(block_table, 4) || !aligned(lens, 4) || !aligned(workspace, 256)) return PCG_ERR_MISALIGNED;
  return workspace_bytes < needed ? PCG_ERR_WORKSPACE_TOO_SMALL : PCG_OK;
}

void take_table(AttendArgs &a, const int32_t *block_table, int64_t table_stride, int32_t max_blocks, const int32_t *lens, int32_t page_size,
                int32_t num_pages) {
  a.lens = lens;
  a.table = block_table;
  a.table_stride = table_stride;
  a.max_blocks = max_blocks;
  a.max_ctx = max_blocks * page_size;
  a.page_size = page_size;
  a.num_pages = num_pages;
  a.magic_page = magic(page_size);
}

}  // namespace

extern "C" {

int pcg_pages_step(const pcg_pages *pages, const int32_t *state_in, int32_t *state_out, const int32_t *commit,
                   int32_t commit_extra, const int32_t *add, int32_t add_all, int64_t max_tokens, int32_t *q_start,
                   int32_t *slots, int32_t *positions, int32_t *refused, void *hip_stream) {
  if (!pages) return PCG_ERR_NULL_ARG;
  const pcg_pages &g = *pages;
  if (g.B < 1 || g.B > kPagesMaxRequests || g.num_pages < 1 || g.page_size < 1 || g.max_blocks < 1 || max_tokens < 0 ||
      max_tokens >= kInt31 || (int64_t) g.num_pages * g.page_size >= kInt31 || (int64_t) g.max_blocks * g.page_size >= kInt31 ||
      (int64_t) g.max_blocks * g.B >= kInt31)
    return PCG_ERR_BAD_SHAPE;
  if (g.B > 1 && (g.table_stride < g.max_blocks || g.table_stride >= kFar)) return PCG_ERR_BAD_STRIDE;
  if (!g.block_table || !g.free_pages || !state_in || !state_out || !q_start || (max_tokens && !slots)) return PCG_ERR_NULL_ARG;
  for (const void *x : {(const void *) g.block_table, (const void *) g.free_pages, (const void *) state_in,
                        (const void *) state_out, (const void *) commit, (const void *) add, (const void *) q_start,
                        (const void *) slots, (const void *) positions, (const void *) refused})
    if (!aligned(x, 4)) return PCG_ERR_MISALIGNED;
  PagesArgs p;
  p.B = g.B;
  p.num_pages = g.num_pages;
  p.page_size = g.page_size;
  p.max_blocks = g.max_blocks;
  p.table = g.block_table;
  p.table_stride = g.table_stride;
  p.free_pages = g.free_pages;
  p.state_in = state_in;
  p.state_out = state_out;
  p.commit = commit;
  p.add = add;
  p.commit_extra = commit_extra;
  p.add_all = add_all;
  p.max_tokens = max_tokens;
  p.q_start = q_start;
  p.slots = slots;
  p.positions = positions;
  p.refused = refused;
  return finish(launch_pages_step(p, (hipStream_t) hip_stream));
}

int pcg_cache_write(const pcg_kv_cache *cache, const void *k_new, const void *v_new, int64_t T, int64_t k_tok_stride,
                    int64_t k_head_stride, int64_t v_tok_stride, int64_t v_head_stride, const int32_t *slots,
                    void *hip_stream) {
  if (int rc = check_cache(cache)) return rc;
  if (T < 0) return PCG_ERR_BAD_SHAPE;
  const pcg_kv_cache &c = *cache;
  WriteArgs w;
  w.elem = elem_bytes(c.dt);
  w.part_elems = 16 / w.elem;
  w.head_parts = c.head_dim / w.part_elems;
  w.parts = (int64_t) w.head_parts * c.kv_heads;
  // a grid's threads, one a part, are counted in 32 bits
  if (T >= kInt31 || T * w.parts >= kInt31) return PCG_ERR_BAD_SHAPE;
  if (T == 0) return PCG_OK;
  if (!k_new || !v_new || !slots) return PCG_ERR_NULL_ARG;
  if (!stride16(k_tok_stride, c.dt, T == 1) || !stride16(v_tok_stride, c.dt, T == 1) ||
      !stride16(k_head_stride, c.dt, c.kv_heads == 1) || !stride16(v_head_stride, c.dt, c.kv_heads == 1))
    return PCG_ERR_BAD_STRIDE;
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(slots, 4)) return PCG_ERR_MISALIGNED;
  w.k_new = k_new;
  w.v_new = v_new;
  w.k = c.k;
  w.v = c.v;
  w.slots = slots;
  w.T = T;
  w.k_tok = k_tok_stride;
  w.k_head = k_head_stride;
  w.v_tok = v_tok_stride;
  w.v_head = v_head_stride;
  w.page_stride = c.page_stride;
  w.slot_stride = c.slot_stride;
  w.head_stride = c.head_stride;
  w.num_pages = c.num_pages;
  w.page_size = c.page_size;
  return finish(launch_cache_write(w, (hipStream_t) hip_stream));
}

int pcg_cache_append(const pcg_kv_cache *cache, const pcg_rotation *rotation, const int32_t *positions, const void *q,
                     int64_t q_tok_stride, int64_t q_head_stride, int32_t heads, void *q_out, int64_t q_out_tok_stride,
                     int64_t q_out_head_stride, const void *k_new, int64_t k_tok_stride, int64_t k_head_stride, const void *v_new,
                     int64_t v_tok_stride, int64_t v_head_stride, int64_t T, const int32_t *slots, void *hip_stream) {
  if (int rc = check_cache(cache)) return rc;
  const pcg_kv_cache &c = *cache;
  AppendArgs a;
  if (int rc = check_append(a, c.dt, c.kv_heads, c.head_dim, rotation, positions, q, q_tok_stride, q_head_stride, heads, q_out, q_out_tok_stride,
                            q_out_head_stride, k_new, k_tok_stride, k_head_stride, v_new, v_tok_stride, v_head_stride, T, slots))
    return rc;
  if (T == 0) return PCG_OK;
  a.k = c.k;
  a.v = c.v;
  a.page_stride = c.page_stride;
  a.slot_stride = c.slot_stride;
  a.head_stride = c.head_stride;
  a.num_pages = c.num_pages;
  a.page_size = c.page_size;
  return finish(launch_append(a, c.dt == PCG_BF16, (hipStream_t) hip_stream));
}

int pcg_cache4_append(const pcg_kv4_cache *cache, pcg_dtype dt, const pcg_rotation *rotation, const int32_t *positions, const void *q,
                      int64_t q_tok_stride, int64_t q_head_stride, int32_t heads, void *q_out, int64_t q_out_tok_stride,
                      int64_t q_out_head_stride, const void *k_new, int64_t k_tok_stride, int64_t k_head_stride, const void *v_new,
                      int64_t v_tok_stride, int64_t v_head_stride, int64_t T, const int32_t *slots, void *hip_stream) {
  if (int rc = check_cache4(cache)) return rc;
  if (!good_dtype(dt)) return PCG_ERR_BAD_DTYPE;
  const pcg_kv4_cache &c = *cache;
  AppendArgs a;
  if (int rc = check_append(a, dt, c.kv_heads, c.head_dim, rotation, positions, q, q_tok_stride, q_head_stride, heads, q_out, q_out_tok_stride,
                            q_out_head_stride, k_new, k_tok_stride, k_head_stride, v_new, v_tok_stride, v_head_stride, T, slots))
    return rc;
  if (T == 0) return PCG_OK;
  a.k = c.k;
  a.v = c.v;
  a.scales = c.scales;
  a.page_stride = c.page_stride;
  a.slot_stride = c.slot_stride;
  a.head_stride = c.head_stride;
  a.s_page = c.scale_page_stride;
  a.s_slot = c.scale_slot_stride;
  a.s_head = c.scale_head_stride;
  a.num_pages = c.num_pages;
  a.page_size = c.page_size;
  return finish(launch_append(a, dt == PCG_BF16, (hipStream_t) hip_stream));
}

int pcg_cache4_read(const pcg_kv4_cache *cache, pcg_dtype dt, void *k_out, int64_t k_tok_stride, int64_t k_head_stride, void *v_out,
                    int64_t v_tok_stride, int64_t v_head_stride, int64_t T, const int32_t *slots, void *hip_stream) {
  if (int rc = check_cache4(cache)) return rc;
  if (!good_dtype(dt)) return PCG_ERR_BAD_DTYPE;
  const pcg_kv4_cache &c = *cache;
  if (T < 0 || T >= kInt31 || T * ((int64_t) c.kv_heads * (c.head_dim / 4) + 256) >= kInt31) return PCG_ERR_BAD_SHAPE;
  if (T == 0) return PCG_OK;
  if (!k_out || !v_out || !slots) return PCG_ERR_NULL_ARG;
  if (!stride16(k_tok_stride, dt, T == 1) || !stride16(v_tok_stride, dt, T == 1) || !stride16(k_head_stride, dt, c.kv_heads == 1) ||
      !stride16(v_head_stride, dt, c.kv_heads == 1))
    return PCG_ERR_BAD_STRIDE;
  if (!aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(slots, 4)) return PCG_ERR_MISALIGNED;
  ReadArgs r;
  r.k = c.k;
  r.v = c.v;
  r.scales = c.scales;
  r.k_out = k_out;
  r.v_out = v_out;
  r.slots = slots;
  r.T = T;
  r.k_tok = k_tok_stride;
  r.k_head = k_head_stride;
  r.v_tok = v_tok_stride;
  r.v_head = v_head_stride;
  r.page_stride = c.page_stride;
  r.slot_stride = c.slot_stride;
  r.head_stride = c.head_stride;
  r.s_page = c.scale_page_stride;
  r.s_slot = c.scale_slot_stride;
  r.s_head = c.scale_head_stride;
  r.kv_heads = c.kv_heads;
  r.D = c.head_dim;
  r.num_pages = c.num_pages;
  r.page_size = c.page_size;
  return finish(launch_cache4_read(r, dt == PCG_BF16, (hipStream_t) hip_stream));
}

size_t pcg_cache_attend_workspace_bytes(int32_t B, int64_t T, int32_t heads, int32_t kv_heads, int32_t head_dim,
                                        int64_t longest) {
  if (B < 0 || T < 0 || longest < 0 || longest >= kInt31 || check_heads(heads, kv_heads, head_dim)) return 0;
  return attend_workspace_bytes(heads / kv_heads, head_dim, longest);
}

int pcg_cache_attend(const pcg_kv_cache *cache, const void *q, int64_t q_tok_stride, int64_t q_head_stride, int32_t heads,
                     int64_t T, const int32_t *block_table, int64_t table_stride, int32_t max_blocks, const int32_t *lens,
                     const int32_t *q_start, int32_t B, int64_t longest, float scale, int32_t window, void *out,
                     int64_t out_tok_stride, int64_t out_head_stride, void *workspace, size_t workspace_bytes,
                     void *hip_stream) {
  if (int rc = check_cache(cache)) return rc;
  const pcg_kv_cache &c = *cache;
  AttendArgs a;
  if (int rc = check_queries(a, q, q_tok_stride, q_head_stride, c.dt, heads, c.kv_heads, c.head_dim, T, q_start, B, longest,
                             scale, window, out, out_tok_stride, out_head_stride))
    return rc;
  if (int rc = check_table(c.page_size, T, block_table, table_stride, max_blocks, lens, B, workspace, workspace_bytes,
                           attend_workspace_bytes(heads / c.kv_heads, c.head_dim, longest)))
    return rc;
  if (B == 0 || T == 0) return PCG_OK;
  a.k = c.k;
  a.v = c.v;
  a.k_page = a.v_page = c.page_stride;
  a.k_tok = a.v_tok = c.slot_stride;
  a.k_head = a.v_head = c.head_stride;
  take_table(a, block_table, table_stride, max_blocks, lens, c.page_size, c.num_pages);
  return finish(launch_cache_attend(a, c.dt == PCG_BF16, longest, workspace, (hipStream_t) hip_stream));
}

size_t pcg_cache4_attend_workspace_bytes(int32_t B, int64_t T, int32_t heads, int32_t kv_heads, int32_t head_dim,
                                         int64_t longest) {
  if (B < 0 || T < 0 || longest < 0 || longest >= kInt31 || check_heads(heads, kv_heads, head_dim)) return 0;
  return attend4_workspace_bytes(head_dim);
}

int pcg_cache4_attend(const pcg_kv4_cache *cache, pcg_dtype dt, const void *q, int64_t q_tok_stride, int64_t q_head_stride,
                      int32_t heads, int64_t T, const int32_t *block_table, int64_t table_stride, int32_t max_blocks,
                      const int32_t *lens, const int32_t *q_start, int32_t B, int64_t longest, float scale, int32_t window,
                      void *out, int64_t out_tok_stride, int64_t out_head_stride, void *workspace, size_t workspace_bytes,
                      void *hip_stream) {
  if (int rc = check_cache4(cache)) return rc;
  if (!good_dtype(dt)) return PCG_ERR_BAD_DTYPE;
  const pcg_kv4_cache &c = *cache;
  Attend4Args a;
  if (int rc = check_queries(a, q, q_tok_stride, q_head_stride, dt, heads, c.kv_heads, c.head_dim, T, q_start, B, longest, scale,
                             window, out, out_tok_stride, out_head_stride))
    return rc;
  if (int rc = check_table(c.page_size, T, block_table, table_stride, max_blocks, lens, B, workspace, workspace_bytes,
                           attend4_workspace_bytes(c.head_dim)))
    return rc;
  if (B == 0 || T == 0) return PCG_OK;
  a.k = c.k;
  a.v = c.v;
  a.k_page = c.page_stride;
  a.k_tok = c.slot_stride;
  a.k_head = c.head_stride;
  a.scales = reinterpret_cast<const uint32_t *>(c.scales);
  a.s_page = c.scale_page_stride;
  a.s_tok = c.scale_slot_stride;
  a.s_head = c.scale_head_stride;
  a.pairs = c.kv_heads % 2 == 0 && c.head_stride < c.slot_stride;
  take_table(a, block_table, table_stride, max_blocks, lens, c.page_size, c.num_pages);
  return finish(launch_cache4_attend(a, dt == PCG_BF16, longest, workspace, (hipStream_t) hip_stream));
}

int pcg_prompt_attend(const void *q, const void *k, const void *v, pcg_dtype dt, int64_t T, int32_t heads, int32_t kv_heads,
                      int32_t head_dim, int64_t q_tok_stride, int64_t q_head_stride, int64_t k_tok_stride,
                      int64_t k_head_stride, int64_t v_tok_stride, int64_t v_head_stride, const int32_t *q_start, int32_t B,
                      int64_t longest, float scale, int32_t window, void *out, int64_t out_tok_stride,
                      int64_t out_head_stride, void *hip_stream) {
  if (!good_dtype(dt)) return PCG_ERR_BAD_DTYPE;
  AttendArgs a;
  if (int rc = check_queries(a, q, q_tok_stride, q_head_stride, dt, heads, kv_heads, head_dim, T, q_start, B, longest, scale,
                             window, out, out_tok_stride, out_head_stride))
    return rc;
  if (B == 0 || T == 0) return PCG_OK;
  if (!k || !v) return PCG_ERR_NULL_ARG;
  if (!stride16(k_tok_stride, dt, T == 1) || !stride16(v_tok_stride, dt, T == 1) ||
      !stride16(k_head_stride, dt, kv_heads == 1) || !stride16(v_head_stride, dt, kv_heads == 1))
    return PCG_ERR_BAD_STRIDE;
  // sixteen tokens' keys at a time, whose offsets from the first are counted in 32 bits
  if (T > 1 && std::max(k_tok_stride, v_tok_stride) * 16 * elem_bytes(dt) >= kInt31) return PCG_ERR_BAD_STRIDE;
  if (!aligned(k, 16) || !aligned(v, 16)) return PCG_ERR_MISALIGNED;
  a.k = k;
  a.v = v;
  a.k_tok = T > 1 ? k_tok_stride : 0;      // of a single token any stride will do
  a.k_head = k_head_stride;
  a.v_tok = T > 1 ? v_tok_stride : 0;
  a.v_head = v_head_stride;
  return finish(launch_prompt_attend(a, dt == PCG_BF16, longest, (hipStream_t) hip_stream));
}

}  // extern "C"
