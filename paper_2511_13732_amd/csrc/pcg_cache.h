// Arguments of the page table and cache write kernels (pcg_cache.hip), filled by the C ABI layer (pcg_cache_api.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pcg {

constexpr int32_t kPagesMaxRequests = 65536;

struct PagesArgs {
  int32_t B, num_pages, page_size, max_blocks;
  int32_t *table;
  int64_t table_stride;
  int32_t *free_pages;
  const int32_t *state_in;
  int32_t *state_out;
  const int32_t *commit, *add;
  int32_t commit_extra, add_all;
  int64_t max_tokens;
  int32_t *q_start, *slots, *positions, *refused;
};
hipError_t launch_pages_step(const PagesArgs &p, hipStream_t stream);

struct WriteArgs {
  const void *k_new, *v_new;
  void *k, *v;
  const int32_t *slots;
  int64_t T, k_tok, k_head, v_tok, v_head, page_stride, slot_stride, head_stride;   // strides in elements
  int64_t parts;                 // 16-byte parts of a token's keys
  int32_t head_parts, part_elems, elem, num_pages, page_size;
};
hipError_t launch_cache_write(const WriteArgs &w, hipStream_t stream);

// New rows on their way into a cache (pcg_append.hip), of the rows' own type or (scales) of 4-bit codes.
struct AppendArgs {
  const void *q, *k_new, *v_new;       // q NULL: none
  void *q_out, *k, *v;
  uint16_t *scales;
  const float *table;                  // NULL: no rotation
  const int32_t *positions, *slots;
  int64_t T, table_stride;
  // strides: of rows in elements; of the cache in elements, or in bytes of codes and pairs of scales
  int64_t q_tok, q_head, o_tok, o_head, k_tok, k_head, v_tok, v_head, page_stride, slot_stride, head_stride, s_page, s_slot, s_head;
  int32_t heads, kv_heads, D, rot, places;      // places: rows of the table
  int32_t num_pages, page_size;
  bool interleaved;
};
// Threads that a token takes at most: T times that has to stay below 2^31.
int64_t append_threads(int32_t heads, int32_t kv_heads, int32_t head_dim);
hipError_t launch_append(const AppendArgs &a, bool bf16, hipStream_t stream);

struct ReadArgs {
  const uint8_t *k, *v;
  const uint16_t *scales;
  void *k_out, *v_out;
  const int32_t *slots;
  int64_t T, k_tok, k_head, v_tok, v_head, page_stride, slot_stride, head_stride, s_page, s_slot, s_head;
  int32_t kv_heads, D, num_pages, page_size;
};
hipError_t launch_cache4_read(const ReadArgs &r, bool bf16, hipStream_t stream);

}  // namespace pcg
