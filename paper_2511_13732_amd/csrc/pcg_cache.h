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

}  // namespace pcg
