// Arguments of the attention kernels (pcg_attend.hip), filled by the C ABI layer (pcg_cache_api.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pcg {

struct AttendArgs {
  const void *q, *k, *v;
  void *out;
  // Strides in elements.  A key is at k + page * k_page + slot * k_tok + head * k_head; without pages at
  // k + token * k_tok + head * k_head.
  int64_t q_tok, q_head, o_tok, o_head, k_page, k_tok, k_head, v_page, v_tok, v_head;
  const int32_t *q_start;          // [B + 1]
  const int32_t *lens;             // [B] tokens ahead of the chunk; NULL: none, keys lie beside the queries
  const int32_t *table;            // [B, >= blocks], NULL: no pages
  int64_t table_stride;
  int32_t B, T, G, heads_kv, D, window;
  int32_t page_size, num_pages, max_blocks, max_ctx;
  uint32_t magic_page, magic_G;    // see split_by
  float c;                         // log2(e) * scale
};

size_t attend_workspace_bytes(int32_t G, int32_t D, int64_t longest);
hipError_t launch_cache_attend(const AttendArgs &a, bool bf16, int64_t longest, void *workspace, hipStream_t stream);
hipError_t launch_prompt_attend(const AttendArgs &a, bool bf16, int64_t longest, hipStream_t stream);

}  // namespace pcg
