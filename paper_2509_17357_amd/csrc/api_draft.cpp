// C ABI entry points for drafted tokens (include/cronus.h): argument checks, launches.  Lengths are the device's to check.
#include <cmath>
#include <utility>

#include "api_checks.h"
#include "cronus_internal.h"

using namespace cronus;

static constexpr int32_t kMostTableSeqs = 1 << 30;  // sequences are counted in steps of a work-group, in 32 bits

extern "C" {

int cronus_build_tables(const cronus_paged_tables* tables, const int32_t* kv_lens, const int32_t* new_lens, int32_t n_seqs,
                        int32_t* cu_tokens, int32_t* start_pos, int32_t* cu_blocks, int64_t* slot_map, int32_t max_tokens,
                        int32_t* report, void* hip_stream) {
  if (!tables || n_seqs < 0 || n_seqs > kMostTableSeqs || max_tokens < 0 || tables->max_blocks_per_seq <= 0 || tables->free_capacity < 0)
    return CRONUS_ERR_INVALID_ARG;
  if ((tables->free_capacity > 0 && !tables->free_blocks) || !tables->free_count || !tables->free_count_out) return CRONUS_ERR_INVALID_ARG;
  if (!cu_tokens || !cu_blocks || !report) return CRONUS_ERR_INVALID_ARG;
  if (n_seqs > 0 && (!tables->block_tables || !tables->held || !tables->held_out || !kv_lens || !new_lens || !start_pos))
    return CRONUS_ERR_INVALID_ARG;
  return launch_build_tables(tables, kv_lens, new_lens, n_seqs, cu_tokens, start_pos, cu_blocks, slot_map, max_tokens, report, hip_stream);
}

// What both tree entry points refuse by the rows alone: a KV head's rows are counted in 32 bits.
static bool tree_rows_refused(const cronus_kv_cache* cache, int32_t max_rows) {
  return max_rows < 0 || (long long)max_rows * (cache->num_q_heads / cache->num_kv_heads) > 0x3fffffffLL;
}

size_t cronus_attn_tree_workspace_bytes(const cronus_kv_cache* cache, int32_t max_rows) {
  if (check_shape(cache) || tree_rows_refused(cache, max_rows)) return 0;
  return attn_tree_workspace(cache, max_rows, device_cus());
}

int cronus_attn_tree(const cronus_kv_cache* cache, const void* q, void* out, const int32_t* prefix_lens, const int32_t* cu_rows,
                     const uint64_t* mask, int32_t mask_words, const int32_t* block_tables, int32_t max_blocks_per_seq, int32_t n_seqs,
                     int32_t max_rows, float sm_scale, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (int rc = check_cache(cache)) return rc;
  if (n_seqs < 0 || max_blocks_per_seq <= 0 || tree_rows_refused(cache, max_rows)) return CRONUS_ERR_INVALID_ARG;
  if (!(sm_scale > 0.f) || !std::isfinite(sm_scale)) return CRONUS_ERR_INVALID_ARG;
  if (n_seqs == 0 || max_rows == 0) return CRONUS_OK;
  if (!q || !out || !prefix_lens || !cu_rows || !block_tables) return CRONUS_ERR_INVALID_ARG;
  if (mask && (mask_words <= 0 || (long long)mask_words * 64 < max_rows || (reinterpret_cast<uintptr_t>(mask) & 7u))) return CRONUS_ERR_INVALID_ARG;
  const int n_cus = device_cus();
  if (workspace_refused(workspace) || workspace_bytes < attn_tree_workspace(cache, max_rows, n_cus)) return CRONUS_ERR_WORKSPACE;
  return launch_attn_tree(cache, q, out, prefix_lens, cu_rows, mask, mask_words, block_tables, max_blocks_per_seq, n_seqs, max_rows,
                          sm_scale, workspace, n_cus, hip_stream);
}

int cronus_kv_commit(const cronus_kv_cache* caches, int32_t n_caches, const int32_t* start_pos, const int32_t* cu_rows,
                     const int32_t* paths, int32_t max_path, const int32_t* path_lens, const int32_t* block_tables,
                     int32_t max_blocks_per_seq, int32_t n_seqs, int32_t* kv_lens_out, void* hip_stream) {
  if (!caches || n_caches <= 0) return CRONUS_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n_caches; ++i) {
    if (int rc = check_cache(caches + i)) return rc;
    if (caches[i].num_kv_heads != caches->num_kv_heads || caches[i].head_dim != caches->head_dim || caches[i].kv_dtype != caches->kv_dtype)
      return CRONUS_ERR_INVALID_ARG;
    for (int32_t j = 0; j < i; ++j)  // two wavefronts would move the same rows, one from where the other has been
      if (caches[j].k_cache == caches[i].k_cache || caches[j].v_cache == caches[i].v_cache) return CRONUS_ERR_INVALID_ARG;
  }
  if (n_seqs < 0 || max_path < 0 || max_blocks_per_seq <= 0) return CRONUS_ERR_INVALID_ARG;
  if (n_seqs == 0) return CRONUS_OK;
  if (!start_pos || !cu_rows || !path_lens || !block_tables || (max_path > 0 && !paths)) return CRONUS_ERR_INVALID_ARG;
  if (kv_lens_out) {  // one work-group of a sequence writes it while others read these
    const size_t ints = sizeof(int32_t), n = (size_t)n_seqs;
    for (auto [p, count] : {std::pair<const int32_t*, size_t>{start_pos, n}, {cu_rows, n + 1}, {path_lens, n}, {paths, n * max_path}}) {
      const uintptr_t a = reinterpret_cast<uintptr_t>(kv_lens_out), b = reinterpret_cast<uintptr_t>(p);
      if (p && a < b + count * ints && b < a + n * ints) return CRONUS_ERR_INVALID_ARG;
    }
  }
  return launch_kv_commit(caches, n_caches, start_pos, cu_rows, paths, max_path, path_lens, block_tables, max_blocks_per_seq, n_seqs,
                          kv_lens_out, hip_stream);
}

}  // extern "C"
