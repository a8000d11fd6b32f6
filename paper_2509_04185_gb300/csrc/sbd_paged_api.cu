// C ABI of the paged 8-bit KV cache: argument validation and dispatch to
// paged_cache.cu and paged_attention.cu.
#include <math.h>

#include "paged.cuh"

using sbd::check_pointers;
using sbd::fail;
using sbd::Named;

namespace {

constexpr long long kMax32 = 0x7fffffffll;

sbd_status check_pool(int page_size, int n_pages) {
  if (page_size < 1 || n_pages < 1)
    return fail(SBD_ERR_INVALID_ARG, "bad sizes: page_size=%d n_pages=%d", page_size, n_pages);
  if (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128)
    return fail(SBD_ERR_UNSUPPORTED, "page_size %d not in {16, 32, 64, 128}", page_size);
  if ((long long)n_pages * page_size > kMax32)
    return fail(SBD_ERR_UNSUPPORTED, "n_pages * page_size = %lld >= 2^31",
                (long long)n_pages * page_size);
  return SBD_OK;
}

sbd_status check_heads(int n_kv_heads, int n_pages, int head_dim, int dtype) {
  if (n_kv_heads < 1 || head_dim < 1)
    return fail(SBD_ERR_INVALID_ARG, "bad sizes: n_kv_heads=%d head_dim=%d", n_kv_heads, head_dim);
  if (dtype != SBD_DTYPE_F32 && dtype != SBD_DTYPE_BF16)
    return fail(SBD_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  if (head_dim != 64 && head_dim != 128)
    return fail(SBD_ERR_UNSUPPORTED, "head_dim %d not in {64, 128}", head_dim);
  if ((long long)n_pages * n_kv_heads > kMax32)
    return fail(SBD_ERR_UNSUPPORTED, "n_pages * n_kv_heads = %lld >= 2^31",
                (long long)n_pages * n_kv_heads);
  if (n_kv_heads > 65535) return fail(SBD_ERR_UNSUPPORTED, "n_kv_heads %d > 65535", n_kv_heads);
  return SBD_OK;
}

sbd_status check_attn_q8_desc(const sbd_attn_q8_desc* d, int max_block) {
  if (!d) return fail(SBD_ERR_INVALID_ARG, "desc is NULL");
  if (d->batch < 0 || d->block_k < 1 || d->n_q_heads < 1 || d->max_pages < 1)
    return fail(SBD_ERR_INVALID_ARG, "bad sizes: batch=%d block_k=%d n_q_heads=%d max_pages=%d",
                d->batch, d->block_k, d->n_q_heads, d->max_pages);
  sbd_status s = check_heads(d->n_kv_heads, d->n_pages, d->head_dim, d->dtype);
  if (s != SBD_OK) return s;
  s = check_pool(d->page_size, d->n_pages);
  if (s != SBD_OK) return s;
  if (!(isfinite(d->scale) && d->scale >= 0.f))
    return fail(SBD_ERR_INVALID_ARG, "scale must be finite and >= 0 (0 = 1/sqrt(D))");
  if (d->n_q_heads % d->n_kv_heads != 0)
    return fail(SBD_ERR_INVALID_ARG, "n_q_heads (%d) must be a multiple of n_kv_heads (%d)",
                d->n_q_heads, d->n_kv_heads);
  if (d->num_splits < 0) return fail(SBD_ERR_INVALID_ARG, "num_splits must be >= 0");
  if (d->n_causal < 0 || d->n_causal > d->block_k)
    return fail(SBD_ERR_INVALID_ARG, "n_causal %d outside [0, block_k = %d]", d->n_causal,
                d->block_k);
  if (d->block_k > max_block) return fail(SBD_ERR_UNSUPPORTED, "block_k %d > %d", d->block_k, max_block);
  if (d->batch > 65535) return fail(SBD_ERR_UNSUPPORTED, "batch %d > 65535", d->batch);
  if ((long long)d->max_pages * d->page_size + d->block_k > kMax32)
    return fail(SBD_ERR_UNSUPPORTED, "max_pages * page_size + block_k = %lld >= 2^31",
                (long long)d->max_pages * d->page_size + d->block_k);
  // CTAs of a sequence: KV heads x row chunks (8 rows a chunk at least) in grid.y
  if ((long long)d->n_q_heads * d->block_k > 65535)
    return fail(SBD_ERR_UNSUPPORTED, "n_q_heads * block_k = %lld > 65535",
                (long long)d->n_q_heads * d->block_k);
  return SBD_OK;
}

}  // namespace

extern "C" {

sbd_status sbd_block_tables(const sbd_tables_desc* desc, const int32_t* cache_len,
                            const int32_t* target_len, const int32_t* block_table,
                            int32_t* free_pages, const int32_t* n_free,
                            int32_t* block_table_out, int32_t* len_out, int32_t* new_start,
                            int32_t* slot_map, int32_t* n_free_out, void* stream) {
  if (!desc) return fail(SBD_ERR_INVALID_ARG, "desc is NULL");
  if (desc->batch < 1 || desc->max_pages < 1 || desc->max_new < 0)
    return fail(SBD_ERR_INVALID_ARG, "bad sizes: batch=%d max_pages=%d max_new=%d", desc->batch,
                desc->max_pages, desc->max_new);
  sbd_status s = check_pool(desc->page_size, desc->n_pages);
  if (s != SBD_OK) return s;
  if (desc->batch > 4096) return fail(SBD_ERR_UNSUPPORTED, "batch %d > 4096", desc->batch);
  if ((long long)desc->batch * desc->max_pages > kMax32)
    return fail(SBD_ERR_UNSUPPORTED, "batch * max_pages = %lld >= 2^31",
                (long long)desc->batch * desc->max_pages);
  if ((long long)desc->max_pages * desc->page_size > kMax32)
    return fail(SBD_ERR_UNSUPPORTED, "max_pages * page_size = %lld >= 2^31",
                (long long)desc->max_pages * desc->page_size);
  const Named ptrs[] = {{cache_len, "cache_len"}, {target_len, "target_len"},
                        {block_table, "block_table"}, {free_pages, "free_pages"},
                        {n_free, "n_free"}, {block_table_out, "block_table_out"},
                        {len_out, "len_out"}, {new_start, "new_start"},
                        {n_free_out, "n_free_out"}};
  s = check_pointers(ptrs);
  if (s != SBD_OK) return s;
  if (desc->max_new > 0) {
    const Named slots[] = {{slot_map, "slot_map"}};
    s = check_pointers(slots);
    if (s != SBD_OK) return s;
  }
  if (block_table_out == block_table)
    return fail(SBD_ERR_INVALID_ARG, "block_table_out must not be block_table");
  if (len_out == cache_len || len_out == target_len || n_free_out == n_free)
    return fail(SBD_ERR_INVALID_ARG, "len_out and n_free_out must not be inputs");
  s = sbd::device_ready();
  if (s != SBD_OK) return s;
  return sbd::tables_launch(*desc, cache_len, target_len, block_table, free_pages, n_free,
                            block_table_out, len_out, new_start, slot_map, n_free_out,
                            (cudaStream_t)stream);
}

sbd_status sbd_cache_append_q8(const sbd_append_q8_desc* desc, const void* k_new,
                               const void* v_new, const int32_t* slot_map, void* k_cache,
                               void* v_cache, float* k_scale, float* v_scale, void* stream) {
  if (!desc) return fail(SBD_ERR_INVALID_ARG, "desc is NULL");
  if (desc->tokens < 0 || desc->group < 1)
    return fail(SBD_ERR_INVALID_ARG, "bad sizes: tokens=%d group=%d", desc->tokens, desc->group);
  sbd_status s = check_heads(desc->n_kv_heads, desc->n_pages, desc->head_dim, desc->dtype);
  if (s != SBD_OK) return s;
  s = check_pool(desc->page_size, desc->n_pages);
  if (s != SBD_OK) return s;
  const int64_t strides[] = {desc->k_group_stride, desc->k_token_stride, desc->v_group_stride,
                             desc->v_token_stride};
  s = sbd::check_strides(strides, desc->dtype);
  if (s != SBD_OK) return s;
  if (desc->tokens == 0) return SBD_OK;
  const Named ptrs[] = {{k_new, "k_new"},     {v_new, "v_new"},     {slot_map, "slot_map"},
                        {k_cache, "k_cache"}, {v_cache, "v_cache"}, {k_scale, "k_scale"},
                        {v_scale, "v_scale"}};
  s = check_pointers(ptrs);
  if (s != SBD_OK) return s;
  s = sbd::device_ready();
  if (s != SBD_OK) return s;
  return sbd::append_q8_launch(*desc, k_new, v_new, slot_map, k_cache, v_cache, k_scale, v_scale,
                               (cudaStream_t)stream);
}

size_t sbd_block_attention_q8_workspace_size(const sbd_attn_q8_desc* desc) {
  check_attn_q8_desc(desc, 32);
  return 0;                                  // splits merge on the chip
}

sbd_status sbd_block_attention_q8(const sbd_attn_q8_desc* desc, const void* q,
                                  const void* k_cache, const void* v_cache,
                                  const float* k_scale, const float* v_scale,
                                  const int32_t* block_table, const int32_t* cache_len,
                                  const void* k_blk, const void* v_blk, void* out,
                                  void*, size_t, void* stream) {
  sbd_status s = check_attn_q8_desc(desc, 32);
  if (s != SBD_OK) return s;
  if (desc->batch == 0) return SBD_OK;
  const Named ptrs[] = {{q, "q"},
                        {k_cache, "k_cache"},
                        {v_cache, "v_cache"},
                        {k_scale, "k_scale"},
                        {v_scale, "v_scale"},
                        {block_table, "block_table"},
                        {cache_len, "cache_len"},
                        {k_blk, "k_blk"},
                        {v_blk, "v_blk"},
                        {out, "out"}};
  s = check_pointers(ptrs);
  if (s != SBD_OK) return s;
  s = sbd::device_ready();
  if (s != SBD_OK) return s;
  const sbd::AttnQ8Tensors t{q,         k_cache, v_cache, k_scale, v_scale, block_table,
                             cache_len, k_blk,   v_blk,   nullptr, out};
  return sbd::attn_q8_launch(sbd::attn_q8_plan(*desc, false), t, (cudaStream_t)stream);
}

size_t sbd_tree_attention_q8_workspace_size(const sbd_attn_q8_desc* desc) {
  check_attn_q8_desc(desc, sbd_dev::kMaxNodes);
  return 0;
}

sbd_status sbd_tree_attention_q8(const sbd_attn_q8_desc* desc, const void* q, const void* k_cache,
                                 const void* v_cache, const float* k_scale, const float* v_scale,
                                 const int32_t* block_table, const int32_t* cache_len,
                                 const void* k_blk, const void* v_blk, const int32_t* parent,
                                 void* out, void*, size_t, void* stream) {
  sbd_status s = check_attn_q8_desc(desc, sbd_dev::kMaxNodes);
  if (s != SBD_OK) return s;
  if (desc->n_causal != 0)
    return fail(SBD_ERR_INVALID_ARG, "n_causal %d: a tree's rows see what parent says", desc->n_causal);
  if (desc->batch == 0) return SBD_OK;
  const Named ptrs[] = {{q, "q"},
                        {k_cache, "k_cache"},
                        {v_cache, "v_cache"},
                        {k_scale, "k_scale"},
                        {v_scale, "v_scale"},
                        {block_table, "block_table"},
                        {cache_len, "cache_len"},
                        {k_blk, "k_blk"},
                        {v_blk, "v_blk"},
                        {parent, "parent"},
                        {out, "out"}};
  s = check_pointers(ptrs);
  if (s != SBD_OK) return s;
  s = sbd::device_ready();
  if (s != SBD_OK) return s;
  const sbd::AttnQ8Tensors t{q,         k_cache, v_cache, k_scale, v_scale, block_table,
                             cache_len, k_blk,   v_blk,   parent,  out};
  return sbd::attn_q8_launch(sbd::attn_q8_plan(*desc, true), t, (cudaStream_t)stream);
}

sbd_status sbd_cache_append_path_q8(const sbd_append_path_desc* desc, const void* k_new,
                                    const void* v_new, const int32_t* path,
                                    const int32_t* new_start, const int32_t* slot_map,
                                    void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                                    void* stream) {
  if (!desc) return fail(SBD_ERR_INVALID_ARG, "desc is NULL");
  if (desc->batch < 0 || desc->nodes < 1 || desc->max_new < 0)
    return fail(SBD_ERR_INVALID_ARG, "bad sizes: batch=%d nodes=%d max_new=%d", desc->batch,
                desc->nodes, desc->max_new);
  sbd_status s = check_heads(desc->n_kv_heads, desc->n_pages, desc->head_dim, desc->dtype);
  if (s != SBD_OK) return s;
  s = check_pool(desc->page_size, desc->n_pages);
  if (s != SBD_OK) return s;
  if (desc->nodes > sbd_dev::kMaxNodes)
    return fail(SBD_ERR_UNSUPPORTED, "nodes %d > %d", desc->nodes, sbd_dev::kMaxNodes);
  if (desc->batch > 65535) return fail(SBD_ERR_UNSUPPORTED, "batch %d > 65535", desc->batch);
  const int64_t strides[] = {desc->k_batch_stride, desc->k_node_stride, desc->v_batch_stride,
                             desc->v_node_stride};
  s = sbd::check_strides(strides, desc->dtype);
  if (s != SBD_OK) return s;
  if (desc->batch == 0 || desc->max_new == 0) return SBD_OK;
  const Named ptrs[] = {{k_new, "k_new"},         {v_new, "v_new"},       {path, "path"},
                        {new_start, "new_start"}, {slot_map, "slot_map"}, {k_cache, "k_cache"},
                        {v_cache, "v_cache"},     {k_scale, "k_scale"},   {v_scale, "v_scale"}};
  s = check_pointers(ptrs);
  if (s != SBD_OK) return s;
  s = sbd::device_ready();
  if (s != SBD_OK) return s;
  return sbd::append_path_launch(*desc, k_new, v_new, path, new_start, slot_map, k_cache, v_cache,
                                 k_scale, v_scale, (cudaStream_t)stream);
}

}  // extern "C"
