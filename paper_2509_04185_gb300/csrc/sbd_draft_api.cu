// C ABI of drafted decoding, what of it has no paged cache: argument validation and
// dispatch to qk_norm_rope.cu and verify_tree.cu.
#include <math.h>

#include "sbd_internal.cuh"

using sbd::aligned16;
using sbd::check_pointers;
using sbd::fail;
using sbd::Named;

namespace {

constexpr int kMaxNodes = 64;

sbd_status check_dtype(int dtype) {
  if (dtype != SBD_DTYPE_F32 && dtype != SBD_DTYPE_BF16)
    return fail(SBD_ERR_INVALID_ARG, "unknown dtype %d", dtype);
  return SBD_OK;
}

sbd_status check_verify_desc(const sbd_verify_desc* d) {
  if (!d) return fail(SBD_ERR_INVALID_ARG, "desc is NULL");
  if (d->batch < 0 || d->nodes < 1 || d->vocab < 1)
    return fail(SBD_ERR_INVALID_ARG, "bad sizes: batch=%d nodes=%d vocab=%d", d->batch, d->nodes,
                d->vocab);
  const sbd_status s = check_dtype(d->dtype);
  if (s != SBD_OK) return s;
  if (d->nodes > kMaxNodes) return fail(SBD_ERR_UNSUPPORTED, "nodes %d > %d", d->nodes, kMaxNodes);
  if (d->batch > 65535) return fail(SBD_ERR_UNSUPPORTED, "batch %d > 65535", d->batch);
  if (d->vocab > 1 << 24) return fail(SBD_ERR_UNSUPPORTED, "vocab %d > 2^24", d->vocab);
  return SBD_OK;
}

// A pointer that may be NULL unless `need`.
sbd_status check_optional(const Named& x, bool need) {
  if (!x.p && !need) return SBD_OK;
  const Named one[] = {x};
  return check_pointers(one);
}

}  // namespace

extern "C" {

sbd_status sbd_qk_norm_rope(const sbd_norm_rope_desc* desc, const void* q, const void* k,
                            const void* v, const int32_t* positions, const float* inv_freq,
                            const void* q_weight, const void* k_weight, void* q_out, void* k_out,
                            void* v_out, void* stream) {
  if (!desc) return fail(SBD_ERR_INVALID_ARG, "desc is NULL");
  if (desc->tokens < 0 || desc->group < 1 || desc->n_q_heads < 1 || desc->n_kv_heads < 1 ||
      desc->head_dim < 1)
    return fail(SBD_ERR_INVALID_ARG,
                "bad sizes: tokens=%d group=%d n_q_heads=%d n_kv_heads=%d head_dim=%d",
                desc->tokens, desc->group, desc->n_q_heads, desc->n_kv_heads, desc->head_dim);
  sbd_status s = check_dtype(desc->dtype);
  if (s != SBD_OK) return s;
  if (desc->head_dim != 64 && desc->head_dim != 128)
    return fail(SBD_ERR_UNSUPPORTED, "head_dim %d not in {64, 128}", desc->head_dim);
  if (desc->rotary_dim < 0 || desc->rotary_dim > desc->head_dim)
    return fail(SBD_ERR_INVALID_ARG, "rotary_dim %d outside [0, head_dim = %d]", desc->rotary_dim,
                desc->head_dim);
  if (desc->rotary_dim % 16 != 0)
    return fail(SBD_ERR_UNSUPPORTED, "rotary_dim %d is not a multiple of 16", desc->rotary_dim);
  if (!(isfinite(desc->eps) && desc->eps >= 0.f))
    return fail(SBD_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (desc->n_q_heads > 65535 || desc->n_kv_heads > 65535)
    return fail(SBD_ERR_UNSUPPORTED, "n_q_heads %d or n_kv_heads %d > 65535", desc->n_q_heads,
                desc->n_kv_heads);
  const int64_t strides[] = {desc->q_group_stride, desc->q_token_stride, desc->k_group_stride,
                             desc->k_token_stride, desc->v_group_stride, desc->v_token_stride};
  s = sbd::check_strides(strides, desc->dtype);
  if (s != SBD_OK) return s;
  if ((v == nullptr) != (v_out == nullptr))
    return fail(SBD_ERR_INVALID_ARG, "v and v_out: only one of them is NULL");
  if (desc->tokens == 0) return SBD_OK;
  const Named ptrs[] = {{q, "q"}, {k, "k"}, {q_out, "q_out"}, {k_out, "k_out"}};
  s = check_pointers(ptrs);
  if (s != SBD_OK) return s;
  const bool turns = desc->rotary_dim > 0;
  const Named optional[] = {{v, "v"}, {v_out, "v_out"}, {q_weight, "q_weight"}, {k_weight, "k_weight"}};
  for (const Named& x : optional)
    if ((s = check_optional(x, false)) != SBD_OK) return s;
  if ((s = check_optional({positions, "positions"}, turns)) != SBD_OK) return s;
  if ((s = check_optional({inv_freq, "inv_freq"}, turns)) != SBD_OK) return s;
  if (q_out == q || k_out == k || q_out == k_out || (v && (v_out == v || v_out == q_out || v_out == k_out)))
    return fail(SBD_ERR_INVALID_ARG, "outputs must be other memory than the inputs and one another");
  s = sbd::device_ready();
  if (s != SBD_OK) return s;
  const sbd::NormRopeTensors t{q,        k,        v,     positions, inv_freq,
                               q_weight, k_weight, q_out, k_out,     v_out};
  return sbd::norm_rope_launch(*desc, t, (cudaStream_t)stream);
}

size_t sbd_verify_tree_workspace_size(const sbd_verify_desc* desc) {
  check_verify_desc(desc);
  return 0;                                  // a request is one cluster
}

sbd_status sbd_verify_tree(const sbd_verify_desc* desc, const void* target_logits,
                           const void* draft_logits, const int32_t* parent, const int32_t* token,
                           const float* uniform, const float* gumbel, float tau, int32_t* path,
                           int32_t* out_tokens, float* logprob, int32_t* count, void*, size_t,
                           void* stream) {
  sbd_status s = check_verify_desc(desc);
  if (s != SBD_OK) return s;
  if (!(isfinite(tau) && tau >= 0.f)) return fail(SBD_ERR_INVALID_ARG, "tau must be finite and >= 0");
  if (tau != 0.f && !(tau >= 0x1p-20f && tau <= 0x1p20f))
    return fail(SBD_ERR_UNSUPPORTED, "tau %g outside [2^-20, 2^20]", tau);
  if (desc->batch == 0) return SBD_OK;
  const Named ptrs[] = {{target_logits, "target_logits"}, {parent, "parent"},
                        {token, "token"},                 {path, "path"},
                        {out_tokens, "out_tokens"},       {logprob, "logprob"},
                        {count, "count"}};
  s = check_pointers(ptrs);
  if (s != SBD_OK) return s;
  if ((s = check_optional({draft_logits, "draft_logits"}, false)) != SBD_OK) return s;
  if ((s = check_optional({uniform, "uniform"}, tau != 0.f)) != SBD_OK) return s;
  if ((s = check_optional({gumbel, "gumbel"}, tau != 0.f)) != SBD_OK) return s;
  if (path == parent || path == token || out_tokens == parent || out_tokens == token ||
      path == out_tokens)
    return fail(SBD_ERR_INVALID_ARG, "path and out_tokens must be other memory than parent, token and one another");
  s = sbd::device_ready();
  if (s != SBD_OK) return s;
  const sbd::VerifyTensors t{target_logits, draft_logits, parent,  token, uniform, gumbel,
                             path,          out_tokens,   logprob, count};
  return sbd::verify_launch(*desc, t, tau, (cudaStream_t)stream);
}

}  // extern "C"
