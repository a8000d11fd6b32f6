// The paged 8-bit KV cache: declarations shared by its kernels and the C ABI.
//
// Codes are e4m3 (4 exponent bits, bias 7, 3 mantissa bits; largest 448, no
// infinity), [n_pages, Hkv, P, D]: the P tokens of a page and head lie together,
// 16 D bytes at least in a piece.  Scales are fp32 [n_pages, Hkv].
#pragma once

#include <cuda_fp16.h>

#include "sbd_internal.cuh"

namespace sbd {

inline int log2_page(int P) { return P == 16 ? 4 : P == 32 ? 5 : P == 64 ? 6 : 7; }
size_t tables_smem_bytes(int B);
sbd_status tables_launch(const sbd_tables_desc& d, const int32_t* len, const int32_t* target,
                         const int32_t* table, int32_t* free_pages, const int32_t* n_free,
                         int32_t* table_out, int32_t* len_out, int32_t* new_start,
                         int32_t* slot_map, int32_t* n_free_out, cudaStream_t st);
sbd_status append_q8_launch(const sbd_append_q8_desc& d, const void* k_new, const void* v_new,
                            const int32_t* slot_map, void* k_cache, void* v_cache, float* k_scale,
                            float* v_scale, cudaStream_t st);

struct AttnQ8Plan {
  int B, k, Hq, Hkv, G, D, P, max_pages, n_pages, M, n_causal;
  int rows, chunks;   // packed rows of a CTA, and how many CTAs share a KV head's rows
  int splits;         // key ranges of a (sequence, KV head, chunk): a thread-block cluster
  int ctas;           // tcgen05 kernel: that share an SM
  float scale_log2;   // softmax scale * log2(e)
  bool bf16;
};
struct AttnQ8Tensors {
  const void *q, *k_cache, *v_cache;
  const float *k_scale, *v_scale;
  const int32_t *table, *lens;
  const void *kb, *vb;
  void* out;
};
AttnQ8Plan attn_q8_plan(const sbd_attn_q8_desc& d);
// The tcgen05 kernels: their rows, chunks and splits, and the launch.
void paged_tc_plan(AttnQ8Plan* p, int num_splits);
sbd_status paged_tc_launch(const AttnQ8Plan& p, const AttnQ8Tensors& t, cudaStream_t st);
sbd_status attn_q8_launch(const AttnQ8Plan& p, const AttnQ8Tensors& t, cudaStream_t st);

}  // namespace sbd

namespace sbd_dev {

// Four e4m3 codes, the first in the low byte (round to nearest even, saturating).
__device__ __forceinline__ uint32_t e4m3x4(float x0, float x1, float x2, float x3) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x1), "f"(x0));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x3), "f"(x2));
  return (uint32_t)lo | (uint32_t)hi << 16;
}
// The values of four codes (every e4m3 value is an fp16 value).
__device__ __forceinline__ void e4m3x4_values(uint32_t c, float (&x)[4]) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)(c & 0xffffu)));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(c >> 16)));
  const float2 a = __half22float2(*reinterpret_cast<__half2*>(&lo));
  const float2 b = __half22float2(*reinterpret_cast<__half2*>(&hi));
  x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
}
// The codes of f times the values of four codes.
__device__ __forceinline__ uint32_t e4m3x4_times(uint32_t c, float f) {
  float x[4];
  e4m3x4_values(c, x);
  return e4m3x4(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
}
// The smallest power of two s >= 2^-126 with amax <= 448 s = 1.75 * 2^8 s
// (amax >= 0, finite).
__device__ __forceinline__ float scale_for(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - ((u & 0x7fffffu) <= 0x600000u ? 8 : 7);
  return __uint_as_float((uint32_t)max(e, 1) << 23);
}

}  // namespace sbd_dev
