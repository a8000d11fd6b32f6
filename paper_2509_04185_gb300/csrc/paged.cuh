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

sbd_status append_path_launch(const sbd_append_path_desc& d, const void* k_new, const void* v_new,
                              const int32_t* path, const int32_t* new_start,
                              const int32_t* slot_map, void* k_cache, void* v_cache, float* k_scale,
                              float* v_scale, cudaStream_t st);

struct AttnQ8Plan {
  int B, k, Hq, Hkv, G, D, P, max_pages, n_pages, M, n_causal;
  int rows, chunks;   // packed rows of a CTA, and how many CTAs share a KV head's rows
  int splits;         // key ranges of a (sequence, KV head, chunk): a thread-block cluster
  int ctas;           // tcgen05 kernel: that share an SM
  float scale_log2;   // softmax scale * log2(e)
  bool bf16;
  bool tree;          // block rows see themselves and their ancestors
};
struct AttnQ8Tensors {
  const void *q, *k_cache, *v_cache;
  const float *k_scale, *v_scale;
  const int32_t *table, *lens;
  const void *kb, *vb;
  const int32_t* parent;   // [B, k], of a tree
  void* out;
};
AttnQ8Plan attn_q8_plan(const sbd_attn_q8_desc& d, bool tree);
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
// Which block keys a tree's rows see, bit j of seen[i]: row i sees key j, which is i or an
// ancestor.  One warp, two rows a lane, in jumps that double: after s of them `up` is 2^s
// steps up and `seen` has the 2^s nodes from the row on.
constexpr int kMaxNodes = 64;
struct BlockViews {
  uint64_t seen[kMaxNodes];
  int up[kMaxNodes];
};
struct Parents {                                 // of this lane's rows; loaded ahead of their use
  int p[2];
  __device__ __forceinline__ void load(const int32_t* parent, int k) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = (threadIdx.x & 31) + 32 * h;
      p[h] = i < k ? parent[i] : -1;
    }
  }
};
__device__ __forceinline__ void block_views(BlockViews& v, Parents x, int* err) {
  const int lane = threadIdx.x & 31;
  uint64_t seen[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = lane + 32 * h;
    if (x.p[h] >= i) {                           // not below its node
      record_error(err, SBD_DEVERR_TREE);
      x.p[h] = -1;
    }
    seen[h] = 1ull << i;
    v.seen[i] = seen[h];
    v.up[i] = x.p[h];
  }
  __syncwarp();
  while (__any_sync(0xffffffffu, x.p[0] >= 0 || x.p[1] >= 0)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (x.p[h] < 0) continue;
      seen[h] |= v.seen[x.p[h]];
      x.p[h] = v.up[x.p[h]];
    }
    __syncwarp();
#pragma unroll
    for (int h = 0; h < 2; ++h) v.seen[lane + 32 * h] = seen[h], v.up[lane + 32 * h] = x.p[h];
    __syncwarp();
  }
}
// The smallest power of two s >= 2^-126 with amax <= 448 s = 1.75 * 2^8 s
// (amax >= 0, finite).
__device__ __forceinline__ float scale_for(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - ((u & 0x7fffffu) <= 0x600000u ? 8 : 7);
  return __uint_as_float((uint32_t)max(e, 1) << 23);
}

}  // namespace sbd_dev
