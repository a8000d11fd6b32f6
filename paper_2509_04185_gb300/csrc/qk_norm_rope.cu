// Norms of queries and keys by head and their rotation by position, in one pass over a
// fused projection, whose values are copied on the way:
//   y = w x / sqrt(mean x^2 + eps),  pair j of y turned by positions[t] * inv_freq[j].
//
// A row (token, head) of D dimensions lies with D / 16 lanes, 16 dimensions each in two
// pieces of 8: pieces l and l + R / 16 of the R rotated dimensions, so that both halves of
// a pair are one lane's (neighbours as pairs are so anyway), then the rest.  A lane's pairs
// are the same in every head, so a warp computes a token's cosines and sines once and takes
// several heads of it.
//
// Angles.  inv_freq / 2 pi in turns goes to fixed point, 64 bits behind the point; times
// the position, whole turns fall off the top of the product by themselves, and what is
// left is exact to |position| 2^-64 and the rounding of inv_freq / 2 pi to 53 bits.  The
// top 32 bits are the angle in (-1/2, 1/2] turns, for sincospi.
#include "sbd_internal.cuh"

namespace {

using namespace sbd_dev;

constexpr int kThreads = 128;

struct Args {
  const void *q, *k, *v;
  const int32_t* positions;
  const float* inv_freq;
  const void *q_weight, *k_weight;
  void *q_out, *k_out, *v_out;
  long long q_group_stride, q_token_stride, k_group_stride, k_token_stride, v_group_stride, v_token_stride;
  int tokens, group, Hq, Hkv, R;
  int heads;                 // Hq + Hkv, and Hkv more where values are copied
  int share;                 // heads of a warp
  int shares;                // warps of a token
  float eps;
};

template <typename T>
struct Piece;                // 8 consecutive elements
template <>
struct Piece<__nv_bfloat16> {
  uint4 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = w; }
  __device__ __forceinline__ void get(float* x) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(u[e] << 16);
      x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float* x) {
    uint32_t u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
      u[e] = *reinterpret_cast<const uint32_t*>(&v);
    }
    w = make_uint4(u[0], u[1], u[2], u[3]);
  }
};
template <>
struct Piece<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<float4*>(p)[0] = a, reinterpret_cast<float4*>(p)[1] = b;
  }
  __device__ __forceinline__ void get(float* x) const {
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
  __device__ __forceinline__ void set(const float* x) {
    a = make_float4(x[0], x[1], x[2], x[3]), b = make_float4(x[4], x[5], x[6], x[7]);
  }
};

// Cosine and sine of position * f.
__device__ __forceinline__ void rotation(int position, float f, float* c, float* s) {
  const double turns = (double)f * 0.15915494309189533577;          // 1 / (2 pi)
  const double part = turns - floor(turns);                         // whole turns a position: none
  const uint64_t fixed = (uint64_t)(part * 18446744073709551616.0);  // (part = 1 by rounding: 2^64 - 1, a turn)
  const int32_t angle = (int32_t)((fixed * (uint64_t)(int64_t)position) >> 32);
  sincospif((float)angle * 4.656612873077392578125e-10f, s, c);     // 2^-31: half turns
}

template <typename T, int D, bool kNeighbours>
__global__ void __launch_bounds__(kThreads) norm_rope_kernel(const Args a) {
  constexpr int kLanes = D / 16;             // of a row
  constexpr int kRows = 32 / kLanes;         // of a warp
  grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long job = (long long)blockIdx.x * (kThreads / 32) + warp;
  const int t = (int)(job / a.shares), share = (int)(job - (long long)t * a.shares);
  if (t >= a.tokens) return;
  const int l = lane % kLanes, r = lane / kLanes;
  const int turned = a.R / 16;               // lanes whose pieces are rotated
  const bool turn = l < turned;
  const int d0 = turn ? 8 * l : a.R + 16 * (l - turned);
  const int d1 = turn ? a.R / 2 + 8 * l : d0 + 8;
  // Of pair i of this lane: halves (d0 + i, d1 + i), or neighbours d0 + 2 i, of d1 from i = 4.
  float c[8], s[8];
  if (turn) {
    const int position = a.positions[t];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = kNeighbours ? (i < 4 ? d0 : d1) / 2 + i % 4 : d0 + i;
      rotation(position, a.inv_freq[j], &c[i], &s[i]);
    }
  }
  const int g = t / a.group, in_group = t - g * a.group;
  const int end = min(a.heads, (share + 1) * a.share);
  for (int h = share * a.share + r; h < end; h += kRows) {
    const bool is_q = h < a.Hq, is_v = h >= a.Hq + a.Hkv;
    const int hh = is_q ? h : is_v ? h - a.Hq - a.Hkv : h - a.Hq;
    const T* src = (const T*)(is_q ? a.q : is_v ? a.v : a.k) + (long long)hh * D +
                   g * (is_q ? a.q_group_stride : is_v ? a.v_group_stride : a.k_group_stride) +
                   in_group * (is_q ? a.q_token_stride : is_v ? a.v_token_stride : a.k_token_stride);
    T* dst = (T*)(is_q ? a.q_out : is_v ? a.v_out : a.k_out) + ((long long)t * (is_q ? a.Hq : a.Hkv) + hh) * D;
    Piece<T> p0, p1;
    p0.load(src + d0), p1.load(src + d1);
    const T* weight = (const T*)(is_q ? a.q_weight : a.k_weight);
    if (!is_v) {
      float x[16];
      p0.get(x), p1.get(x + 8);
      if (weight) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fmaf(x[i], x[i], sum);
        const uint32_t mask = (kLanes == 32 ? 0xffffffffu : (1u << kLanes) - 1) << (r * kLanes);
#pragma unroll
        for (int o = kLanes / 2; o > 0; o /= 2) sum += __shfl_xor_sync(mask, sum, o);
        const float inv = rsqrtf(sum * (1.f / D) + a.eps);
        Piece<T> w0, w1;
        w0.load(weight + d0), w1.load(weight + d1);
        float w[16];
        w0.get(w), w1.get(w + 8);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= inv * w[i];
      }
      if (turn) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int one = kNeighbours ? 2 * i : i, two = kNeighbours ? 2 * i + 1 : i + 8;
          const float y1 = x[one], y2 = x[two];
          x[one] = y1 * c[i] - y2 * s[i];
          x[two] = y2 * c[i] + y1 * s[i];
        }
      }
      p0.set(x), p1.set(x + 8);
    }
    p0.store(dst + d0), p1.store(dst + d1);
  }
  grid_dependents_launch();
}

template <typename T, int D>
const void* kernel_of(bool neighbours) {
  return neighbours ? (const void*)norm_rope_kernel<T, D, true> : (const void*)norm_rope_kernel<T, D, false>;
}

}  // namespace

namespace sbd {

sbd_status norm_rope_launch(const sbd_norm_rope_desc& d, const NormRopeTensors& t, cudaStream_t st) {
  Args a;
  a.q = t.q;
  a.k = t.k;
  a.v = t.v;
  a.positions = t.positions;
  a.inv_freq = t.inv_freq;
  a.q_weight = t.q_weight;
  a.k_weight = t.k_weight;
  a.q_out = t.q_out;
  a.k_out = t.k_out;
  a.v_out = t.v_out;
  a.q_group_stride = d.q_group_stride;
  a.q_token_stride = d.q_token_stride;
  a.k_group_stride = d.k_group_stride;
  a.k_token_stride = d.k_token_stride;
  a.v_group_stride = d.v_group_stride;
  a.v_token_stride = d.v_token_stride;
  a.tokens = d.tokens;
  a.group = d.group;
  a.Hq = d.n_q_heads;
  a.Hkv = d.n_kv_heads;
  a.R = d.rotary_dim;
  a.eps = d.eps;
  a.heads = d.n_q_heads + d.n_kv_heads * (t.v ? 2 : 1);
  const int rows = 512 / d.head_dim;                       // of a warp's turn
  a.share = (a.heads + rows - 1) / rows * rows;
  // few tokens: a token's heads go to several warps
  while (a.share > rows && (long long)d.tokens * ((a.heads + a.share - 1) / a.share) < 16ll * num_sms())
    a.share = (a.share / rows + 1) / 2 * rows;
  a.shares = (a.heads + a.share - 1) / a.share;
  const long long warps = (long long)d.tokens * a.shares, ctas = (warps + kThreads / 32 - 1) / (kThreads / 32);
  if (ctas > 0x7fffffffll) return fail(SBD_ERR_UNSUPPORTED, "%lld CTAs >= 2^31", ctas);
  const bool f32 = d.dtype == SBD_DTYPE_F32, pairs = d.interleaved != 0;
  const void* fn = d.head_dim == 128 ? (f32 ? kernel_of<float, 128>(pairs) : kernel_of<__nv_bfloat16, 128>(pairs))
                                     : (f32 ? kernel_of<float, 64>(pairs) : kernel_of<__nv_bfloat16, 64>(pairs));
  void* args[] = {(void*)&a};
  return launch_pdl(fn, dim3((unsigned)ctas), dim3(kThreads), 0, st, args, "norm_rope_kernel launch");
}

}  // namespace sbd
