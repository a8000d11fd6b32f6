// Norms of queries and keys by head and their rotation by position, in one pass over a
// fused projection, whose values are copied on the way:
//   y = w x / sqrt(mean x^2 + eps),  pair j of y turned by positions[t] * inv_freq[j].
//
// A row (token, head) of D dimensions lies with D / 16 lanes, 16 dimensions each in two
// pieces of 8: pieces l and l + R / 16 of the R rotated dimensions, so that both halves of
// a pair are one lane's (neighbours as pairs are so anyway), then the rest.  A lane's pairs
// are the same in every head, so norm weights, cosines and sines become two factors an
// element, A and B, once for a token's queries and once for its keys:
//   y_d = (x_d A_d + x_d' B_d) / sqrt(mean x^2 + eps),   d' the other half of d's pair,
// and a row costs a sum of squares and two products an element, in pairs an instruction.  A
// warp takes all of a token's heads (several warps share them where tokens are few), a row
// ahead of the one that it works on.
//
// Angles.  inv_freq / 2 pi in turns goes to fixed point, 64 bits behind the point; times
// the position, whole turns fall off the top of the product by themselves, and what is
// left is exact to |position| 2^-64 and the rounding of inv_freq / 2 pi to 53 bits.  The
// top 32 bits are the angle in (-1/2, 1/2] turns, for sincospi.  A lane computes two of
// the token's angles and gets the others by shuffles.
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

// Two fp32 operations an instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "mul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// kNeighbours: pairs are (2 j, 2 j + 1), else (j, j + R / 2).
template <typename T, int D, bool kNeighbours>
__global__ void __launch_bounds__(kThreads, 5) norm_rope_kernel(const Args a) {
  constexpr int kLanes = D / 16;             // of a row
  constexpr int kRows = 32 / kLanes;         // of a warp
  constexpr int kAhead = sizeof(T) == 2 ? 3 : 2;       // rows that a lane has in flight
  grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long job = (long long)blockIdx.x * (kThreads / 32) + warp;
  const int t = (int)(job / a.shares), share = (int)(job - (long long)t * a.shares);
  if (t >= a.tokens) return;
  const int l = lane % kLanes, r = lane / kLanes;
  const uint32_t row_mask = ((1u << kLanes) - 1) << (r * kLanes);
  const int turned = a.R / 16;               // lanes whose pieces are rotated
  const bool turn = l < turned;
  const int d0 = turn ? 8 * l : a.R + 16 * (l - turned);
  const int d1 = turn ? a.R / 2 + 8 * l : d0 + 8;
  // Of pair i of this lane: halves (d0 + i, d1 + i), or neighbours d0 + 2 i, of d1 from i = 4.
  float c[8], s[8];
  {
    float cj[2], sj[2];                      // of angles 2 lane, 2 lane + 1
    const int position = a.R ? a.positions[t] : 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      cj[i] = 1.f, sj[i] = 0.f;
      if (2 * lane < a.R / 2) rotation(position, a.inv_freq[2 * lane + i], &cj[i], &sj[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = turn ? (kNeighbours ? (i < 4 ? d0 : d1) / 2 + i % 4 : d0 + i) : 0;
      c[i] = __shfl_sync(0xffffffffu, cj[i & 1], j >> 1);
      s[i] = __shfl_sync(0xffffffffu, sj[i & 1], j >> 1);
    }
  }
  const int g = t / a.group, in_group = t - g * a.group;
  const int begin = share * a.share, end = min(a.heads, begin + a.share);
  // Heads begin .. end of queries (h < Hq), keys and values.
  auto rows = [&](int first, int count, const T* src, T* dst, const T* weight, bool copy) {
    const int lo = max(begin, first) - first, hi = min(end, first + count) - first;
    if (lo >= hi) return;
    float2 A[8], B[8];                       // of elements 2 e, 2 e + 1: d0 + 2 e, from e = 4 d1 + 2 (e - 4)
    if (!copy) {
      float w[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) w[e] = 1.f;
      if (weight) {
        Piece<T> w0, w1;
        w0.load(weight + d0), w1.load(weight + d1);
        w0.get(w), w1.get(w + 8);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (!turn) {
          A[e] = make_float2(w[2 * e], w[2 * e + 1]), B[e] = make_float2(0.f, 0.f);
        } else if (kNeighbours) {
          A[e] = make_float2(w[2 * e] * c[e], w[2 * e + 1] * c[e]);
          B[e] = make_float2(-w[2 * e + 1] * s[e], w[2 * e] * s[e]);
        } else {
          const int i = 2 * (e & 3);
          const float sign = e < 4 ? -1.f : 1.f;
          A[e] = make_float2(w[2 * e] * c[i], w[2 * e + 1] * c[i + 1]);
          B[e] = make_float2(sign * w[(2 * e + 8) % 16] * s[i], sign * w[(2 * e + 9) % 16] * s[i + 1]);
        }
      }
    }
    Piece<T> p0[kAhead], p1[kAhead];
    constexpr int kStep = kRows * D;
    src += (lo + r) * D, dst += (lo + r) * D;
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (lo + r + u * kRows < hi) p0[u].load(src + u * kStep + d0), p1[u].load(src + u * kStep + d1);
#pragma unroll 1
    for (int h0 = lo + r; h0 < hi; h0 += kAhead * kRows) {
      src += kAhead * kStep;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
      if (h0 + u * kRows >= hi) break;
      Piece<T> x0 = p0[u], x1 = p1[u];
      if (h0 + (u + kAhead) * kRows < hi) p0[u].load(src + u * kStep + d0), p1[u].load(src + u * kStep + d1);
      if (!copy) {
        float x[16];
        x0.get(x), x1.get(x + 8);
        float2 X[8], Y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) X[e] = make_float2(x[2 * e], x[2 * e + 1]);
        float inv = 1.f;
        if (weight) {
          float2 sum = mul2(X[0], X[0]);
#pragma unroll
          for (int e = 1; e < 8; ++e) sum = fma2(X[e], X[e], sum);
          float all = sum.x + sum.y;
#pragma unroll
          for (int o = kLanes / 2; o > 0; o /= 2) all += __shfl_xor_sync(row_mask, all, o);
          inv = rsqrtf(fmaf(all, 1.f / D, a.eps));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float2 other = kNeighbours ? make_float2(X[e].y, X[e].x) : X[e ^ 4];
          // (a part that is not turned is not touched by what an infinity times 0 is)
          if (!turn) other = make_float2(0.f, 0.f);
          Y[e] = fma2(X[e], A[e], mul2(other, B[e]));
          if (weight) Y[e] = mul2(Y[e], make_float2(inv, inv));
          x[2 * e] = Y[e].x, x[2 * e + 1] = Y[e].y;
        }
        x0.set(x), x1.set(x + 8);
      }
      x0.store(dst + u * kStep + d0), x1.store(dst + u * kStep + d1);
      }
      dst += kAhead * kStep;
    }
  };
  rows(0, a.Hq, (const T*)a.q + g * a.q_group_stride + in_group * a.q_token_stride, (T*)a.q_out + (long long)t * a.Hq * D,
       (const T*)a.q_weight, false);
  rows(a.Hq, a.Hkv, (const T*)a.k + g * a.k_group_stride + in_group * a.k_token_stride,
       (T*)a.k_out + (long long)t * a.Hkv * D, (const T*)a.k_weight, false);
  rows(a.Hq + a.Hkv, a.heads - a.Hq - a.Hkv, (const T*)a.v + g * a.v_group_stride + in_group * a.v_token_stride,
       (T*)a.v_out + (long long)t * a.Hkv * D, nullptr, true);
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
