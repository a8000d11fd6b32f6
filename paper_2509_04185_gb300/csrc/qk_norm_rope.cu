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
// and a row costs a sum of squares and two products an element, in pairs an instruction.
//
// Angles.  inv_freq / 2 pi in turns goes to fixed point, 64 bits behind the point; times
// the position, whole turns fall off the top of the product by themselves, and what is
// left is exact to |position| 2^-64 and the rounding of inv_freq / 2 pi to 53 bits.  The
// top 32 bits are the angle in [-1/2, 1/2) turns, which becomes a float (2^-26 of a turn off
// at most) for sincospi.  A lane computes two of the token's angles and gets the others by
// shuffles.
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
  int* err;
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

// f / 2 pi, what of it is behind the point, times 2^64, modulo 2^64.  (Of |f|, whose part behind
// the point has all its bits; that of a small negative f would be rounded next to 1.)
__device__ __forceinline__ uint64_t turns_of(float f) {
  const double turns = fabs((double)f) * 0.15915494309189533577;    // 1 / (2 pi)
  const double part = turns - floor(turns);                         // whole turns a position: none
  const uint64_t u = (uint64_t)(part * 18446744073709551616.0);
  return f < 0.f ? 0 - u : u;
}
// Cosine and sine of position * f.
__device__ __forceinline__ void rotation(int position, uint64_t turns, float* c, float* s) {
  const int32_t angle = (int32_t)((turns * (uint64_t)(int64_t)position) >> 32);
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

// What a lane does with its 16 dimensions of a row.  kNeighbours: pairs are (2 j, 2 j + 1),
// else (j, j + R / 2).  kAll: all D dimensions are rotated.
template <typename T, int D, bool kNeighbours, bool kAll>
struct Lane {
  static constexpr int kLanes = D / 16;      // of a row
  static constexpr int kRows = 32 / kLanes;  // of a warp
  uint32_t row_mask;
  int d0, d1;                                // its pieces
  bool turn;                                 // they are rotated
  float2 A[8], B[8];                         // of elements 2 e, 2 e + 1: d0 + 2 e, from e = 4 d1 + 2 (e - 4)

  __device__ __forceinline__ Lane(int R) {
    const int lane = threadIdx.x & 31, l = lane % kLanes, turned = R / 16;
    row_mask = ((1u << kLanes) - 1) << (lane - l);
    turn = kAll || l < turned;
    d0 = turn ? 8 * l : R + 16 * (l - turned);
    d1 = turn ? R / 2 + 8 * l : d0 + 8;
  }
  // The factors, from the token's angles 2 lane, 2 lane + 1 (whole warp).
  __device__ __forceinline__ void factors(const T* weight, const float (&cj)[2], const float (&sj)[2]) {
    float w[16], c[8], s[8];
#pragma unroll
    for (int e = 0; e < 16; ++e) w[e] = 1.f;
    if (weight) {
      Piece<T> w0, w1;
      w0.load(weight + d0), w1.load(weight + d1);
      w0.get(w), w1.get(w + 8);
    }
    // Of pair i: halves (d0 + i, d1 + i), or neighbours d0 + 2 i, of d1 from i = 4.
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = turn ? (kNeighbours ? (i < 4 ? d0 : d1) / 2 + i % 4 : d0 + i) : 0;
      c[i] = __shfl_sync(0xffffffffu, cj[i & 1], j >> 1);
      s[i] = __shfl_sync(0xffffffffu, sj[i & 1], j >> 1);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (!kAll && !turn) {
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
  // The sum of a row's squares (the lanes of a row together).
  __device__ __forceinline__ float squares(const float2 (&X)[8]) const {
    float2 sum = mul2(X[0], X[0]);
#pragma unroll
    for (int e = 1; e < 8; ++e) sum = fma2(X[e], X[e], sum);
    float all = sum.x + sum.y;
#pragma unroll
    for (int o = kLanes / 2; o > 0; o /= 2) all += __shfl_xor_sync(row_mask, all, o);
    return all;
  }
  // Of 1 / rms: whether squares have left fp32's range (0), or may have lost bits below it (from
  // 2^60 on), or there is a NaN; as `odd`, of which the largest tells of several rows.
  static constexpr uint32_t kOdd = 0x5d800000;
  // A row's pieces (the lanes of a row together).  An odd row comes out right only with kScaled:
  // it is taken times a power of two, and eps times its square.  (The loops do not ask row by row:
  // a branch there cost prompts 3 us of 128, and some thousand tokens 8 %.  A warp that had an odd
  // row takes all of its rows again at its end.)
  template <bool kScaled>
  __device__ __forceinline__ void row(Piece<T>& x0, Piece<T>& x1, bool norm, float eps, uint32_t& odd) const {
    float x[16];
    x0.get(x), x1.get(x + 8);
    float2 X[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) X[e] = make_float2(x[2 * e], x[2 * e + 1]);
    float inv = 1.f;
    if (norm) {
      float all = squares(X);
      inv = rsqrtf(fmaf(all, 1.f / D, eps));
      const uint32_t how = __float_as_uint(inv) - 1;
      odd = max(odd, how);
      if (kScaled && how >= kOdd) {
        const float s = all > 1.f ? 0x1p-80f : 0x1p100f;
#pragma unroll
        for (int e = 0; e < 8; ++e) X[e] = mul2(X[e], make_float2(s, s));
        all = squares(X);
        inv = rsqrtf(fmaf(all, 1.f / D, eps * s * s));
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float2 other = kNeighbours ? make_float2(X[e].y, X[e].x) : X[e ^ 4];
      // (a part that is not turned is not touched by what an infinity times 0 is)
      if (!kAll && !turn) other = make_float2(0.f, 0.f);
      float2 y = fma2(X[e], A[e], mul2(other, B[e]));
      if (norm) y = mul2(y, make_float2(inv, inv));
      x[2 * e] = y.x, x[2 * e + 1] = y.y;
    }
    x0.set(x), x1.set(x + 8);
  }
};

// Queries and keys of a token once more, heads begin .. end of both together, odd rows among them
// (whole warp; behind a call that makes everything itself, so that nothing is kept for it).
template <typename T, int D, bool kNeighbours>
__device__ __noinline__ void again(const Args& a, int t, int begin, int end) {
  using L = Lane<T, D, kNeighbours, false>;
  const int lane = threadIdx.x & 31, g = t / a.group, i = t - g * a.group;
  L my(a.R);
  float cj[2] = {1.f, 1.f}, sj[2] = {0.f, 0.f};
  if (2 * lane < a.R / 2) {
    rotation(a.positions[t], turns_of(a.inv_freq[2 * lane]), &cj[0], &sj[0]);
    rotation(a.positions[t], turns_of(a.inv_freq[2 * lane + 1]), &cj[1], &sj[1]);
  }
  uint32_t odd = 0;
#pragma unroll 1
  for (int keys = 0; keys < 2; ++keys) {
    const T* weight = (const T*)(keys ? a.k_weight : a.q_weight);
    if (!weight) continue;
    const int first = keys ? a.Hq : 0, count = keys ? a.Hkv : a.Hq;
    const int lo = max(begin, first) - first, hi = min(end, first + count) - first;
    const T* src = keys ? (const T*)a.k + g * a.k_group_stride + i * a.k_token_stride
                        : (const T*)a.q + g * a.q_group_stride + i * a.q_token_stride;
    T* dst = (T*)(keys ? a.k_out : a.q_out) + (long long)t * count * D;
    my.factors(weight, cj, sj);
#pragma unroll 1
    for (int h = lo + lane / L::kLanes; h < hi; h += L::kRows) {
      Piece<T> x0, x1;
      x0.load(src + h * D + my.d0), x1.load(src + h * D + my.d1);
      my.template row<true>(x0, x1, true, a.eps, odd);
      x0.store(dst + h * D + my.d0), x1.store(dst + h * D + my.d1);
    }
  }
}

// Few tokens, or fp32: a warp has some heads of one, three turns of rows (a turn: a row for
// each lane group) in flight.  Bound: latency up to some hundred tokens (16 tokens 3.4 us, of
// which a launch 2), HBM for prompts (fp32, 16000 tokens 126 us, 6.3 TB/s).  Instances spill 24 to
// 32 bytes (of 96 registers in bf16, 128 in fp32).
template <typename T, int D, bool kNeighbours>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 5 : 4) norm_rope_kernel(const __grid_constant__ Args a) {
  using L = Lane<T, D, kNeighbours, false>;
  constexpr int kRows = L::kRows;
  constexpr int kAhead = sizeof(T) == 2 ? 3 : 2;       // rows that a lane has in flight
  grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long job = (long long)blockIdx.x * (kThreads / 32) + warp;
  const int t = (int)(job / a.shares), share = (int)(job - (long long)t * a.shares);
  if (t >= a.tokens) return;
  const int r = lane / L::kLanes;
  L my(a.R);
  float cj[2], sj[2];                        // of angles 2 lane, 2 lane + 1
  const int position = a.R ? a.positions[t] : 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    cj[i] = 1.f, sj[i] = 0.f;
    if (2 * lane < a.R / 2) rotation(position, turns_of(a.inv_freq[2 * lane + i]), &cj[i], &sj[i]);
  }
  const int g = t / a.group, in_group = t - g * a.group;
  const int begin = share * a.share, end = min(a.heads, begin + a.share);
  uint32_t odd = 0;
  // Heads begin .. end of queries (h < Hq), keys and values.
  auto rows = [&](int first, int count, const T* src, T* dst, const T* weight, bool copy) {
    const int lo = max(begin, first) - first, hi = min(end, first + count) - first;
    if (lo >= hi) return;
    if (!copy) my.factors(weight, cj, sj);
    Piece<T> p0[kAhead], p1[kAhead];
    constexpr int kStep = kRows * D;
    src += (lo + r) * D, dst += (lo + r) * D;
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (lo + r + u * kRows < hi) p0[u].load(src + u * kStep + my.d0), p1[u].load(src + u * kStep + my.d1);
#pragma unroll 1
    for (int h0 = lo + r; h0 < hi; h0 += kAhead * kRows) {
      src += kAhead * kStep;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (h0 + u * kRows >= hi) break;
        Piece<T> x0 = p0[u], x1 = p1[u];
        if (h0 + (u + kAhead) * kRows < hi) p0[u].load(src + u * kStep + my.d0), p1[u].load(src + u * kStep + my.d1);
        if (!copy) my.template row<false>(x0, x1, weight != nullptr, a.eps, odd);
        x0.store(dst + u * kStep + my.d0), x1.store(dst + u * kStep + my.d1);
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
  if (__any_sync(0xffffffffu, odd >= L::kOdd)) {
    const long long at = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const int token = (int)(at / a.shares), begin = (int)(at - (long long)token * a.shares) * a.share;
    again<T, D, kNeighbours>(a, token, begin, min(a.heads, begin + a.share));
  }
  grid_dependents_launch();
}

// Many tokens (bf16): every warp streams whole tokens through a ring in shared memory, pieces of up
// to kPiece bytes (heads of queries, keys or values of a token) that bulk copies bring and
// take away; rows are worked on in place, values not touched at all.  What is in flight does
// not depend on registers or on where a token ends.
// Bound: HBM.  32768 tokens of 32 + 8 + 8 heads of 128 dimensions 128 us, 6.3 TB/s, 0.93 of the
// copy rate (a plain copy of as many bytes 120; from registers 143).  More in flight than 128
// KB an SM is slower: rings of 4 pieces with as many warps 147 us, of 3 pieces and 12 warps 146,
// pieces copied and not worked on 123 with 128 KB and 129 with 192.
constexpr int kPiece = 4096;
constexpr int kStages = 2;
constexpr int kStreamCtas = 4;               // that share an SM

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void bulk_store(void* dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n\tcp.async.bulk.commit_group;" ::"l"(dst),
               "r"(smem_u32(src)), "r"(bytes)
               : "memory");
}

template <typename T, int D, bool kNeighbours, bool kAll>
__global__ void __launch_bounds__(kThreads) norm_rope_stream_kernel(const __grid_constant__ Args a) {
  using L = Lane<T, D, kNeighbours, kAll>;
  constexpr int kHeads = kPiece / (D * (int)sizeof(T));        // of a piece
  static_assert(kHeads % L::kRows == 0, "whole turns");
  constexpr int kRow = D * (int)sizeof(T);
  extern __shared__ __align__(16) uint8_t ring_raw[];
  __shared__ __align__(8) uint64_t full[kThreads / 32][kStages];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint8_t* const ring = ring_raw + warp * kStages * kPiece;
  if (lane == 0) {
    for (int s = 0; s < kStages; ++s) mbar_init(&full[warp][s], 1);
    fence_mbar_init();
  }
  __syncwarp();
  grid_dependency_wait();
  const int warps = gridDim.x * (kThreads / 32), first = blockIdx.x * (kThreads / 32) + warp;
  const bool values = a.heads > a.Hq + a.Hkv;
  auto next_token = [&](int t) { return t > a.tokens - 1 - warps ? a.tokens : t + warps; };
  // The place that is loaded from: a token's queries, keys, values, so many bytes into them.
  int load_t = first, load_part = 0, load_at = 0, loaded = 0;
  const uint8_t* load_src = nullptr;
  auto load_begin = [&]() {
    const int g = a.group >= a.tokens ? 0 : load_t / a.group, i = load_t - g * a.group;
    const long long at = load_part == 0   ? g * a.q_group_stride + i * a.q_token_stride
                         : load_part == 1 ? g * a.k_group_stride + i * a.k_token_stride
                                          : g * a.v_group_stride + i * a.v_token_stride;
    load_src = (const uint8_t*)(load_part == 0 ? a.q : load_part == 1 ? a.k : a.v) + at * (int)sizeof(T);
  };
  auto load = [&]() {                        // (one lane)
    if (load_t >= a.tokens) return;
    const int all = (load_part == 0 ? a.Hq : a.Hkv) * kRow, n = min(kPiece, all - load_at), s = loaded % kStages;
    mbar_arrive_expect_tx(&full[warp][s], n);
    bulk_load(ring + s * kPiece, load_src + load_at, n, &full[warp][s]);
    ++loaded;
    load_at += kPiece;
    if (load_at < all) return;
    load_at = 0;
    if (++load_part == (values ? 3 : 2)) load_part = 0, load_t = next_token(load_t);
    if (load_t < a.tokens) load_begin();
  };
  if (lane == 0 && load_t < a.tokens) {
    load_begin();
    for (int s = 0; s < kStages; ++s) load();
  }
  L my(a.R);
  const bool has_angle = 2 * lane < a.R / 2;
  uint64_t turns[2] = {0, 0};
  float cj[2] = {1.f, 1.f}, sj[2] = {0.f, 0.f};
  if (has_angle) turns[0] = turns_of(a.inv_freq[2 * lane]), turns[1] = turns_of(a.inv_freq[2 * lane + 1]);
  int position = has_angle && first < a.tokens ? a.positions[first] : 0;
  int done = 0;
  bool ok = true;
  // A part of a token, piece by piece.
  uint32_t odd = 0;
  auto part = [&](int heads, uint8_t* dst, const T* weight, bool copy) {
    if (!copy) my.factors(weight, cj, sj);
#pragma unroll 1
    for (int h0 = 0; h0 < heads; h0 += kHeads, ++done, dst += kPiece) {
      const int n = min(kHeads, heads - h0), s = done % kStages;
      ok = mbar_wait(&full[warp][s], (done / kStages) & 1, a.err);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) return;
      uint8_t* const x = ring + s * kPiece;
      if (!copy) {
        T* row = (T*)x + lane / L::kLanes * D;
#pragma unroll 2
        for (int h = lane / L::kLanes; h < n; h += L::kRows, row += L::kRows * D) {
          Piece<T> x0, x1;
          x0.load(row + my.d0), x1.load(row + my.d1);
          my.template row<false>(x0, x1, weight != nullptr, a.eps, odd);
          x0.store(row + my.d0), x1.store(row + my.d1);
        }
        fence_proxy_async_smem();
        __syncwarp();
      }
      if (lane == 0) {
        bulk_store(dst, x, n * kRow);
        // The piece before this one has left its place by now, or nearly: the next one comes there.
        if (done > 0) {
          asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
          load();
        }
      }
      __syncwarp();
    }
  };
  for (int t = first; t < a.tokens; t = next_token(t)) {
    if (has_angle) {
      rotation(position, turns[0], &cj[0], &sj[0]);
      rotation(position, turns[1], &cj[1], &sj[1]);
      const int next = next_token(t);
      if (next < a.tokens) position = a.positions[next];
    }
    part(a.Hq, (uint8_t*)a.q_out + (long long)t * a.Hq * kRow, (const T*)a.q_weight, false);
    if (ok) part(a.Hkv, (uint8_t*)a.k_out + (long long)t * a.Hkv * kRow, (const T*)a.k_weight, false);
    if (ok && values) part(a.Hkv, (uint8_t*)a.v_out + (long long)t * a.Hkv * kRow, nullptr, true);
    if (!ok) break;
  }
  grid_dependents_launch();
  // No copy is in flight when the CTA ends, whatever became of the waits.
  if (lane == 0) {
    for (int i = done; i < loaded; ++i) mbar_wait(&full[warp][i % kStages], (i / kStages) & 1, a.err);
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  // This warp's tokens once more, where one has an odd row; what the copies wrote is there.
  __syncwarp();
  if (!__any_sync(0xffffffffu, odd >= L::kOdd) || !ok) return;
  for (int t = first; t < a.tokens; t = next_token(t)) again<T, D, kNeighbours>(a, t, 0, a.Hq + a.Hkv);
}

template <typename T, int D, bool kNeighbours>
const void* kernel_of(bool stream, bool all) {
  if constexpr (sizeof(T) == 2)
    if (stream)
      return all ? (const void*)norm_rope_stream_kernel<T, D, kNeighbours, true>
                 : (const void*)norm_rope_stream_kernel<T, D, kNeighbours, false>;
  return (const void*)norm_rope_kernel<T, D, kNeighbours>;
}
template <typename T>
const void* kernel_for(const sbd_norm_rope_desc& d, bool stream) {
  const bool all = d.rotary_dim == d.head_dim;
  if (d.head_dim == 128) return d.interleaved ? kernel_of<T, 128, true>(stream, all) : kernel_of<T, 128, false>(stream, all);
  return d.interleaved ? kernel_of<T, 64, true>(stream, all) : kernel_of<T, 64, false>(stream, all);
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
  a.err = device_error_word();
  a.heads = d.n_q_heads + d.n_kv_heads * (t.v ? 2 : 1);
  const int rows = 512 / d.head_dim;                       // of a warp's turn
  a.share = (a.heads + rows - 1) / rows * rows;
  // few tokens: a token's heads go to several warps
  while (a.share > rows && (long long)d.tokens * ((a.heads + a.share - 1) / a.share) < 16ll * num_sms())
    a.share = (a.share / rows + 1) / 2 * rows;
  a.shares = (a.heads + a.share - 1) / a.share;
  // bf16 tokens are streamed from two for every warp on (of 32 + 8 + 8 heads of 128: 2600 tokens
  // 18.3 us streamed and 15.9 spread, 5000 27.6 and 27.7, 10000 45.6 and 49.3, 16000 66 and 73; with
  // few heads instructions are the limit, 2 to 3.5 TB/s, and streamed is ahead, too: 8 + 2 + 2 of 128,
  // 32768 tokens 57.5 and 64.6, 4 + 1 + 1 of 128 50.3 and 56.9, 8000 tokens 15.7 and 17.5, 2 + 1 + 1 of
  // 64 47.6 and 51.0, 8000 tokens 14.7 and 16.2);
  // fp32 ones never (16000 tokens 134 and 125).
  const bool stream = d.dtype == SBD_DTYPE_BF16 && d.tokens >= 2ll * kStreamCtas * (kThreads / 32) * num_sms();
  const void* fn = d.dtype == SBD_DTYPE_F32 ? kernel_for<float>(d, stream) : kernel_for<__nv_bfloat16>(d, stream);
  void* args[] = {(void*)&a};
  if (stream) {
    const size_t smem = (size_t)(kThreads / 32) * kStages * kPiece;
    const sbd_status s = allow_smem(fn, smem, "cudaFuncSetAttribute(norm_rope_stream_kernel)");
    if (s != SBD_OK) return s;
    return launch_pdl(fn, dim3(kStreamCtas * num_sms()), dim3(kThreads), smem, st, args, "norm_rope_stream_kernel launch");
  }
  const long long warps = (long long)d.tokens * a.shares, ctas = (warps + kThreads / 32 - 1) / (kThreads / 32);
  if (ctas > 0x7fffffffll) return fail(SBD_ERR_UNSUPPORTED, "%lld CTAs >= 2^31", ctas);
  return launch_pdl(fn, dim3((unsigned)ctas), dim3(kThreads), 0, st, args, "norm_rope_kernel launch");
}

}  // namespace sbd
