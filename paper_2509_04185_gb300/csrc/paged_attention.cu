// Block attention over the paged 8-bit cache: the plan, the launch, and the
// kernel on fp32 FMAs (fp32 activations; bf16 ones go to paged_attention_tc.cu).
//
//   O_r = sum_j p_rj v_j,   p_r = softmax_j(scale q_r . k_j)
//
// over the cached keys j < len_b, k_j = ks[page, head] * code, v_j alike, and the
// k block keys, which are not cached and come in the activations' type.  Packed
// rows r = i*G + g (block position i, query head g of the KV head's group).
#include <math.h>

#include "key_ranges.h"
#include "paged.cuh"

namespace {

using namespace sbd_dev;

constexpr float kLog2e = 1.4426950408889634f;

// ------------------------------------------------------- FMA kernel
// One CTA per (key range, KV head and chunk of W RW packed rows, sequence), the
// key ranges of a chunk one thread-block cluster that merges through distributed
// shared memory.  Keys pass in tiles of 64: a thread fetches its 16-byte pieces of
// the next tile's codes into registers while the present one is worked on, and
// leaves their values in shared memory as fp32 (every e4m3 value is exact there).
// Key scales multiply the scores, value scales the values.  A warp owns RW rows in
// both products: S with lane = key (lane, lane + 32), O with lane = D / 32
// dimensions, P through shared memory within the warp.
// It serves fp32 activations: one product of the tensor cores' 16-bit types does not meet
// their tolerance.  (Rows as three bf16 parts each would, in three products; not built.)
// Bound: latency while the ranges are short (one request of 128 keys, 2 KV heads of 64
// dimensions, 4 rows: 5.2 us, a launch and the chain lengths -> page -> keys -> merge);
// then shared memory, every warp reading the tile for its few rows: 8 requests of 2000
// keys, 8 KV heads of 128 dimensions, 32 rows: 81 us, 26 of 80 TFLOP/s; 4 rows: 39 us;
// 128 rows, four chunks: 295 us.
// (Divisions by the page size and stores that met in a bank took a quarter more.)
constexpr int kKeys = 64;                    // keys per tile
constexpr int kGranule = 16;                 // key ranges are multiples of this

__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\t"
               "barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A float at this CTA's shared location `p`, read in CTA `rank` of the cluster.
__device__ __forceinline__ float ld_rank(const float* p, int rank) {
  uint32_t a;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

// Words n, n + 1, ... of four.
__device__ __forceinline__ uint4 rotated(uint4 v, int n) {
  if (n & 1) v = make_uint4(v.y, v.z, v.w, v.x);
  if (n & 2) v = make_uint4(v.z, v.w, v.x, v.y);
  return v;
}

struct Args {
  const float* q;
  const uint8_t *kc, *vc;
  const float *ks, *vs;
  const int32_t *table, *lens;
  const float *kb, *vb;
  float* out;
  int* err;
  int k, Hq, Hkv, G, M, log2P, max_pages, n_pages, n_causal, splits, chunks;
  float scale_log2;
};

template <int D>
__host__ __device__ constexpr int k_stride() { return D + 4; }   // lanes' rows in distinct banks

template <int D, int RW, int W>
constexpr size_t fma_smem_bytes() {
  return sizeof(float) * ((size_t)W * RW * D                        // Q
                          + (size_t)kKeys * (k_stride<D>() + D)     // K, V tile
                          + (size_t)W * RW * kKeys                  // P
                          + 2 * W * RW                              // m, l of the merge
                          + kKeys);                                 // key scales
}

template <int D, int RW, int W>
__global__ void __launch_bounds__(32 * W, W == 4 ? 3 : 2) paged_fma_kernel(const Args a) {
  constexpr int kThreads = 32 * W;
  constexpr int kRowsCta = W * RW;
  constexpr int kKS = k_stride<D>();
  constexpr int kPer = D / 32;                 // output dimensions per lane
  constexpr int kC4 = D / 4;
  constexpr int kC16 = D / 16;                 // 16-byte pieces of a row of codes
  constexpr int kFetch = kKeys * kC16 / kThreads;
  static_assert(kFetch * kThreads == kKeys * kC16, "a tile is a whole number of turns");
  extern __shared__ __align__(16) float sm[];
  float* q_s = sm;                             // [kRowsCta][D]
  float* k_s = q_s + kRowsCta * D;             // [kKeys][kKS]
  float* v_s = k_s + kKeys * kKS;              // [kKeys][D]
  float* p_s = v_s + kKeys * D;                // [kRowsCta][kKeys]
  float* st_s = p_s + kRowsCta * kKeys;        // m, then l: [kRowsCta] each
  float* sc_s = st_s + 2 * kRowsCta;           // [kKeys] key scales of the tile
  float* o_s = k_s;                            // merge: [kRowsCta][D], over the dead K tile
  static_assert(kRowsCta * D <= kKeys * kKS, "the partial rows fit the K tile");

  grid_dependency_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int split = blockIdx.x, hkv = blockIdx.y / a.chunks, chunk = blockIdx.y % a.chunks;
  const int b = blockIdx.z;
  const int cap = a.max_pages << a.log2P;
  int cached = a.lens[b];
  if (cached < 0 || cached > cap) {
    if (tid == 0) record_error(a.err, SBD_DEVERR_CACHE_LEN);
    cached = cached < 0 ? 0 : cap;
  }
  // Places of keys are unsigned: the length may be 2^31 - 1 less the block, and a tile
  // reaches past it.
  const uint32_t len = cached;
  const sbd::KeyRange keys = sbd::key_range(len + a.k, a.splits, split, kGranule);
  const uint32_t u_begin = keys.begin, u_end = keys.end;
  const int32_t* table = a.table + (size_t)b * a.max_pages;

  uint4 kf[kFetch], vf[kFetch];
  float ksf[kFetch], vsf[kFetch];
  auto fetch = [&](uint32_t t0) {
#pragma unroll
    for (int e = 0; e < kFetch; ++e) {
      const uint32_t u = t0 + (tid + e * kThreads) / kC16;
      const int c = (tid + e * kThreads) % kC16;
      kf[e] = vf[e] = make_uint4(0, 0, 0, 0);
      ksf[e] = vsf[e] = 0.f;
      if (u < u_end && u < len) {
        const int page = table[u >> a.log2P];
        if (page < 0 || page >= a.n_pages) {
          record_error(a.err, SBD_DEVERR_PAGE);
          continue;
        }
        const size_t ph = (size_t)page * a.Hkv + hkv;
        const size_t at = ((ph << a.log2P) + (u & ((1 << a.log2P) - 1))) * D + 16 * c;
        kf[e] = *reinterpret_cast<const uint4*>(a.kc + at);
        vf[e] = *reinterpret_cast<const uint4*>(a.vc + at);
        ksf[e] = a.ks[ph];
        vsf[e] = a.vs[ph];
      }
    }
  };
  // rows past u_end are zeros (PV takes 4 keys at a time)
  auto commit = [&](uint32_t t0) {
#pragma unroll
    for (int e = 0; e < kFetch; ++e) {
      const int j = (tid + e * kThreads) / kC16, c = (tid + e * kThreads) % kC16;
      const uint32_t u = t0 + j;
      float* kd = k_s + j * kKS + 16 * c;
      float* vd = v_s + j * D + 16 * c;
      if (u >= len && u < u_end) {
        const size_t at = (((size_t)b * a.k + (u - len)) * a.Hkv + hkv) * D + 16 * c;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          *reinterpret_cast<float4*>(kd + i) = *reinterpret_cast<const float4*>(a.kb + at + i);
          *reinterpret_cast<float4*>(vd + i) = *reinterpret_cast<const float4*>(a.vb + at + i);
        }
        if (c == 0) sc_s[j] = 1.f;
        continue;
      }
      // The words of a piece go in an order that differs between lanes, so that eight of
      // them store to eight places of 128 bytes.
      const int turn = (c >> 1) & 3;
      const uint4 kw = rotated(kf[e], turn), vw = rotated(vf[e], turn);
      const uint32_t kx[4] = {kw.x, kw.y, kw.z, kw.w}, vx[4] = {vw.x, vw.y, vw.z, vw.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x[4], y[4];
        e4m3x4_values(kx[i], x);
        e4m3x4_values(vx[i], y);
        const int to = 4 * ((i + turn) & 3);
        *reinterpret_cast<float4*>(kd + to) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(vd + to) =
            make_float4(y[0] * vsf[e], y[1] * vsf[e], y[2] * vsf[e], y[3] * vsf[e]);
      }
      if (c == 0) sc_s[j] = ksf[e];
    }
  };
  if (u_begin < u_end) fetch(u_begin);

  // Q rows of the chunk (zeros past M)
  for (int e = tid; e < kRowsCta * kC4; e += kThreads) {
    const int rl = e / kC4, c = e % kC4, r = chunk * kRowsCta + rl;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < a.M)
      v = *reinterpret_cast<const float4*>(
          a.q + (((size_t)b * a.k + r / a.G) * a.Hq + hkv * a.G + r % a.G) * D + 4 * c);
    *reinterpret_cast<float4*>(q_s + rl * D + 4 * c) = v;
  }

  // this warp's rows: local rows RW*warp .. + RW - 1; keys u < vis[r] are seen
  uint32_t vis[RW], vis_min = u_end;
#pragma unroll
  for (int r = 0; r < RW; ++r) {
    const int i = (chunk * kRowsCta + RW * warp + r) / a.G;
    vis[r] = min(u_end, len + (i < a.n_causal ? i + 1 : a.k));
    vis_min = min(vis_min, vis[r]);
  }
  float m[RW], l[RW];                          // l: this lane's share of the row sum
  float o[RW][kPer];
#pragma unroll
  for (int r = 0; r < RW; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < kPer; ++c) o[r][c] = 0.f;
  }
  const float* qw = q_s + RW * warp * D;
  float* pw = p_s + RW * warp * kKeys;

  for (uint32_t t0 = u_begin; t0 < u_end; t0 += kKeys) {
    const int n = min((uint32_t)kKeys, u_end - t0);
    commit(t0);
    __syncthreads();
    if (t0 + kKeys < u_end) fetch(t0 + kKeys);
    // ---- S: keys lane and lane + 32 of the tile
    const bool two = n > 32;
    float s[RW][2];
    {
      float acc[RW][2];
#pragma unroll
      for (int r = 0; r < RW; ++r) acc[r][0] = acc[r][1] = 0.f;
      const float* k0 = k_s + lane * kKS;
      const float* k1 = k0 + 32 * kKS;
      if (two) {
#pragma unroll 4
        for (int c = 0; c < kC4; ++c) {
          const float4 x0 = *reinterpret_cast<const float4*>(k0 + 4 * c);
          const float4 x1 = *reinterpret_cast<const float4*>(k1 + 4 * c);
#pragma unroll
          for (int r = 0; r < RW; ++r) {
            const float4 qv = *reinterpret_cast<const float4*>(qw + r * D + 4 * c);
            acc[r][0] = dot4(qv, x0, acc[r][0]);
            acc[r][1] = dot4(qv, x1, acc[r][1]);
          }
        }
      } else {
#pragma unroll 4
        for (int c = 0; c < kC4; ++c) {
          const float4 x0 = *reinterpret_cast<const float4*>(k0 + 4 * c);
#pragma unroll
          for (int r = 0; r < RW; ++r)
            acc[r][0] = dot4(*reinterpret_cast<const float4*>(qw + r * D + 4 * c), x0, acc[r][0]);
        }
      }
      const float f0 = sc_s[lane] * a.scale_log2, f1 = sc_s[lane + 32] * a.scale_log2;
#pragma unroll
      for (int r = 0; r < RW; ++r) {
        s[r][0] = t0 + lane < vis[r] ? acc[r][0] * f0 : -INFINITY;
        s[r][1] = two && t0 + lane + 32 < vis[r] ? acc[r][1] * f1 : -INFINITY;
      }
    }
    // ---- softmax of the tile
#pragma unroll
    for (int r = 0; r < RW; ++r) {
      const float mn = fmaxf(m[r], warp_max(fmaxf(s[r][0], s[r][1])));
      const float alpha = m[r] == -INFINITY ? 0.f : exp2f(m[r] - mn);
      const float p0 = s[r][0] == -INFINITY ? 0.f : exp2f(s[r][0] - mn);
      const float p1 = s[r][1] == -INFINITY ? 0.f : exp2f(s[r][1] - mn);
      m[r] = mn;
      l[r] = fmaf(l[r], alpha, p0 + p1);
#pragma unroll
      for (int c = 0; c < kPer; ++c) o[r][c] *= alpha;
      pw[r * kKeys + lane] = p0;
      pw[r * kKeys + lane + 32] = p1;
    }
    __syncwarp();
    // ---- O += P V, 4 keys at a time, as far as every row of the warp sees them
    const int n_all = t0 + n <= vis_min ? n : t0 < vis_min ? (int)(vis_min - t0) & ~3 : 0;
#pragma unroll 2
    for (int j = 0; j < n_all; j += 4) {
      float v[4][kPer];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (kPer == 4) {
          const float4 x = *reinterpret_cast<const float4*>(v_s + (j + e) * D + 4 * lane);
          v[e][0] = x.x, v[e][1] = x.y, v[e][2] = x.z, v[e][3] = x.w;
        } else {
          const float2 x = *reinterpret_cast<const float2*>(v_s + (j + e) * D + 2 * lane);
          v[e][0] = x.x, v[e][1] = x.y;
        }
      }
#pragma unroll
      for (int r = 0; r < RW; ++r) {
        const float4 p = *reinterpret_cast<const float4*>(pw + r * kKeys + j);
#pragma unroll
        for (int c = 0; c < kPer; ++c) {
          o[r][c] = fmaf(p.x, v[0][c], o[r][c]);
          o[r][c] = fmaf(p.y, v[1][c], o[r][c]);
          o[r][c] = fmaf(p.z, v[2][c], o[r][c]);
          o[r][c] = fmaf(p.w, v[3][c], o[r][c]);
        }
      }
    }
    // The rest, block keys that some causal row must not see: their values are
    // left out there, not multiplied by 0 (they may be infinite or NaN).
#pragma unroll 1
    for (int j = n_all; j < n; ++j) {
      float v[kPer];
#pragma unroll
      for (int c = 0; c < kPer; ++c) v[c] = v_s[j * D + kPer * lane + c];
#pragma unroll
      for (int r = 0; r < RW; ++r) {
        if (t0 + j >= vis[r]) continue;
        const float p = pw[r * kKeys + j];
#pragma unroll
        for (int c = 0; c < kPer; ++c) o[r][c] = fmaf(p, v[c], o[r][c]);
      }
    }
    __syncthreads();                           // the tile is consumed
  }
  grid_dependents_launch();

  auto store_row = [&](int rl, const float (&x)[kPer], float sum) {
    const int r = chunk * kRowsCta + rl;
    if (r >= a.M) return;
    float* dst = a.out + (((size_t)b * a.k + r / a.G) * a.Hq + hkv * a.G + r % a.G) * D + kPer * lane;
#pragma unroll
    for (int c = 0; c < kPer; c += 2)
      *reinterpret_cast<float2*>(dst + c) = make_float2(x[c] / sum, x[c + 1] / sum);
  };
  if (a.splits == 1) {
#pragma unroll
    for (int r = 0; r < RW; ++r) store_row(RW * warp + r, o[r], warp_sum(l[r]));
    return;
  }
  // ---- merge over the cluster: every CTA leaves its rows' maximum, sum and
  // unnormalised O in shared memory; CTA `split` merges rows split,
  // split + splits, ...  The second barrier keeps shared memory alive until
  // every CTA has read it.
#pragma unroll
  for (int r = 0; r < RW; ++r) {
    const int rl = RW * warp + r;
    const float lr = warp_sum(l[r]);
#pragma unroll
    for (int c = 0; c < kPer; ++c) o_s[rl * D + kPer * lane + c] = o[r][c];
    if (lane == 0) {
      st_s[rl] = m[r];
      st_s[kRowsCta + rl] = lr;
    }
  }
  cluster_sync_all();
  for (int rl = split + a.splits * warp; rl < kRowsCta && chunk * kRowsCta + rl < a.M;
       rl += a.splits * W) {
    const float ms = lane < a.splits ? ld_rank(st_s + rl, lane) : -INFINITY;
    const float ls = lane < a.splits ? ld_rank(st_s + kRowsCta + rl, lane) : 0.f;
    const float mx = warp_max(ms);
    const float w = ms == -INFINITY ? 0.f : exp2f(ms - mx);
    const float lsum = warp_sum(w * ls);
    float acc[kPer];
#pragma unroll
    for (int c = 0; c < kPer; ++c) acc[c] = 0.f;
#pragma unroll 4
    for (int e = 0; e < a.splits; ++e) {
      const float we = __shfl_sync(0xffffffffu, w, e);
#pragma unroll
      for (int c = 0; c < kPer; ++c)
        acc[c] = fmaf(we, ld_rank(o_s + rl * D + kPer * lane + c, e), acc[c]);
    }
    store_row(rl, acc, lsum);
  }
  cluster_sync_all();
}

// The instance for M packed rows: few rows per warp at small M (a small block
// keeps every warp busy), else chunks of 32 rows on 8 warps.
struct Kernel {
  const void* fn;
  size_t smem;
  int rows;          // packed rows per CTA
  int threads;
};
template <int D>
Kernel fma_kernel_of(int M) {
  if (M <= 8) return {(const void*)paged_fma_kernel<D, 2, 4>, fma_smem_bytes<D, 2, 4>(), 8, 128};
  if (M <= 16) return {(const void*)paged_fma_kernel<D, 4, 4>, fma_smem_bytes<D, 4, 4>(), 16, 128};
  return {(const void*)paged_fma_kernel<D, 4, 8>, fma_smem_bytes<D, 4, 8>(), 32, 256};
}
Kernel fma_kernel_for(int D, int M) { return D == 128 ? fma_kernel_of<128>(M) : fma_kernel_of<64>(M); }

// Key ranges per (sequence, KV head, row chunk): as many as three CTAs per SM (of four
// warps, two of eight) allow, one range per kGranule keys at most, in a cluster size whose clusters
// the device holds all at once.
int fma_splits(const sbd::AttnQ8Plan& p, const Kernel& kern, int asked) {
  const long long jobs = (long long)p.B * p.Hkv * p.chunks;
  const long long by_keys = ((long long)p.max_pages * p.P + p.k + kGranule - 1) / kGranule;
  if (jobs <= 0) return 1;
  for (int s : {16, 12, 10, 8, 6, 5, 4, 3, 2}) {
    if (asked > 0 ? s > asked : s > by_keys || s * jobs > (kern.threads == 128 ? 3ll : 2ll) * sbd::num_sms()) continue;
    if (sbd::cluster_slots(kern.fn, kern.threads, kern.smem, s) >= (asked > 0 ? 1 : jobs)) return s;
  }
  return 1;
}

sbd_status fma_launch(const sbd::AttnQ8Plan& p, const sbd::AttnQ8Tensors& t, cudaStream_t st) {
  const Kernel kern = fma_kernel_for(p.D, p.M);
  Args a;
  a.q = (const float*)t.q;
  a.kc = (const uint8_t*)t.k_cache;
  a.vc = (const uint8_t*)t.v_cache;
  a.ks = t.k_scale;
  a.vs = t.v_scale;
  a.table = t.table;
  a.lens = t.lens;
  a.kb = (const float*)t.kb;
  a.vb = (const float*)t.vb;
  a.out = (float*)t.out;
  a.err = sbd::device_error_word();
  a.k = p.k;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.G = p.G;
  a.M = p.M;
  a.log2P = sbd::log2_page(p.P);
  a.max_pages = p.max_pages;
  a.n_pages = p.n_pages;
  a.n_causal = p.n_causal;
  a.splits = p.splits;
  a.chunks = p.chunks;
  a.scale_log2 = p.scale_log2;
  const sbd_status s = sbd::allow_smem(kern.fn, kern.smem, "cudaFuncSetAttribute(paged_fma_kernel)");
  if (s != SBD_OK) return s;
  void* args[] = {(void*)&a};
  return sbd::launch_pdl(kern.fn, dim3(p.splits, p.Hkv * p.chunks, p.B), dim3(kern.threads),
                         kern.smem, st, args, "paged_fma_kernel launch", p.splits);
}

}  // namespace

namespace sbd {

AttnQ8Plan attn_q8_plan(const sbd_attn_q8_desc& d) {
  AttnQ8Plan p;
  p.B = d.batch;
  p.k = d.block_k;
  p.Hq = d.n_q_heads;
  p.Hkv = d.n_kv_heads;
  p.G = d.n_q_heads / d.n_kv_heads;
  p.D = d.head_dim;
  p.P = d.page_size;
  p.max_pages = d.max_pages;
  p.n_pages = d.n_pages;
  p.M = p.G * p.k;
  p.n_causal = d.n_causal;
  p.bf16 = d.dtype == SBD_DTYPE_BF16;
  const float scale = d.scale != 0.f ? d.scale : 1.0f / sqrtf((float)d.head_dim);
  p.scale_log2 = scale * kLog2e;
  if (p.bf16) {
    paged_tc_plan(&p, d.num_splits);
    return p;
  }
  const Kernel kern = fma_kernel_for(p.D, p.M);
  p.rows = kern.rows;
  p.chunks = (p.M + kern.rows - 1) / kern.rows;
  p.splits = fma_splits(p, kern, d.num_splits);
  p.ctas = 1;
  return p;
}

sbd_status attn_q8_launch(const AttnQ8Plan& p, const AttnQ8Tensors& t, cudaStream_t st) {
  return p.bf16 ? paged_tc_launch(p, t, st) : fma_launch(p, t, st);
}

}  // namespace sbd
