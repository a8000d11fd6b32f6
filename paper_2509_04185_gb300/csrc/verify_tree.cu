// Verification of drafted tokens: the walk down a tree of nodes that accepts tokens by
// the target's probabilities and given random numbers (include/sbd.h has the rule).
//
// What a row of logits is needed for is its maximum m, its sum S = sum exp((z - m) / tau),
// the values at a few drafted tokens, and, where the walk ends, one argmax over
//   ln r(v) + gumbel(v),   r = what is left of p after the rejected children:
//   r_0 = p,  r_(k+1)(v) = max(r_k(v) - q(v), 0) / Z_k   (draft with probabilities)
//                        = r_k(v) / Z_k, 0 at the rejected token  (without)
// r_k is a function of the logits at v and of the scalars Z, so nothing is stored for it:
// a pass over the row evaluates it.  A request is a thread-block cluster, each CTA has a
// slice of the vocabulary, and what they need of one another goes through distributed
// shared memory: every CTA leaves its share of a sum in all of them, adds up in rank order,
// and so comes to the same numbers and decisions as the others.  Only rows that the walk
// comes to are read.
#include <float.h>
#include <math.h>

#include "sbd_internal.cuh"

namespace {

using namespace sbd_dev;

constexpr int kMaxNodes = 64;
constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 16;

enum Mode { kGreedy, kGiven, kDrawn };       // tau = 0; drafts without, with probabilities

struct Args {
  const void *target, *draft;
  const int32_t *parent, *token;
  const float *uniform, *gumbel;
  int32_t *path, *out_tokens;
  float* logprob;
  int32_t* count;
  int* err;
  long long total;           // elements of target
  int n, V, splits;
  float inv_tau, scale;      // 1 / tau and log2(e) / tau (1 and log2(e) where tau = 0)
};

// What is kept of a part of a row.
struct Sum {
  float m, s;                // largest logit, sum of 2^((z - m) scale)
};
struct Best {
  float score, z;
  int v;
};

__device__ __forceinline__ Sum merge(Sum a, Sum b, float scale) {
  Sum r;
  r.m = fmaxf(a.m, b.m);
  r.s = (a.s > 0.f ? a.s * exp2f((a.m - r.m) * scale) : 0.f) + (b.s > 0.f ? b.s * exp2f((b.m - r.m) * scale) : 0.f);
  return r;
}
__device__ __forceinline__ Best better(Best a, Best b) {
  return b.score > a.score || (b.score == a.score && b.v < a.v) ? b : a;
}

// NaN counts as -inf, +inf as the largest number.
__device__ __forceinline__ float tame(float z) { return fminf(fmaxf(z, -INFINITY), FLT_MAX); }

__device__ __forceinline__ float value(const __nv_bfloat16* p) { return tame(__bfloat162float(*p)); }
__device__ __forceinline__ float value(const float* p) { return tame(*p); }

// The logits of a row in words of 16 bytes from the aligned place at or before its
// beginning; word w has elements kPer w - shift ... of the row, outside of it -inf.
template <typename T>
struct Row {
  static constexpr int kPer = 16 / sizeof(T);
  const T* base;             // aligned
  const T* end;              // of the tensor
  int shift, V;
  __device__ __forceinline__ Row(const T* tensor, long long total, long long first, int V_) : end(tensor + total), V(V_) {
    shift = (int)(first % kPer);
    base = tensor + (first - shift);
  }
  __device__ __forceinline__ int words() const { return (V + shift + kPer - 1) / kPer; }
  __device__ __forceinline__ void load(int w, float (&z)[kPer]) const {
    const T* p = base + (long long)w * kPer;
    if (p + kPer <= end) {
      const uint4 x = *reinterpret_cast<const uint4*>(p);
      const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 2) {
          z[2 * e] = tame(__uint_as_float(u[e] << 16));
          z[2 * e + 1] = tame(__uint_as_float(u[e] & 0xffff0000u));
        } else {
          z[e] = tame(__uint_as_float(u[e]));
        }
      }
    } else {                                 // the tensor's last word
#pragma unroll
      for (int e = 0; e < kPer; ++e) z[e] = p + e < end ? value(p + e) : -INFINITY;
    }
    const int v = w * kPer - shift;
    if (v < 0 || v + kPer > V) {
#pragma unroll
      for (int e = 0; e < kPer; ++e)
        if (v + e < 0 || v + e >= V) z[e] = -INFINITY;
    }
  }
};

__device__ __forceinline__ uint32_t mapa(uint32_t addr, int rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w)
               : "memory");
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Reductions over the cluster of four floats a thread; every thread of all CTAs gets the
// same result.  `warp_sh` is the CTA's own, `all_sh` has every rank's share, in two
// buffers taken in turn: a CTA that writes into one of them again has passed the barrier
// of the other, before which everyone had read the first.
struct Exchange {
  float4 warp_sh[kWarps];
  float4 all_sh[2][kMaxCluster];
};
template <typename F>
__device__ __forceinline__ float4 reduce(Exchange& x, int& turn, int splits, float4 mine, F&& join) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    mine = join(mine, make_float4(__shfl_xor_sync(0xffffffffu, mine.x, o), __shfl_xor_sync(0xffffffffu, mine.y, o),
                                  __shfl_xor_sync(0xffffffffu, mine.z, o), __shfl_xor_sync(0xffffffffu, mine.w, o)));
  if (lane == 0) x.warp_sh[warp] = mine;
  __syncthreads();
  float4 r = x.warp_sh[0];
#pragma unroll 1
  for (int w = 1; w < kWarps; ++w) r = join(r, x.warp_sh[w]);
  if (splits == 1) {
    __syncthreads();                         // read before they are written again
    return r;
  }
  uint32_t rank;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  turn ^= 1;
  if (threadIdx.x < splits) st_cluster(mapa(smem_u32(&x.all_sh[turn][rank]), threadIdx.x), r);
  cluster_sync();
  r = x.all_sh[turn][0];
  for (int i = 1; i < splits; ++i) r = join(r, x.all_sh[turn][i]);
  return r;
}

template <typename T, Mode kMode>
__global__ void __launch_bounds__(kThreads) verify_kernel(const Args a) {
  constexpr int kPer = Row<T>::kPer;
  __shared__ Exchange ex;
  __shared__ int parent_sh[kMaxNodes], token_sh[kMaxNodes];
  __shared__ float uniform_sh[kMaxNodes];
  __shared__ float z_sh[kMaxNodes], q_sh[kMaxNodes];   // logits at a child's token: the target's, the draft's
  __shared__ int rejected_sh[kMaxNodes];               // tokens
  __shared__ float left_sh[kMaxNodes];                 // 1 / Z
  if (a.splits > 1) cluster_sync();          // every CTA is there before one writes into another
  grid_dependency_wait();
  const int split = blockIdx.x, b = blockIdx.y, n = a.n, V = a.V;
  const T* target = (const T*)a.target;
  const T* draft = (const T*)a.draft;
  if (threadIdx.x < n) {
    const int i = threadIdx.x;
    const size_t at = (size_t)b * n + i;
    int p = a.parent[at];
    bool bad = p >= i;
    if (bad) p = -1;
    if (i > 0 && p >= 0) {
      const int x = a.token[at];
      token_sh[i] = x;
      if (x < 0 || x >= V) bad = true, p = -1;         // passed over
      if (kMode != kGreedy) uniform_sh[i] = a.uniform[at];
    }
    if (bad && split == 0) record_error(a.err, SBD_DEVERR_TREE);
    parent_sh[i] = i == 0 ? -1 : p;
  }
  __syncthreads();
  int turn = 0, node = 0, count = 1;
  const bool writer = split == 0 && threadIdx.x == 0;
  const size_t out = (size_t)b * n;
  if (split == 0 && threadIdx.x < n) {
    a.path[out + threadIdx.x] = threadIdx.x == 0 ? 0 : -1;
    a.out_tokens[out + threadIdx.x] = -1;
    a.logprob[out + threadIdx.x] = 0.f;
  }
  __syncthreads();                           // (written before single places of them are)
  while (true) {
    // ---- the row's largest logit and its sum (and the draft's, where it is asked for)
    bool inner = false;
    for (int c = node + 1; c < n; ++c) inner |= parent_sh[c] == node;
    const Row<T> row(target, a.total, ((long long)b * n + node) * V, V);
    const Row<T> row_q(draft, a.total, ((long long)b * n + node) * V, V);
    const int words = row.words();
    const int w0 = (int)((long long)split * words / a.splits), w1 = (int)((long long)(split + 1) * words / a.splits);
    __syncthreads();                         // the level before is done with z_sh and q_sh
    if (threadIdx.x < n && parent_sh[threadIdx.x] == node) {
      const long long at = ((long long)b * n + node) * V + token_sh[threadIdx.x];
      z_sh[threadIdx.x] = value(target + at);
      if (kMode == kDrawn) q_sh[threadIdx.x] = value(draft + at);
    }
    Sum st{-INFINITY, 0.f}, sq{-INFINITY, 0.f};
    Best best{-INFINITY, -INFINITY, 0x7fffffff};
    auto take = [&](Sum& s, const float (&z)[kPer]) {
      float m = s.m;
#pragma unroll
      for (int e = 0; e < kPer; ++e) m = fmaxf(m, z[e]);
      if (m == -INFINITY) return;
      float sum = s.s > 0.f ? s.s * exp2f((s.m - m) * a.scale) : 0.f;
#pragma unroll
      for (int e = 0; e < kPer; ++e) sum += ex2_ftz((z[e] - m) * a.scale);
      s.m = m, s.s = sum;
    };
    for (int w = w0 + threadIdx.x; w < w1; w += kThreads) {
      float z[kPer];
      row.load(w, z);
      take(st, z);
      if (kMode == kGreedy) {
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const int v = w * kPer - row.shift + e;
          if (v >= 0 && v < V) best = better(best, Best{z[e], z[e], v});
        }
      }
      if (kMode == kDrawn && inner) {
        float q[kPer];
        row_q.load(w, q);
        take(sq, q);
      }
    }
    const float scale = a.scale;
    const float4 sums = reduce(ex, turn, a.splits, make_float4(st.m, st.s, sq.m, sq.s), [scale](float4 x, float4 y) {
      const Sum t = merge(Sum{x.x, x.y}, Sum{y.x, y.y}, scale), q = merge(Sum{x.z, x.w}, Sum{y.z, y.w}, scale);
      return make_float4(t.m, t.s, q.m, q.s);
    });
    const float m_t = sums.x == -INFINITY ? 0.f : sums.x, inv_t = sums.y > 0.f ? 1.f / sums.y : 0.f;
    const float m_q = sums.z == -INFINITY ? 0.f : sums.z, inv_q = sums.w > 0.f ? 1.f / sums.w : 0.f;
    const float log_s = logf(sums.y);
    auto join_best = [](float4 x, float4 y) {
      const Best r = better(Best{x.x, x.y, __float_as_int(x.z)}, Best{y.x, y.y, __float_as_int(y.z)});
      return make_float4(r.score, r.z, __int_as_float(r.v), 0.f);
    };
    auto prob = [&](float z) { return ex2_ftz((z - m_t) * scale) * inv_t; };
    auto prob_q = [&](float z) { return ex2_ftz((z - m_q) * scale) * inv_q; };
    // What is left of p(v) and of the draft's q(v) after the first k rejections.
    auto left = [&](float r, float q, int v, int k) {
      for (int i = 0; i < k; ++i) {
        if (kMode == kDrawn) r = fmaxf(r - q, 0.f);
        else if (v == rejected_sh[i]) r = 0.f;
        r *= left_sh[i];
      }
      return r;
    };
    // One rejection more, not normalised.
    auto rest = [&](float r, float q, int v, int k) {
      return kMode == kDrawn ? fmaxf(r - q, 0.f) : v == rejected_sh[k] ? 0.f : r;
    };
    int next = -1, said = -1;
    float said_z = 0.f;
    int k = 0;                               // rejections whose remainder is known
    bool pending = false;                    // one more, of which nothing is known yet
    if (kMode == kGreedy) {
      const float4 r = reduce(ex, turn, a.splits, make_float4(best.score, best.z, __int_as_float(best.v), 0.f), join_best);
      said = __float_as_int(r.z), said_z = r.y;
      for (int c = node + 1; c < n && next < 0; ++c)
        if (parent_sh[c] == node && token_sh[c] == said && r.x > -INFINITY) next = c;
    } else {
      for (int c = node + 1; c < n && next < 0; ++c) {
        if (parent_sh[c] != node) continue;
        if (pending) {
          // the remainder's sum, to go on with the next child
          float sum = 0.f;
          for (int w = w0 + threadIdx.x; w < w1; w += kThreads) {
            float z[kPer], q[kPer];
            row.load(w, z);
            if (kMode == kDrawn) row_q.load(w, q);
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
              const int v = w * kPer - row.shift + e;
              const float x = kMode == kDrawn ? prob_q(q[e]) : 0.f;
              sum += rest(left(prob(z[e]), x, v, k), x, v, k);
            }
          }
          const float total = reduce(ex, turn, a.splits, make_float4(sum, 0.f, 0.f, 0.f), [](float4 x, float4 y) {
                                return make_float4(x.x + y.x, 0.f, 0.f, 0.f);
                              }).x;
          if (total > 0.f) {
            __syncthreads();
            if (threadIdx.x == 0) left_sh[k] = 1.f / total;
            __syncthreads();
            ++k;
          }
          pending = false;
        }
        const int x = token_sh[c];
        const float q = kMode == kDrawn ? prob_q(q_sh[c]) : 1.f;
        const float r = left(prob(z_sh[c]), q, x, k);
        if (uniform_sh[c] * q < r) {
          next = c, said = x, said_z = z_sh[c];
        } else {
          __syncthreads();
          if (threadIdx.x == 0) rejected_sh[k] = x;
          __syncthreads();
          pending = true;
        }
      }
    }
    if (next >= 0) {
      if (writer) {
        a.path[out + count] = next;
        a.out_tokens[out + count - 1] = said;
        a.logprob[out + count - 1] = (said_z - m_t) * a.inv_tau - log_s;
      }
      ++count;
      node = next;
      continue;
    }
    // ---- the last token
    if (kMode != kGreedy) {
      // of what the last rejection leaves; where that is nothing, of what was before it
      Best after{-INFINITY, -INFINITY, 0x7fffffff}, before = after;
      const float* g = a.gumbel + (size_t)b * V;
      for (int w = w0 + threadIdx.x; w < w1; w += kThreads) {
        float z[kPer], q[kPer];
        row.load(w, z);
        if (kMode == kDrawn && (k > 0 || pending)) row_q.load(w, q);
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
          const int v = w * kPer - row.shift + e;
          if (v < 0 || v >= V) continue;
          const float noise = g[v];
          if (k == 0 && !pending) {
            before = better(before, Best{(z[e] - m_t) * a.inv_tau + noise, z[e], v});
            continue;
          }
          const float x = kMode == kDrawn ? prob_q(q[e]) : 0.f;
          const float r = left(prob(z[e]), x, v, k);
          before = better(before, Best{logf(r) + noise, z[e], v});
          if (pending) after = better(after, Best{logf(rest(r, x, v, k)) + noise, z[e], v});
        }
      }
      float4 r = make_float4(-INFINITY, 0.f, 0.f, 0.f);
      if (pending)
        r = reduce(ex, turn, a.splits, make_float4(after.score, after.z, __int_as_float(after.v), 0.f), join_best);
      if (!(r.x > -INFINITY))
        r = reduce(ex, turn, a.splits, make_float4(before.score, before.z, __int_as_float(before.v), 0.f), join_best);
      said = __float_as_int(r.z), said_z = r.y;
    }
    if (said == 0x7fffffff) said = 0, said_z = -INFINITY;   // (no number among the scores)
    if (writer) {
      a.out_tokens[out + count - 1] = said;
      a.logprob[out + count - 1] = sums.y > 0.f ? (said_z - m_t) * a.inv_tau - log_s : -INFINITY;
      a.count[b] = count;
    }
    break;
  }
  grid_dependents_launch();
}

template <typename T>
const void* kernel_of(Mode m) {
  return m == kGreedy ? (const void*)verify_kernel<T, kGreedy>
                      : m == kGiven ? (const void*)verify_kernel<T, kGiven> : (const void*)verify_kernel<T, kDrawn>;
}

}  // namespace

namespace sbd {

sbd_status verify_launch(const sbd_verify_desc& d, const VerifyTensors& t, float tau, cudaStream_t st) {
  Args a;
  const Mode mode = tau == 0.f ? kGreedy : t.draft ? kDrawn : kGiven;
  a.target = t.target;
  a.draft = t.draft;
  a.parent = t.parent;
  a.token = t.token;
  a.uniform = t.uniform;
  a.gumbel = t.gumbel;
  a.path = t.path;
  a.out_tokens = t.out_tokens;
  a.logprob = t.logprob;
  a.count = t.count;
  a.err = device_error_word();
  a.total = (long long)d.batch * d.nodes * d.vocab;
  a.n = d.nodes;
  a.V = d.vocab;
  a.inv_tau = tau == 0.f ? 1.f : 1.f / tau;
  a.scale = a.inv_tau * 1.4426950408889634f;
  const void* fn = d.dtype == SBD_DTYPE_F32 ? kernel_of<float>(mode) : kernel_of<__nv_bfloat16>(mode);
  // As many CTAs a request as one wave holds, 2048 logits each at least.
  int s = 1;
  while (s < kMaxCluster && 2ll * s * d.batch <= 2ll * num_sms() && d.vocab / (2 * s) >= 2048) s *= 2;
  while (s > 1 && cluster_slots(fn, kThreads, 0, s) < 1) s /= 2;
  a.splits = s;
  void* args[] = {(void*)&a};
  return launch_pdl(fn, dim3(s, d.batch), dim3(kThreads), 0, st, args, "verify_kernel launch", s);
}

}  // namespace sbd
