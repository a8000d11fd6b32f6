// Verification of drafted tokens: the walk down a tree of nodes that accepts tokens by
// the target's probabilities and given random numbers (include/sbd.h has the rule).
//
// Probabilities are powers of two over a sum, p(v) = 2^(z_v c - M) / S with c = log2(e) / tau
// and the whole number M = ceil(max z c): parts of a row that took different M are brought
// together by exact factors, and z c - M is rounded once.  (Where the walk comes to a row whose
// largest logit is so far from 0 that z c has no such M, or that is masked altogether, it begins
// again in a form for any row: far_walk.)  What a row is needed for is M, S, the values at a few
// drafted tokens, and, where the walk ends, one argmax over
//   ln r(v) + gumbel(v),   r = what is left of p after the rejected children:
//   r_0 = p,  r_(k+1)(v) = max(r_k(v) - q(v), 0) / Z_k   (draft with probabilities)
//                        = r_k(v) / Z_k, 0 at the rejected token  (without)
// r_k is a function of the logits at v and of the scalars Z, so nothing is stored for it:
// a pass over the row evaluates it.  A request is a thread-block cluster, each CTA has a
// slice of the vocabulary, and what they need of one another goes through distributed
// shared memory: every CTA leaves its share of a sum in all others, each of which adds up in
// the same order, and so comes to the same numbers and decisions as the others.
//
// Bounds and figures (128256 logits in bf16, draft's rows too).  One request, three of seven
// tokens accepted: 12.4 us, a chain of latencies: launch 2, tree 1.5, a level 2.5 to 3 (loads 1,
// reductions over warps, CTA and cluster 1, the decision with its code 0.7), the last token's
// pass 3.  64 requests of 15 nodes, none to three levels: 50 us, of which the bytes are 14.5;
// the passes of a request follow one another, and at first the exponentials of all of them
// are as long as their bytes (3.5 us a level on 152 SMs), at last few requests are left.
// On the way: maxima that are no whole numbers and reductions in turn 131 us; whole numbers
// and one barrier 89; words of 16 bytes without bounds to check 58; which element is the best
// looked up once and not in every word (16 of 36 instructions) 53.
// Registers: 64 a thread for four CTAs an SM, where the instances with draft's rows spill (bf16
// 108 bytes stored and 168 loaded, fp32 56 and 32); three CTAs, with 12 bytes, take 56 us.
#include <math.h>

#include <type_traits>

#include "sbd_internal.cuh"

namespace {

using namespace sbd_dev;

constexpr int kMaxNodes = 64;
constexpr int kMaxCluster = 16;
constexpr float kLimit = 8388608.f;          // of a largest logit over tau: so far a row is in range

enum Mode { kGreedy, kGiven, kDrawn };       // tau = 0; drafts without, with probabilities

struct Args {
  const void *target, *draft;
  const int32_t *parent, *token;
  const float *uniform, *gumbel;
  int32_t *path, *out_tokens;
  float* logprob;
  int32_t* count;
  int* err;
  int n, V, splits;
  int slice;                 // words of a CTA
  int ahead;                 // rows are fetched ahead
  float scale, limit;        // log2(e) / tau and kLimit tau (tau 1 where it is 0)
};

__device__ __forceinline__ float redux_max(float v) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// log2 x (below 2^-126: -inf); within 2^-22, absolutely near 1.
__device__ __forceinline__ float lg2_ftz(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^x for the whole numbers x <= 0 that references differ by (0 from -126 on).
__device__ __forceinline__ float pow2_diff(float x) { return ex2_ftz(x); }

// The logits of a row: whole words of 16 bytes between the aligned places c0 and c1 (word w
// has elements kPer w - shift ...), and up to 2 kPer - 2 edges, one by one.
template <typename T>
struct Row {
  static constexpr int kPer = 16 / sizeof(T);
  static constexpr uint32_t kNone = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;   // -inf
  const T* base;             // aligned
  int shift, c0, c1, head, edges;
  __device__ __forceinline__ Row() {}
  __device__ __forceinline__ Row(const T* tensor, long long first, int V) {
    shift = (int)first & (kPer - 1);
    base = tensor + (first - shift);
    c0 = shift ? 1 : 0;
    c1 = max(c0, (int)(((uint32_t)V + shift) / kPer));
    head = shift ? min(V, kPer - shift) : 0;
    edges = max(head, V - c1 * kPer + shift + head);
  }
  __device__ __forceinline__ uint4 load(int w) const {
    return *reinterpret_cast<const uint4*>(base + (long long)w * kPer);
  }
  __device__ __forceinline__ int element(int w) const { return w * kPer - shift; }
  // Edge i < edges.
  __device__ __forceinline__ int edge(int i) const { return i < head ? i : c1 * kPer - shift + (i - head); }
  static __device__ __forceinline__ uint4 none() { return make_uint4(kNone, kNone, kNone, kNone); }
  static __device__ __forceinline__ void get(const uint4& x, float (&z)[kPer]) {
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 2) {
        z[2 * e] = __uint_as_float(u[e] << 16);
        z[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
      } else {
        z[e] = __uint_as_float(u[e]);
      }
    }
  }
};
// The largest element of words (NaN left out).
template <int N>
__device__ __forceinline__ float largest(const uint4 (&x)[N], const __nv_bfloat16*) {
  auto two = [](uint32_t u) { return *reinterpret_cast<const __nv_bfloat162*>(&u); };
  __nv_bfloat162 m = __float2bfloat162_rn(-INFINITY);
#pragma unroll
  for (int h = 0; h < N; ++h)
    m = __hmax2(__hmax2(m, __hmax2(two(x[h].x), two(x[h].y))), __hmax2(two(x[h].z), two(x[h].w)));
  return fmaxf(__low2float(m), __high2float(m));
}
template <int N>
__device__ __forceinline__ float largest(const uint4 (&x)[N], const float*) {
  float m = -INFINITY;
#pragma unroll
  for (int h = 0; h < N; ++h)
    m = fmaxf(fmaxf(m, fmaxf(__uint_as_float(x[h].x), __uint_as_float(x[h].y))),
              fmaxf(__uint_as_float(x[h].z), __uint_as_float(x[h].w)));
  return m;
}
// Two fp32 operations an instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float value(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float value(const float* p) { return *p; }

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

// Reductions of up to kN times four floats over the cluster; every warp of it has the same
// results.  `join` reduces over a warp (all lanes have its result); a warp's go to the CTA,
// the CTA's, by a warp each, to all of the cluster.  The buffers are taken in turn: a CTA that
// writes into one of them again has passed the barrier of the other, before which everyone
// had read the first.
template <int kWarps, int kN>
struct Exchange {
  float4 warps[2][kN][kWarps];
  float4 ranks[2][kN][kMaxCluster];
};
template <int kM, int kWarps, int kN, typename F>
__device__ __forceinline__ void reduce(Exchange<kWarps, kN>& x, int& turn, int splits, int count, float4 (&mine)[kM], float4 none,
                                       F&& join) {
  static_assert(kM <= kN && kN <= kWarps, "a warp each");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  turn ^= 1;
#pragma unroll
  for (int i = 0; i < kM; ++i) {
    if (i >= count) continue;
    mine[i] = join(mine[i]);
    if (lane == 0) x.warps[turn][i][warp] = mine[i];
  }
  __syncthreads();
  if (splits == 1) {
#pragma unroll
    for (int i = 0; i < kM; ++i)
      if (i < count) mine[i] = join(lane < kWarps ? x.warps[turn][i][lane] : none);
    return;
  }
  if (warp < count) {
    const float4 all = join(lane < kWarps ? x.warps[turn][warp][lane] : none);
    uint32_t rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    if (lane < splits) st_cluster(mapa(smem_u32(&x.ranks[turn][warp][rank]), lane), all);
  }
  __syncwarp();
  cluster_sync();
#pragma unroll
  for (int i = 0; i < kM; ++i)
    if (i < count) mine[i] = join(lane < splits ? x.ranks[turn][i][lane] : none);
}

// M and S of a part of a row.  A row whose largest logit is beyond the limit, up or down (a
// small tau, a row of nothing but masked logits), has no whole number M to which z c is exact:
// it has the largest logit itself in the place of M, and S, of powers of (z - M) c, negative.
struct Stat {
  float M, S;
};
// z against the largest logit m of a row: the distance, 0 or less.  NaN is the least; of
// infinities the largest are alike and leave nothing to the others.
__device__ __forceinline__ float below(float z, float m) {
  if (fabsf(m) == INFINITY) return fmaxf(z, -INFINITY) == m ? 0.f : -INFINITY;
  return fmaxf(z - m, -INFINITY);
}
__device__ __forceinline__ float ln_prob(float z, Stat x, float c2) {
  const float y = x.S < 0.f ? below(z, x.M) * c2 : fmaf(z, c2, -x.M);
  return fmaf(y, 0.69314718f, -logf(fabsf(x.S)));
}
__device__ __forceinline__ Stat warp_stat(Stat a) {
  const float M = redux_max(a.M);
  return {M, warp_sum(a.S * pow2_diff(a.M - M))};
}
// The best score and where it is: the first element of its word, or an edge.  (Which element
// of the word is looked up once, in the best one: told apart in every word it was 16 of 36
// instructions an element.)
struct Best {
  float score;
  int v;
};
__device__ __forceinline__ void offer(Best& b, float score, int v) {   // (in ascending order, not NaN)
  if (!(score <= b.score)) b.score = score, b.v = v;
}
__device__ __forceinline__ Best better(Best a, Best b) {   // (b may have nothing: NaN)
  return b.score > a.score || (b.score == a.score && b.v < a.v) ? b : a;
}
__device__ __forceinline__ Best warp_best(Best a) {
  const float top = redux_max(a.score);      // (not NaN: a NaN is never better)
  return {top, (int)__reduce_min_sync(0xffffffffu, a.score == top ? a.v : 0x7fffffff)};
}

__device__ __forceinline__ float tame(float z, float limit) { return fminf(fmaxf(z, -limit), limit); }   // NaN: the least
__device__ __forceinline__ void take_one(Stat& s, float z, float c2, float limit) {
  const float M = fmaxf(s.M, ceilf(tame(z, limit) * c2));
  s.S = fmaf(s.S, pow2_diff(s.M - M), ex2_ftz(fmaf(tame(z, limit), c2, -M)));
  s.M = M;
}
// M and S of the elements of words w0, w0 + step, ... below w1 one by one: of a part of a row
// that has a NaN in it.  (What is beyond the limit counts as the limit here: it shows in M.)
template <typename T>
__device__ __noinline__ Stat slow_stat(const T* elements, int w0, int w1, int step, float c2, float limit) {
  Stat s{-2.f * kLimit, 0.f};
  for (int w = w0; w < w1; w += step)
    for (int e = 0; e < Row<T>::kPer; ++e) take_one(s, value(elements + (long long)w * Row<T>::kPer + e), c2, limit);
  return s;
}

// The stat of a row beyond the limit, in two passes: its largest logit, then the sum.  Every
// thread of the cluster comes, with the same result.  (It finds its places itself: what would be
// kept for it costs the walk registers.)
template <typename T, int kWarps, int kN>
__device__ __noinline__ Stat far_stat(Exchange<kWarps, kN>& ex, int turn, const T* tensor, long long first, int V, int slice,
                                      int splits, float c2) {
  constexpr int kPer = Row<T>::kPer, step = 32 * kWarps;
  const int split = blockIdx.x, tid = threadIdx.x;
  const Row<T> row(tensor, first, V);
  const int from = min(row.c1, row.c0 + split * slice), w1 = min(row.c1, from + slice), w0 = from + tid;
  const T* edge = split == 0 && tid < row.edges ? tensor + first + row.edge(tid) : nullptr;
  float m = edge ? fmaxf(value(edge), -INFINITY) : -INFINITY;
  // (four words in flight, as in the walk)
  auto words = [&](auto&& f) {
#pragma unroll 1
    for (int w = w0; w < w1; w += 4 * step) {
      uint4 x[4];
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        x[h] = Row<T>::none();
        if (w + h * step < w1) x[h] = row.load(w + h * step);
      }
      f(x, w);
    }
  };
  words([&](const uint4 (&x)[4], int) { m = fmaxf(m, largest(x, (const T*)nullptr)); });
  float4 part[1] = {make_float4(m, 0.f, 0.f, 0.f)};
  reduce(ex, turn, splits, 1, part, make_float4(-INFINITY, 0.f, 0.f, 0.f),
         [](float4 x) { return make_float4(redux_max(x.x), 0.f, 0.f, 0.f); });
  m = part[0].x;
  float sum = edge ? ex2_ftz(below(value(edge), m) * c2) : 0.f;
  words([&](const uint4 (&x)[4], int w) {
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      float z[kPer], s = 0.f;                // (a word's sum for itself: not one long chain)
      Row<T>::get(x[h], z);
#pragma unroll
      for (int e = 0; e < kPer; ++e) s += ex2_ftz(below(z[e], m) * c2);
      if (w + h * step < w1) sum += s;       // (no words: -inf, which a row of nothing else counts)
    }
  });
  part[0] = make_float4(sum, 0.f, 0.f, 0.f);
  reduce(ex, turn, splits, 1, part, make_float4(0.f, 0.f, 0.f, 0.f),
         [](float4 x) { return make_float4(warp_sum(x.x), 0.f, 0.f, 0.f); });
  return Stat{m, -part[0].x};
}

// What a CTA has in shared memory.
template <int kWarps, int kAhead>
struct Shared {
  Exchange<kWarps, kAhead> ex;
  unsigned long long child[kMaxNodes];       // of a node, a bit each
  int token[kMaxNodes];
  float uniform[kMaxNodes];
  float z[kMaxNodes], q[kMaxNodes];          // logits at a child's token: the target's, the draft's
  float4 stat[kMaxNodes];                    // rows' M and S, of the target and of the draft (greedy: largest, where)
  int path[kMaxNodes], said[kMaxNodes];      // the walk, told at its end: nodes, tokens,
  float said_z[kMaxNodes];                   // their logits, and their rows' M and S
  Stat said_st[kMaxNodes];
  int rejected[kMaxNodes];                   // tokens
  float left[kMaxNodes];                     // 1 / Z
};
// Where requests are few (512 threads a CTA) a level is a chain of latencies, 2.8 us of one
// request's 12.4: so M and S of several rows are made at once, of a node, its first child,
// that one's first child ..., which the walk is likely to come to, and both rows of a node
// together.  Where they are many, one row after the other, only as the walk comes to them.
template <Mode kMode, int kThreads>
constexpr int rows_ahead() { return kMode == kDrawn && kThreads == 512 ? 2 : 1; }

// The walk; `parent`: of node threadIdx.x.  Returns how many nodes are on the path, all told but
// for their outputs, or, unless kFar, 0 where it comes to a row beyond the limit.  (Two walks,
// since the registers and instructions for any row cost the other 3 to 4 us of 50.)
template <typename T, Mode kMode, int kThreads, bool kFar>
__device__ __forceinline__ int walk(const Args& a, Shared<kThreads / 32, rows_ahead<kMode, kThreads>()>& sh, int& turn, int parent) {
  using R = Row<T>;
  constexpr int kPer = R::kPer;
  constexpr int kAhead = kFar ? 1 : rows_ahead<kMode, kThreads>();
  constexpr bool kBoth = kAhead == 2;
  constexpr int kHold = kBoth ? 2 : 4;                 // words of a row that a thread has in flight
  const int split = blockIdx.x, b = blockIdx.y, n = a.n, V = a.V, tid = threadIdx.x;
  const T* target = (const T*)a.target;
  const T* draft = (const T*)a.draft;
  const size_t out = (size_t)b * n;
  int node = 0, count = 1;
  const float c2 = a.scale;
  auto tame = [&](float z) { return ::tame(z, a.limit); };
  // A row's M below the one: its largest logit is beyond the limit, or it has none; from the
  // other on: beyond it on the other side.  In range a logit below the limit counts nothing.
  const float low = 256.f - a.limit * c2, high = a.limit * c2 - 1.f;
  auto is_out = [&](float M) { return M < low || M >= high; };
  unsigned long long known = 0;              // nodes whose rows' M and S are known
  while (true) {
    const unsigned long long children = sh.child[node];
    const bool use_q = kMode == kDrawn && children != 0;
    // ---- M and S of the row (and of the draft's, where it is asked for)
    Stat st, sq;
    Best best;
    if constexpr (kFar) {
      if (parent == node) {                  // a child's logits (behind a barrier when they are read)
        const long long at = ((long long)b * n + node) * V + sh.token[tid];
        sh.z[tid] = value(target + at);
        if (kMode == kDrawn) sh.q[tid] = value(draft + at);
      }
      st = far_stat<T>(sh.ex, turn, target, ((long long)b * n + node) * V, V, a.slice, a.splits, c2);
      if (use_q) sq = far_stat<T>(sh.ex, turn, draft, ((long long)b * n + node) * V, V, a.slice, a.splits, c2);
    } else if (kAhead == 1 || !(known >> node & 1)) {
      int list[kAhead] = {node}, several = 1;
      unsigned long long in = 1ull << node;
#pragma unroll
      for (int i = 1; i < kAhead; ++i) {
        const unsigned long long c = sh.child[list[i - 1]];
        list[i] = c ? __ffsll(c) - 1 : list[i - 1];
        if (c) several = i + 1, in |= 1ull << list[i];
      }
      const int rows = kAhead == 1 ? 1 : several;
      if (kAhead > 1) known |= in;
      // a child's logits, stored once the rows' loads are under way, too
      const bool is_child = kMode != kGreedy && parent >= 0 && in >> parent & 1;
      float child_z = 0.f, child_q = 0.f;
      if (is_child) {
        const long long at = ((long long)b * n + parent) * V + sh.token[tid];
        child_z = value(target + at);
        if (kMode == kDrawn) child_q = value(draft + at);
      }
      Stat t[kAhead], d[kAhead];
      Best top[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) t[i] = d[i] = Stat{-2.f * kLimit, 0.f}, top[i] = Best{NAN, 0x7fffffff};
      // As they are: a NaN shows in the sum, and the thread's share is taken again, slowly.  A
      // logit beyond the limit shows in M (what is only just beyond leaves the sum finite), as
      // does a row that is low altogether.
      auto take = [&](Stat& s, const uint4 (&x)[kHold]) {
        const float M = fmaxf(s.M, ceilf(tame(largest(x, (const T*)nullptr)) * c2));
        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
        for (int h = 0; h < kHold; ++h) {
          float z[kPer];
          R::get(x[h], z);
#pragma unroll
          for (int e = 0; e < kPer; e += 2) {
            const float2 y = fma2(make_float2(z[e], z[e + 1]), make_float2(c2, c2), make_float2(-M, -M));
            sum = add2(sum, make_float2(ex2_ftz(y.x), ex2_ftz(y.y)));
          }
        }
        s.S = fmaf(s.S, pow2_diff(s.M - M), sum.x + sum.y);
        s.M = M;
      };
      // The rows' places in both tensors, and this CTA's words of them.
      R place[kAhead];
      long long first[kAhead];
      int from[kAhead], to[kAhead];
      auto has_q = [&](int i) { return kMode == kDrawn && sh.child[list[i]] != 0; };
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        if (i >= rows) continue;
        first[i] = ((long long)b * n + list[i]) * V;
        place[i] = R(target, first[i], V);
        from[i] = min(place[i].c1, place[i].c0 + split * a.slice), to[i] = min(place[i].c1, from[i] + a.slice);
      }
      // This thread's edge of a single row, on its way with the row (two rows leave no registers for it).
      const int edge0 = kAhead == 1 && split == 0 && tid < place[0].edges ? place[0].edge(tid) : -1;
      float edge_z = 0.f, edge_q = 0.f;
      if (edge0 >= 0) {
        edge_z = value(target + first[0] + edge0);
        if (has_q(0)) edge_q = value(draft + first[0] + edge0);
      }
      const long long to_draft = reinterpret_cast<const char*>(draft) - reinterpret_cast<const char*>(target);
      auto load_q = [&](int i, int w) {
        return *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(place[i].base) + to_draft + 16ll * w);
      };
#pragma unroll 1
      for (int o = tid; o < a.slice; o += kHold * kThreads) {
        uint4 x[kAhead][kHold], y[kBoth ? kAhead : 1][kHold];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          if (i >= rows) continue;
          const bool both = kBoth && has_q(i);
#pragma unroll
          for (int h = 0; h < kHold; ++h) {
            const int w = from[i] + o + h * kThreads;
            x[i][h] = R::none();
            if (w < to[i]) x[i][h] = place[i].load(w);
            if (kBoth) y[kBoth ? i : 0][h] = R::none();
            if (both && w < to[i]) y[kBoth ? i : 0][h] = load_q(i, w);
          }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          if (i >= rows) continue;
          take(t[i], x[i]);
          if (kBoth && has_q(i)) take(d[i], y[kBoth ? i : 0]);
          if (kMode == kGreedy) {
#pragma unroll
            for (int h = 0; h < kHold; ++h) {
              const uint4 one[1] = {x[i][h]};
              const int w = from[i] + o + h * kThreads;
              if (w < to[i]) offer(top[i], fmaxf(largest(one, (const T*)nullptr), -INFINITY), place[i].element(w));
            }
          }
        }
      }
      if (!kBoth && kMode == kDrawn && use_q) {        // (kAhead is 1)
#pragma unroll 1
        for (int w = from[0] + tid; w < to[0]; w += kHold * kThreads) {
          uint4 y[kHold];
#pragma unroll
          for (int h = 0; h < kHold; ++h) {
            y[h] = R::none();
            if (w + h * kThreads < to[0]) y[h] = load_q(0, w + h * kThreads);
          }
          take(d[0], y);
        }
      }
      // The first child's rows on their way to L2: the walk is likely to go there.
      if (kAhead == 1 && a.ahead && children) {
        const int c = __ffsll(children) - 1;
        const T* there = place[0].base + (long long)(c - node) * V;
        const bool its_q = kMode == kDrawn && sh.child[c] != 0;
        for (int w = from[0] + tid * 8; w < to[0]; w += kThreads * 8) {        // a line each
          prefetch_l2(there + (long long)w * kPer);
          if (its_q) prefetch_l2(reinterpret_cast<const char*>(there + (long long)w * kPer) + to_draft);
        }
      }
      if (is_child) sh.z[tid] = child_z, sh.q[tid] = child_q;
      float4 mine[kAhead];
      const float4 none = make_float4(-2.f * kLimit, 0.f, kMode == kGreedy ? -INFINITY : -2.f * kLimit,
                                      __int_as_float(kMode == kGreedy ? 0x7fffffff : 0));
      auto join = [](float4 x) {
        const Stat t = warp_stat(Stat{x.x, x.y});
        if (kMode == kGreedy) {
          const Best r = warp_best(Best{x.z, __float_as_int(x.w)});
          return make_float4(t.M, t.S, r.score, __int_as_float(r.v));
        }
        if (kMode == kGiven) return make_float4(t.M, t.S, 0.f, 0.f);
        const Stat q = warp_stat(Stat{x.z, x.w});
        return make_float4(t.M, t.S, q.M, q.S);
      };
      // The rest of a row's share: slowly what has to be, and the thread's edge.
      auto finish = [&](int i) {
        const R& r = place[i];
        const T* row_t = target + first[i];
        const T* row_d = draft + first[i];
        const int edge = kAhead == 1 ? edge0 : split == 0 && tid < r.edges ? r.edge(tid) : -1;
        if (!(t[i].S < INFINITY)) t[i] = slow_stat<T>(row_t - r.shift, from[i] + tid, to[i], kThreads, c2, a.limit);
        if (has_q(i) && !(d[i].S < INFINITY)) d[i] = slow_stat<T>(row_d - r.shift, from[i] + tid, to[i], kThreads, c2, a.limit);
        if (edge >= 0) {
          const float z = kAhead == 1 ? edge_z : value(row_t + edge);
          take_one(t[i], z, c2, a.limit);
          if (has_q(i)) take_one(d[i], kAhead == 1 ? edge_q : value(row_d + edge), c2, a.limit);
          if (kMode == kGreedy) top[i] = better(Best{fmaxf(z, -INFINITY), edge}, top[i]);
        }
        if (kMode == kGreedy) {                        // the element of the best word
          if (top[i].v == 0x7fffffff) top[i].score = -INFINITY;
          const int v = top[i].v;
          if (top[i].score == redux_max(top[i].score) && v >= r.element(from[i]) && v < r.element(to[i])) {
            float z[kPer];
            R::get(r.load((v + r.shift) / kPer), z);
#pragma unroll
            for (int e = kPer - 1; e >= 0; --e)
              if (fmaxf(z[e], -INFINITY) == top[i].score) top[i].v = v + e;
          }
        }
        mine[i] = make_float4(t[i].M, t[i].S, d[i].M, d[i].S);
        if (kMode == kGreedy) mine[i].z = top[i].score, mine[i].w = __int_as_float(top[i].v);
      };
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (i < rows) finish(i);
      reduce(sh.ex, turn, a.splits, rows, mine, none, join);
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (kAhead > 1 && i < rows && tid == 0) sh.stat[list[i]] = mine[i];
      if (kAhead > 1) __syncthreads();
      else st = Stat{mine[0].x, mine[0].y}, sq = Stat{mine[0].z, mine[0].w}, best = Best{mine[0].z, __float_as_int(mine[0].w)};
    }
    if (kAhead > 1) {
      const float4 x = sh.stat[node];
      st = Stat{x.x, x.y}, sq = Stat{x.z, x.w}, best = Best{x.z, __float_as_int(x.w)};
    }
    const long long first = ((long long)b * n + node) * V;
    const R row(target, first, V), row_q(draft, first, V);       // (alike but for the base)
    const int w0 = min(row.c1, row.c0 + split * a.slice), w1 = min(row.c1, w0 + a.slice);
    const int edge = split == 0 && tid < row.edges ? row.edge(tid) : -1;   // this thread's
    const T* target_row = target + first;
    const T* draft_row = draft + first;
    if (!kFar && (is_out(st.M) || (use_q && is_out(sq.M)))) {
      if (kMode != kGreedy) return 0;
      // (of a greedy walk the row's law is only told)
      st = far_stat<T>(sh.ex, turn, target, first, V, a.slice, a.splits, c2);
    }
    const float inv_s = __fdividef(1.f, fabsf(st.S)), inv_q = __fdividef(1.f, fabsf(sq.S));   // (S is in 1/2 .. 2^31)
    // log2 of what a logit counts, S not taken off (NaN: NaN, or -inf)
    auto log2_p = [&](float z) { return kFar ? below(z, st.M) * c2 : fmaf(z, c2, -st.M); };
    auto log2_q = [&](float z) { return kFar ? below(z, sq.M) * c2 : fmaf(z, c2, -sq.M); };
    auto prob = [&](float z) { return fmaxf(ex2_ftz(log2_p(z)), 0.f) * inv_s; };             // (NaN: 0)
    auto prob_q = [&](float z) { return fmaxf(ex2_ftz(log2_q(z)), 0.f) * inv_q; };
    // (All earlier steps are taken again in every pass: c rejected children cost c passes and c^2 / 2
    // steps an element.  What is left of the vocabulary is not kept between passes.)
    // What is left of p at elements v, v + 1, ... after the first k rejections (and one more,
    // `after`), times S and not normalised by the last ones' sum.
    const float q_of_p = inv_q * fabsf(st.S);
    auto remainder = [&](float (&z)[kPer], float (&q)[kPer], int v, int k, bool after, float (&r)[kPer]) {
#pragma unroll
      for (int e = 0; e < kPer; e += 2) {
        float2 x = kFar ? make_float2(log2_p(z[e]), log2_p(z[e + 1]))
                        : fma2(make_float2(z[e], z[e + 1]), make_float2(c2, c2), make_float2(-st.M, -st.M));
        r[e] = ex2_ftz(x.x), r[e + 1] = ex2_ftz(x.y);
        if (kMode == kDrawn) {
          x = kFar ? make_float2(log2_q(q[e]), log2_q(q[e + 1]))
                   : fma2(make_float2(q[e], q[e + 1]), make_float2(c2, c2), make_float2(-sq.M, -sq.M));
          q[e] = fmaxf(ex2_ftz(x.x), 0.f), q[e + 1] = fmaxf(ex2_ftz(x.y), 0.f);      // (NaN: 0)
        }
      }
      if (kMode == kDrawn) {
#pragma unroll 1
        for (int i = 0; i < k; ++i) {
          const float f = sh.left[i];
#pragma unroll
          for (int e = 0; e < kPer; ++e) r[e] = fmaxf(fmaf(-q_of_p, q[e], r[e]), 0.f) * f;
        }
#pragma unroll
        for (int e = 0; e < kPer; ++e) r[e] = fmaxf(after ? fmaf(-q_of_p, q[e], r[e]) : r[e], 0.f);
      } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e) r[e] = fmaxf(r[e], 0.f);
#pragma unroll 1
        for (int i = 0; i < k + after; ++i) {
          const uint32_t at = (uint32_t)(sh.rejected[i] - v);
          if (at < kPer) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) r[e] = e == (int)at ? 0.f : r[e];
          }
        }
      }
    };
    // The words of this CTA's slice, two in flight with all that belongs to them, as f(values
    // of both rows, noise, first element, places), and this thread's edge alike.
    auto each = [&](bool with_q, auto noisy, const float* g, auto&& f) {
      constexpr bool kNoisy = decltype(noisy)::value;
      // (the noise of a word is as many aligned words of four where the row is)
      const bool aligned = kNoisy && ((long long)b * V - row.shift) % 4 == 0;
#pragma unroll 1
      for (int w = w0 + tid; w < w1; w += 2 * kThreads) {
        uint4 x[2], y[2];
        float noise[2][kPer];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (w + h * kThreads >= w1) continue;
          x[h] = row.load(w + h * kThreads);
          if (with_q) y[h] = row_q.load(w + h * kThreads);
          const float* at = g + row.element(w + h * kThreads);
          if (kNoisy && aligned) {
#pragma unroll
            for (int e = 0; e < kPer; e += 4) {
              const float4 n4 = *reinterpret_cast<const float4*>(at + e);
              noise[h][e] = n4.x, noise[h][e + 1] = n4.y, noise[h][e + 2] = n4.z, noise[h][e + 3] = n4.w;
            }
          } else if (kNoisy) {
#pragma unroll
            for (int e = 0; e < kPer; ++e) noise[h][e] = at[e];
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (w + h * kThreads >= w1) continue;
          float z[kPer], q[kPer];
          R::get(x[h], z);
          if (with_q) R::get(y[h], q);
          f(z, q, noise[h], row.element(w + h * kThreads), kPer);
        }
      }
      if (edge >= 0) {                         // (the other places -inf)
        float z[kPer], q[kPer], noise[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) z[e] = q[e] = noise[e] = -INFINITY;
        z[0] = value(target_row + edge);
        if (with_q) q[0] = value(draft_row + edge);
        if (kNoisy) noise[0] = g[edge];
        f(z, q, noise, edge, 1);
      }
    };
    int next = -1, said = -1;
    float said_z = 0.f;
    int k = 0;                               // rejections whose remainder is known
    bool pending = false;                    // one more, of which nothing is known yet
    if (kMode == kGreedy) {
      said = best.v == 0x7fffffff ? 0 : best.v, said_z = best.score;   // (nothing but NaN: 0)
      for (unsigned long long c = children; c && next < 0; c &= c - 1)
        if (sh.token[__ffsll(c) - 1] == said) next = __ffsll(c) - 1;
    } else {
      for (unsigned long long todo = children; todo && next < 0; todo &= todo - 1) {
        const int c = __ffsll(todo) - 1;
        if (pending) {
          // the remainder's sum, to go on with the next child
          float sum = 0.f;
          each(kMode == kDrawn, std::false_type(), nullptr, [&](float (&z)[kPer], float (&q)[kPer], float (&)[kPer], int v, int places) {
            float r[kPer];
            remainder(z, q, v, k, true, r);
#pragma unroll
            for (int e = 0; e < kPer; ++e) sum += e < places ? r[e] : 0.f;
          });
          float4 part[1] = {make_float4(sum, 0.f, 0.f, 0.f)};
          reduce(sh.ex, turn, a.splits, 1, part, make_float4(0.f, 0.f, 0.f, 0.f),
                 [](float4 x) { return make_float4(warp_sum(x.x), 0.f, 0.f, 0.f); });
          const float total = part[0].x * inv_s;
          if (total > 0.f) {
            if (tid == 0) sh.left[k] = 1.f / total;
            __syncthreads();
            ++k;
          }
          pending = false;
        }
        // r(x): step by step with a draft's probabilities; without, p(x) over what is left of it
        const int x = sh.token[c];
        const float q = kMode == kDrawn ? prob_q(sh.q[c]) : 1.f;
        float r = prob(sh.z[c]);
        for (int i = 0; i < k; ++i) {
          if (kMode == kDrawn) r = fmaxf(r - q, 0.f) * sh.left[i];
          else if (x == sh.rejected[i]) r = 0.f;
        }
        if (kMode == kGiven && k > 0) r *= sh.left[k - 1];
        if (sh.uniform[c] * q < r) {
          next = c, said = x, said_z = sh.z[c];
        } else {
          __syncthreads();                   // (what was here is read)
          if (tid == 0) sh.rejected[k] = x;
          __syncthreads();
          pending = true;
        }
      }
    }
    if (next >= 0) {
      if (tid == 0) sh.path[count] = next, sh.said[count - 1] = said, sh.said_z[count - 1] = said_z, sh.said_st[count - 1] = st;
      ++count;
      node = next;
      continue;
    }
    // ---- the last token
    if (kMode != kGreedy) {
      // of what the last rejection leaves; where that is nothing, of what was before it
      const float* g = a.gumbel + (size_t)b * V;
      bool after = pending;
      auto evaluate = [&](float (&z)[kPer], float (&q)[kPer], float (&score)[kPer], int v) {
        if (k == 0 && !after) {
#pragma unroll
          for (int e = 0; e < kPer; ++e) score[e] = fmaf(log2_p(z[e]), 0.69314718f, score[e]);
        } else {
          float r[kPer];
          remainder(z, q, v, k, after, r);
#pragma unroll
          for (int e = 0; e < kPer; ++e) score[e] = fmaf(lg2_ftz(r[e]), 0.69314718f, score[e]);
        }
      };
      float4 r;
      while (true) {
        best = Best{NAN, 0x7fffffff};
        each(kMode == kDrawn && (k > 0 || after), std::true_type(), g,
             [&](float (&z)[kPer], float (&q)[kPer], float (&score)[kPer], int v, int places) {
               evaluate(z, q, score, v);
               float top = -INFINITY;
#pragma unroll
               for (int e = 0; e < kPer; ++e) top = fmaxf(top, e < places ? score[e] : -INFINITY);
               if (places == kPer) offer(best, top, v);
               else best = better(Best{top, v}, best);
             });
        if (best.v == 0x7fffffff) best.score = -INFINITY;
        float4 part[1] = {make_float4(best.score, __int_as_float(best.v), 0.f, 0.f)};
        reduce(sh.ex, turn, a.splits, 1, part, make_float4(-INFINITY, __int_as_float(0x7fffffff), 0.f, 0.f), [](float4 x) {
          const Best y = warp_best(Best{x.x, __float_as_int(x.y)});
          return make_float4(y.score, __int_as_float(y.v), 0.f, 0.f);
        });
        r = part[0];
        if (!after || r.x > -INFINITY) break;
        after = false;
      }
      // The thread whose word it is finds the element and tells it.
      if (best.v == __float_as_int(r.y)) {
        const int v = best.v;
        said = v, said_z = value(target_row + v);
        if (v >= row.element(w0) && v < row.element(w1)) {
          float z[kPer], q[kPer], score[kPer];
#pragma unroll
          for (int e = 0; e < kPer; ++e) {
            z[e] = value(target_row + v + e);
            if (kMode == kDrawn && (k > 0 || after)) q[e] = value(draft_row + v + e);
            score[e] = g[v + e];
          }
          evaluate(z, q, score, v);
#pragma unroll
          for (int e = kPer - 1; e >= 0; --e)
            if (fmaxf(score[e], -INFINITY) == best.score) said = v + e;
          said_z = value(target_row + said);
        }
        a.out_tokens[out + count - 1] = said;
        a.logprob[out + count - 1] = ln_prob(said_z, st, c2);
      }
    }
    else if (tid == 0) {
      sh.said[count - 1] = said, sh.said_z[count - 1] = said_z, sh.said_st[count - 1] = st;
    }
    break;
  }
  return count;
}

// The walk in the form for any row: every row's largest logit first, in a pass of its own.  (64
// trees at tau = 1e-6, whose rows are all beyond the limit: 98 us, 51 at tau = 1; without draft's
// rows 54 and 36.5.)
template <typename T, Mode kMode, int kThreads>
__device__ __noinline__ int far_walk(const Args& a, Shared<kThreads / 32, rows_ahead<kMode, kThreads>()>& sh, int turn, int parent) {
  __syncthreads();                           // (what the other walk left is read)
  return walk<T, kMode, kThreads, true>(a, sh, turn, parent);
}

template <typename T, Mode kMode, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 256 ? 4 : kMode == kDrawn ? 1 : 2) verify_kernel(const __grid_constant__ Args a) {
  __shared__ Shared<kThreads / 32, rows_ahead<kMode, kThreads>()> sh;
  if (a.splits > 1) cluster_sync();          // every CTA is there before one writes into another
  grid_dependency_wait();
  const int split = blockIdx.x, b = blockIdx.y, n = a.n, V = a.V, tid = threadIdx.x;
  const size_t out = (size_t)b * n;
  if (tid < kMaxNodes) sh.child[tid] = 0;
  __syncthreads();
  int parent = -1;                           // of node tid
  if (tid < n) {
    const int p = a.parent[out + tid];
    bool bad = p >= tid;
    if (!bad && tid > 0 && p >= 0) {
      const int x = a.token[out + tid];
      sh.token[tid] = x;
      bad = x < 0 || x >= V;                 // passed over
      if (kMode != kGreedy) sh.uniform[tid] = a.uniform[out + tid];
      if (!bad) parent = p, atomicOr(&sh.child[p], 1ull << tid);
    }
    if (bad && split == 0) record_error(a.err, SBD_DEVERR_TREE);
  }
  __syncthreads();
  // The walk's noise on its way to L2 (and below, a row ahead).
  if (kMode != kGreedy) {
    const float* g = a.gumbel + (size_t)b * V;
    const int part = (V + a.splits - 1) / a.splits, v1 = min(V, (split + 1) * part);
    for (int v = split * part + tid * 32; v < v1; v += kThreads * 32) prefetch_l2(g + v);
  }
  int turn = 0;
  int count = walk<T, kMode, kThreads, false>(a, sh, turn, parent);
  if constexpr (kMode != kGreedy)
    if (count == 0) count = far_walk<T, kMode, kThreads>(a, sh, turn, parent);
  grid_dependents_launch();
  if (split != 0) return;
  __syncthreads();
  if (tid < n) {
    const bool on = tid < count;
    a.path[out + tid] = !on ? -1 : tid == 0 ? 0 : sh.path[tid];
    if (kMode == kGreedy || tid != count - 1) {          // (the last token is told already)
      a.out_tokens[out + tid] = on ? sh.said[tid] : -1;
      a.logprob[out + tid] = on ? ln_prob(sh.said_z[tid], sh.said_st[tid], a.scale) : 0.f;
    }
    if (tid == 0) a.count[b] = count;
  }
}

template <typename T, int kThreads>
const void* kernel_of(Mode m) {
  return m == kGreedy  ? (const void*)verify_kernel<T, kGreedy, kThreads>
         : m == kGiven ? (const void*)verify_kernel<T, kGiven, kThreads>
                       : (const void*)verify_kernel<T, kDrawn, kThreads>;
}
template <int kThreads>
const void* kernel_for(int dtype, Mode m) {
  return dtype == SBD_DTYPE_F32 ? kernel_of<float, kThreads>(m) : kernel_of<__nv_bfloat16, kThreads>(m);
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
  a.n = d.nodes;
  a.V = d.vocab;
  const float t1 = tau == 0.f ? 1.f : tau;
  a.scale = 1.4426950408889634f / t1;
  a.limit = kLimit * t1;
  // As many CTAs a request as the SMs hold at once, 2048 logits each at least: of 256
  // threads, or of 512 where the largest cluster leaves SMs without work.
  const long long slots = 4ll * num_sms();
  int s = 1;
  while (s < kMaxCluster && 2ll * s * d.batch <= slots && d.vocab / (2 * s) >= 2048) s *= 2;
  const int threads = s * d.batch <= num_sms() ? 512 : 256;
  const void* fn = threads == 512 ? kernel_for<512>(d.dtype, mode) : kernel_for<256>(d.dtype, mode);
  while (s > 1 && cluster_slots(fn, threads, 0, s) < 1) s /= 2;
  a.splits = s;
  const int per = d.dtype == SBD_DTYPE_F32 ? 4 : 8;
  a.ahead = s * d.batch <= 2 * num_sms();
  a.slice = (int)(((long long)d.vocab + per - 1) / per + s - 1) / s;
  void* args[] = {(void*)&a};
  return launch_pdl(fn, dim3(s, d.batch), dim3(threads), 0, st, args, "verify_kernel launch", s);
}

}  // namespace sbd
