// The pages of an 8-bit KV cache: their bookkeeping and their filling.
//
//   block_tables_kernel   grows and releases the requests' pages and builds the
//                         slot map of the tokens they gain;
//   append_q8_kernel      quantises new keys and values into their slots (e4m3
//                         codes, one power-of-two scale for each page and head).
#include <math.h>

#include "paged.cuh"

namespace {

using namespace sbd_dev;

// ---------------------------------------------------------- block tables
// Per request b, with pages of P tokens: held = ceil(len / P), want =
// ceil(target / P); back = max(held - want, 0) pages return to the free stack,
// need = max(want - held, 0) leave it, new = max(target - len, 0) tokens get
// slots.  Inclusive prefix sums over the requests decide everything: page i (of
// all granted, in request order) is the i-th page released in this call, and
// once those are used up the next one from the top of the stack.  So no CTA
// reads what another one writes: all of them compute the same sums (requests
// are few) and then share the outputs out.
// Bound: latency, the chain lengths -> sums -> page -> store.  32 requests gain 8
// tokens: 3.7 us, a launch and that chain; 256 requests gain a million, 4.2 MB of
// slots and 0.6 MB of table: 8.6 us, much of it the sums that every one of 1,216 CTAs
// forms and a search of up to eight steps for four tokens (10.2 with half as many
// CTAs, which go round twice).
constexpr int kTabThreads = 256;
constexpr int kTabWarps = kTabThreads / 32;
constexpr int kTabCols = 128;                // columns of a table row per warp and turn
constexpr int kTabSlots = 4 * kTabThreads;   // slot-map entries per CTA and turn

struct TablesArgs {
  const int32_t *len, *target, *table, *n_free;
  int32_t *free_pages, *table_out, *len_out, *new_start, *slot_map, *n_free_out;
  int* err;
  int B, log2P, max_pages, n_pages, max_new;
};

struct Sums {
  long long fresh;                           // tokens
  int need, back;                            // pages (all tables have less than 2^31 entries)
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) {
  return {a.fresh + b.fresh, a.need + b.need, a.back + b.back};
}
__device__ __forceinline__ Sums shfl_up(const Sums& a, int o) {
  return {__shfl_up_sync(0xffffffffu, a.fresh, o), __shfl_up_sync(0xffffffffu, a.need, o),
          __shfl_up_sync(0xffffffffu, a.back, o)};
}
__device__ __forceinline__ int saturate(long long x) {
  return x > 0x7fffffffll ? 0x7fffffff : (int)x;
}
// The last of n ascending entries that is <= x (entry 0 is).
__device__ __forceinline__ int last_not_above(const int* a, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kTabThreads) block_tables_kernel(const TablesArgs a) {
  extern __shared__ int tab_sm[];
  int* fresh_at = tab_sm;                    // [B] tokens gained by the requests before b
  int* need_at = fresh_at + a.B;             // [B] pages they need
  int* back_at = need_at + a.B;              // [B] pages they release
  int* len_s = back_at + a.B;                // [B]
  int* after_s = len_s + a.B;                // [B] length after the call; ~ of it where one was out of range
  __shared__ Sums warp_sum_sh[kTabWarps];
  __shared__ int used_sh[kTabWarps];
  grid_dependency_wait();

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long capacity = (long long)a.max_pages << a.log2P;
  const int per = (a.B + kTabThreads - 1) / kTabThreads;
  const int b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
  int n_free = a.n_free[0];
  bool bad_page = n_free < 0 || n_free > a.n_pages, bad_len = false;
  n_free = min(max(n_free, 0), a.n_pages);

  const int last = (1 << a.log2P) - 1;
  auto pages = [&](int n) { return (n >> a.log2P) + ((n & last) != 0); };
  // a length out of range is clamped and the request left as it is
  auto request = [&](int b, int* len, int* target) {
    const int l = a.len[b], t = a.target[b];
    const bool bad = l < 0 || l > capacity || t < 0 || t > capacity;
    *len = (int)min((long long)max(l, 0), capacity);
    *target = bad ? *len : t;
    return bad;
  };
  Sums mine = {0, 0, 0};
  for (int b = b0; b < b1; ++b) {
    int l, t;
    bad_len |= request(b, &l, &t);
    mine.fresh += max(t - l, 0);
    mine.need += max(pages(t) - pages(l), 0);
    mine.back += max(pages(l) - pages(t), 0);
  }
  Sums incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Sums up = shfl_up(incl, o);
    if (lane >= o) incl = incl + up;
  }
  if (lane == 31) warp_sum_sh[warp] = incl;
  __syncthreads();
  Sums before = {0, 0, 0}, all = {0, 0, 0};
#pragma unroll
  for (int w = 0; w < kTabWarps; ++w) {
    if (w < warp) before = before + warp_sum_sh[w];
    all = all + warp_sum_sh[w];
  }
  Sums at = {before.fresh + incl.fresh - mine.fresh, before.need + incl.need - mine.need,
             before.back + incl.back - mine.back};
  const long long avail = (long long)n_free + all.back;
  // Served: all of a request's pages and slots fit.  Both sums only grow, so
  // the requests that need pages and get them come before those that do not.
  int used = 0;
  for (int b = b0; b < b1; ++b) {
    int l, t;
    const bool bad = request(b, &l, &t);
    const int fresh = max(t - l, 0), need = max(pages(t) - pages(l), 0);
    const bool served = (need == 0 || (long long)at.need + need <= avail) &&
                        (fresh == 0 || at.fresh + fresh <= a.max_new);
    fresh_at[b] = saturate(at.fresh);
    need_at[b] = at.need;
    back_at[b] = at.back;
    len_s[b] = l;
    after_s[b] = bad ? ~l : served ? t : l;
    if (served) used += need;
    if (blockIdx.x == 0) {
      a.len_out[b] = served ? t : l;
      a.new_start[b] = saturate(at.fresh);
    }
    at.fresh += fresh;
    at.need += need;
    at.back += max(pages(l) - pages(t), 0);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) used += __shfl_xor_sync(0xffffffffu, used, o);
  if (lane == 0) used_sh[warp] = used;
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) {
    used = 0;
    for (int w = 0; w < kTabWarps; ++w) used += used_sh[w];
    a.n_free_out[0] = (int)min(avail - used, (long long)a.n_pages);
    a.new_start[a.B] = saturate(all.fresh);
  }
  const int n_back = all.back;

  // the i-th page released in this call
  auto released = [&](int i) {
    const int b = last_not_above(back_at, a.B, i);
    return a.table[(size_t)b * a.max_pages + pages(after_s[b]) + (i - back_at[b])];
  };
  // the page at column p of request b after the call; -1 where it is none of the cache's,
  // which is told unless the request is left as it is
  auto page_at = [&](int b, int p) {
    const int held = pages(len_s[b]);
    int page;
    if (p < held) {
      page = a.table[(size_t)b * a.max_pages + p];
    } else {
      const int i = need_at[b] + p - held;
      page = i < n_back ? released(i) : a.free_pages[n_free - 1 - (i - n_back)];
    }
    if ((uint32_t)page < (uint32_t)a.n_pages) return page;
    if (after_s[b] < 0) return page;
    bad_page = true;
    return -1;
  };

  const int gwarp = blockIdx.x * kTabWarps + warp, gwarps = gridDim.x * kTabWarps;
  const int chunks = (a.max_pages + kTabCols - 1) / kTabCols;
  const int units = a.B * chunks;                  // <= B max_pages < 2^31
  for (int u = gwarp; u < units; u += gwarps) {
    const int b = u / chunks, c0 = (u - b * chunks) * kTabCols;
    const int after = after_s[b], keeps = pages(after < 0 ? ~after : after);
#pragma unroll
    for (int e = 0; e < kTabCols / 32; ++e) {
      const int p = c0 + 32 * e + lane;
      if (p < a.max_pages) a.table_out[(size_t)b * a.max_pages + p] = p < keeps ? page_at(b, p) : -1;
    }
  }
  // slots: four consecutive tokens a thread, mostly of one request
  for (long long s = (long long)blockIdx.x * kTabSlots + 4 * tid; s < a.max_new;
       s += (long long)gridDim.x * kTabSlots) {
    int v[4];
    // of the requests that begin at s or before, the last: it alone may hold s
    int b = last_not_above(fresh_at, a.B, (int)s), p_prev = -1, page = -1, b_prev = -1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = (int)s + e;
      v[e] = -1;
      if (t >= a.max_new || t >= all.fresh) continue;
      while (b + 1 < a.B && fresh_at[b + 1] <= t) ++b;
      if (after_s[b] <= len_s[b]) continue;          // refused
      const int pos = len_s[b] + (t - fresh_at[b]), p = pos >> a.log2P;
      if (p != p_prev || b != b_prev) page = page_at(b, p);
      p_prev = p, b_prev = b;
      v[e] = page < 0 ? -1 : (page << a.log2P) + (pos & last);
    }
    if (s + 4 <= a.max_new) {
      *reinterpret_cast<int4*>(a.slot_map + s) = make_int4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (s + e < a.max_new) a.slot_map[s + e] = v[e];
    }
  }
  // released pages go on top of the stack, the first one topmost, so that a
  // later call of the same growth gets the same pages back in the same order
  for (uint32_t i = blockIdx.x * kTabThreads + tid; i < (uint32_t)n_back; i += gridDim.x * kTabThreads) {
    int page = released((int)i);
    const long long j = (long long)n_free + n_back - 1 - i;
    if ((uint32_t)page >= (uint32_t)a.n_pages) bad_page = true, page = -1;
    if (j < a.n_pages) a.free_pages[j] = page; else bad_page = true;
  }
  if (bad_page) record_error(a.err, SBD_DEVERR_PAGE);
  if (bad_len) record_error(a.err, SBD_DEVERR_CACHE_LEN);
  grid_dependents_launch();
}

// ------------------------------------------------------ quantising append
// A segment is a run of new tokens with consecutive slots of one page.  Per
// segment and head, with a = max |x| over its finite elements:
//   s_new = 2^e, the smallest with a <= 448 2^e and e >= -126;
//   s     = s_new where the segment begins the page, else max(s_old, s_new);
//   code  = e4m3(x / s), round to nearest even; infinities saturate, NaN stays;
// and where s > s_old the codes the page holds already become e4m3(c s_old / s):
// s_old / s is a power of two, so only codes that leave the normal range round.
// That is why scales are powers of two: x / s is exact, and a page filled over many
// calls loses nothing when its scale grows, but for codes that fall below 2^-6, the
// normal range, and are rounded there to a multiple of 2^-9 s once more.
//
// A CTA finds the segments that begin in its chunk of tokens and works on them for
// some planes (K or V of a head); its 8 warps form as many teams as there are
// segments, so that one long segment (a prompt's page) is eight warps' work and eight
// single tokens are one warp's each.  A thread keeps its share of the segment in
// registers between the maximum and the codes (kHold units of 8 elements).
// Bound: HBM, 3 bytes an element of bf16.  4 x 32768 tokens of 8 heads of 128 144 us,
// 5.6 TB/s; in pages of 16 131 us.  On the way there: 377 us with the chunks of a
// plane as neighbours in the grid, 127 registers and fp32 arithmetic; 213 with maxima
// of pairs and products in bf16; 184 with addresses a constant step apart; 144 with
// the rows brought to L2 while the slots are read.
constexpr int kAppThreads = 256;
constexpr int kAppWarps = kAppThreads / 32;
constexpr int kHold = 8;

struct AppendArgs {
  const void *k_new, *v_new;
  const int32_t* slot_map;
  uint8_t *k_cache, *v_cache;
  float *k_scale, *v_scale;
  int* err;
  long long k_group_stride, k_token_stride, v_group_stride, v_token_stride;   // elements
  long long n_slots;
  int tokens, group, Hkv, log2P, chunk;
  int planes;                                // of a CTA; a plane is K or V of a head
};

// 8 consecutive elements.  Max: their largest |x| so far, NaN left out.
template <typename T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  using Max = __nv_bfloat162;
  uint32_t w[4];
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  }
  __device__ __forceinline__ __nv_bfloat162 two(int e) const {
    return *reinterpret_cast<const __nv_bfloat162*>(&w[e]);
  }
  static __device__ __forceinline__ Max none() { return __float2bfloat162_rn(0.f); }
  __device__ __forceinline__ void take_max(Max& m) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) m = __hmax2(m, __habs2(two(e)));
  }
  static __device__ __forceinline__ float size(Max m) {
    return fmaxf(__low2float(m), __high2float(m));
  }
  // e4m3 codes of 4 h .. 4 h + 3 times a power of two (exact in bf16: the products
  // are 448 at most)
  __device__ __forceinline__ uint32_t codes(int h, float inv) const {
    const __nv_bfloat162 f = __float2bfloat162_rn(inv);
    const float2 a = __bfloat1622float2(__hmul2(two(2 * h), f));
    const float2 b = __bfloat1622float2(__hmul2(two(2 * h + 1), f));
    return e4m3x4(a.x, a.y, b.x, b.y);
  }
  __device__ __forceinline__ float get(int e) const {
    return __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  }
};
template <>
struct Eight<float> {
  using Max = float;
  float w[8];
  __device__ __forceinline__ void load(const float* p) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
    w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  }
  static __device__ __forceinline__ Max none() { return 0.f; }
  __device__ __forceinline__ void take_max(Max& m) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(w[e]));
  }
  static __device__ __forceinline__ float size(Max m) { return m; }
  __device__ __forceinline__ uint32_t codes(int h, float inv) const {
    return e4m3x4(w[4 * h] * inv, w[4 * h + 1] * inv, w[4 * h + 2] * inv, w[4 * h + 3] * inv);
  }
  __device__ __forceinline__ float get(int e) const { return w[e]; }
};

// |x| of a finite x, 0 of another
__device__ __forceinline__ float finite_size(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? __uint_as_float(u) : 0.f;
}

template <typename T, int D>
__global__ void __launch_bounds__(kAppThreads, sizeof(T) == 2 ? 4 : 2) append_q8_kernel(const AppendArgs a) {
  constexpr int kUnits = D / 8;              // units of a row
  __shared__ uint32_t joins[kAppThreads / 32];       // bit i: token t0 + i goes on with a segment
  __shared__ uint32_t starts[kAppThreads / 32];      // bit i: token t0 + i begins one
  __shared__ int start_at[kAppThreads];
  __shared__ float team_max[kAppWarps];
  grid_dependency_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // The planes of a chunk of tokens are neighbours in the grid, as their rows are in
  // memory (with the chunks of a plane as neighbours, prompts of 32768 tokens took
  // 377 us: 256-byte pieces 6 KB apart).
  const int sets = (2 * a.Hkv + a.planes - 1) / a.planes;      // CTAs of a chunk
  const int t0 = (int)(blockIdx.x / sets) * a.chunk, set = (int)(blockIdx.x % sets);
  const int last = (1 << a.log2P) - 1;
  // The chunk's rows of a plane on their way to L2, while its slots are looked at or
  // the plane before is worked on.
  auto fetch_ahead = [&](int plane) {
    constexpr int kLines = D * (int)sizeof(T) / 128;           // of a row
    if (a.group < a.tokens || plane >= 2 * a.Hkv) return;
    const bool is_v = plane >= a.Hkv;
    const T* src = (const T*)(is_v ? a.v_new : a.k_new) + (long long)(is_v ? plane - a.Hkv : plane) * D;
    const long long stride = is_v ? a.v_token_stride : a.k_token_stride;
    for (int i = threadIdx.x; i < a.chunk * kLines; i += kAppThreads)
      if ((uint32_t)t0 + i / kLines < (uint32_t)a.tokens)      // (may pass 2^31)
        prefetch_l2(src + (t0 + i / kLines) * stride + i % kLines * (128 / (int)sizeof(T)));
  };
  fetch_ahead(set);

  // ---- the segments that begin in this chunk; chunk + P <= kAppThreads tokens
  // are looked at, as far as the last of them can reach
  {
    const bool here = tid < a.tokens - t0;
    const int s = here ? a.slot_map[t0 + tid] : -1;
    const int prev = here && t0 + tid > 0 ? a.slot_map[t0 + tid - 1] : -1;
    const bool valid = s >= 0 && s < a.n_slots;
    if (s >= a.n_slots && set == 0) record_error(a.err, SBD_DEVERR_PAGE);
    const bool join = valid && prev >= 0 && prev + 1 == s && (s & last) != 0;
    const uint32_t j = __ballot_sync(0xffffffffu, join);
    const uint32_t f = __ballot_sync(0xffffffffu, valid && !join && tid < a.chunk);
    if (lane == 0) joins[warp] = j, starts[warp] = f;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < warp; ++w) before += __popc(starts[w]);
    if (valid && !join && tid < a.chunk) start_at[before + __popc(f & ((1u << lane) - 1))] = tid;
    __syncthreads();
  }
  int n_seg = 0;
#pragma unroll
  for (int w = 0; w < kAppWarps; ++w) n_seg += __popc(starts[w]);
  if (n_seg == 0) return;
  int teams = 1;
  while (teams < kAppWarps && teams < n_seg) teams *= 2;
  const int team_warps = kAppWarps / teams, team_threads = 32 * team_warps;
  const int team = warp / team_warps, rank = tid - team * team_threads;

  for (int plane = set; plane < 2 * a.Hkv; plane += sets) {
  const bool is_v = plane >= a.Hkv;
  const int h = is_v ? plane - a.Hkv : plane;
  fetch_ahead(plane + sets);
  const T* src = (const T*)(is_v ? a.v_new : a.k_new) + (long long)h * D;
  const long long group_stride = is_v ? a.v_group_stride : a.k_group_stride;
  const long long token_stride = is_v ? a.v_token_stride : a.k_token_stride;
  uint8_t* cache = is_v ? a.v_cache : a.k_cache;
  float* scales = is_v ? a.v_scale : a.k_scale;

  for (int g = team; g < n_seg; g += teams) {
    const int i0 = start_at[g], t = t0 + i0;
    int end = i0 + 1;                        // the next token that does not join
    while (end < kAppThreads) {
      const int room = 32 - (end & 31);
      const uint32_t stop = ~(joins[end >> 5] >> (end & 31));
      const int run = stop ? __ffs(stop) - 1 : 32;
      end += min(run, room);
      if (run < room) break;
    }
    const int n = end - i0;
    const int slot = a.slot_map[t], off = slot & last;
    const long long page = slot >> a.log2P;
    const int units = n * kUnits;
    // A thread's units are team_threads apart, a whole number of tokens: their
    // addresses a constant step apart where tokens are.
    const T* first = src + (rank % kUnits) * 8;
    const int tok = t + rank / kUnits, step = team_threads / kUnits;
    const bool even = a.group >= a.tokens;
    auto at = [&](int e) {                   // unit rank + e team_threads
      const int i = tok + e * step;
      if (even) return first + i * token_stride;
      const int g = i / a.group;
      return first + g * group_stride + (i - g * a.group) * token_stride;
    };
    const int mine = (units - rank + team_threads - 1) / team_threads;   // this thread's units
    Eight<T> hold[kHold];
    typename Eight<T>::Max m = Eight<T>::none();
    if (even) {
      const T* p = first + tok * token_stride;
      const long long jump = step * token_stride;
#pragma unroll
      for (int e = 0; e < kHold; ++e)
        if (e < mine) hold[e].load(p + e * jump);
    } else {
#pragma unroll
      for (int e = 0; e < kHold; ++e)
        if (e < mine) hold[e].load(at(e));
    }
    const long long sc = page * a.Hkv + h;
    const float s_old = off > 0 ? scales[sc] : 0.f;
#pragma unroll
    for (int e = 0; e < kHold; ++e)
      if (e < mine) hold[e].take_max(m);
#pragma unroll 1
    for (int e = kHold; e < mine; ++e) {
      Eight<T> v;
      v.load(at(e));
      v.take_max(m);
    }
    float amax = Eight<T>::size(m);
    if (!(amax < INFINITY)) {                // some are infinite: those do not count
      amax = 0.f;
#pragma unroll 1
      for (int e = 0; e < mine; ++e) {
        Eight<T> v;
        v.load(at(e));
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, finite_size(v.get(i)));
      }
    }
    amax = warp_max(amax);
    if (team_warps > 1) {
      if (lane == 0) team_max[warp] = amax;
      asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(team_threads) : "memory");
      for (int w = 0; w < team_warps; ++w) amax = fmaxf(amax, team_max[team * team_warps + w]);
      // the maxima are read before the next segment's are written
      asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(team_threads) : "memory");
    } else {
      __syncwarp();                          // every lane has the old scale
    }
    const float s = fmaxf(s_old, scale_for(amax));
    if (rank == 0) scales[sc] = s;
    uint8_t* dst = cache + ((page * a.Hkv + h) << a.log2P) * D;
    uint8_t* to = dst + off * D + 8 * rank;
    const int hop = 8 * team_threads;
    // s is a power of two unless a caller's own scale is kept: products are exact
    if ((__float_as_uint(s) & 0x007fffffu) == 0) {
      const float inv = 1.f / s;
#pragma unroll
      for (int e = 0; e < kHold; ++e)
        if (e < mine) *reinterpret_cast<uint2*>(to + e * hop) = make_uint2(hold[e].codes(0, inv), hold[e].codes(1, inv));
#pragma unroll 1
      for (int e = kHold; e < mine; ++e) {
        Eight<T> v;
        v.load(at(e));
        *reinterpret_cast<uint2*>(to + e * hop) = make_uint2(v.codes(0, inv), v.codes(1, inv));
      }
    } else {
#pragma unroll 1
      for (int e = 0; e < mine; ++e) {
        Eight<T> v;
        v.load(at(e));
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = v.get(i) / s;
        *reinterpret_cast<uint2*>(to + e * hop) =
            make_uint2(e4m3x4(x[0], x[1], x[2], x[3]), e4m3x4(x[4], x[5], x[6], x[7]));
      }
    }
    if (off > 0 && s != s_old) {             // the page's earlier codes move to the new scale
      const float f = s_old / s;
      for (int u = rank; u < off * D / 16; u += team_threads) {
        uint4 c = *reinterpret_cast<const uint4*>(dst + 16 * u);
        c.x = e4m3x4_times(c.x, f), c.y = e4m3x4_times(c.y, f);
        c.z = e4m3x4_times(c.z, f), c.w = e4m3x4_times(c.w, f);
        *reinterpret_cast<uint4*>(dst + 16 * u) = c;
      }
    }
  }
  }
  grid_dependents_launch();
}

}  // namespace

namespace sbd {

size_t tables_smem_bytes(int B) { return (size_t)5 * B * sizeof(int); }

sbd_status tables_launch(const sbd_tables_desc& d, const int32_t* len, const int32_t* target,
                         const int32_t* table, int32_t* free_pages, const int32_t* n_free,
                         int32_t* table_out, int32_t* len_out, int32_t* new_start,
                         int32_t* slot_map, int32_t* n_free_out, cudaStream_t st) {
  TablesArgs a{len,     target,    table,    n_free,     free_pages,          table_out,
               len_out, new_start, slot_map, n_free_out, device_error_word(), d.batch,
               log2_page(d.page_size), d.max_pages, d.n_pages, d.max_new};
  const size_t smem = tables_smem_bytes(d.batch);
  if (smem > 48 * 1024) {
    const sbd_status s = allow_smem((const void*)block_tables_kernel, smem,
                                    "cudaFuncSetAttribute(block_tables_kernel)");
    if (s != SBD_OK) return s;
  }
  const long long rows = (long long)d.batch * ((d.max_pages + kTabCols - 1) / kTabCols);
  long long ctas = (rows + kTabWarps - 1) / kTabWarps;
  const long long by_slots = ((long long)d.max_new + kTabSlots - 1) / kTabSlots;
  if (by_slots > ctas) ctas = by_slots;
  if (ctas > 8 * num_sms()) ctas = 8 * num_sms();    // all that the SMs hold at once
  if (ctas < 1) ctas = 1;
  void* args[] = {(void*)&a};
  return launch_pdl((const void*)block_tables_kernel, dim3((unsigned)ctas), dim3(kTabThreads), smem,
                    st, args, "block_tables_kernel launch");
}

sbd_status append_q8_launch(const sbd_append_q8_desc& d, const void* k_new, const void* v_new,
                            const int32_t* slot_map, void* k_cache, void* v_cache, float* k_scale,
                            float* v_scale, cudaStream_t st) {
  AppendArgs a;
  a.k_new = k_new;
  a.v_new = v_new;
  a.slot_map = slot_map;
  a.k_cache = (uint8_t*)k_cache;
  a.v_cache = (uint8_t*)v_cache;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.err = device_error_word();
  a.k_group_stride = d.k_group_stride;
  a.k_token_stride = d.k_token_stride;
  a.v_group_stride = d.v_group_stride;
  a.v_token_stride = d.v_token_stride;
  a.n_slots = (long long)d.n_pages * d.page_size;
  a.tokens = d.tokens;
  a.group = d.group;
  a.Hkv = d.n_kv_heads;
  a.log2P = log2_page(d.page_size);
  // Few tokens: short chunks and a plane a CTA, so that every SM has some of them
  // (256 tokens of 16 segments 4.1 us; chunks of 8: 4.7).  Many: as many tokens as
  // kHold units a thread hold (at 64 dimensions as many as the chunk's table allows:
  // 65536 tokens of 8 heads 49 us, 60 in chunks of 128), and two planes a CTA where
  // that leaves enough CTAs (one: 10 % slower, four: 2 to 7 %).
  const int planes = 2 * d.n_kv_heads;
  const long long jobs = planes * ((d.tokens + 63ll) / 64);
  a.chunk = jobs < 4ll * num_sms() ? 16 : d.head_dim == 64 ? kAppThreads - d.page_size : 128;
  a.planes = 1;
  while (a.planes < 2 && planes * ((d.tokens + 127ll) / 128) / (2 * a.planes) >= 8ll * num_sms()) a.planes *= 2;
  const bool f32 = d.dtype == SBD_DTYPE_F32;
  const void* fn = d.head_dim == 128
                       ? (f32 ? (const void*)append_q8_kernel<float, 128>
                              : (const void*)append_q8_kernel<__nv_bfloat16, 128>)
                       : (f32 ? (const void*)append_q8_kernel<float, 64>
                              : (const void*)append_q8_kernel<__nv_bfloat16, 64>);
  void* args[] = {(void*)&a};
  const long long ctas =
      (d.tokens + (long long)a.chunk - 1) / a.chunk * ((planes + a.planes - 1) / a.planes);
  if (ctas > 0x7fffffffll) return fail(SBD_ERR_UNSUPPORTED, "%lld CTAs >= 2^31", ctas);
  return launch_pdl(fn, dim3((unsigned)ctas), dim3(kAppThreads), 0, st, args,
                    "append_q8_kernel launch");
}

}  // namespace sbd
