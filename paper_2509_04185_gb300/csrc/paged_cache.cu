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
// Bound: latency.  The arrays are kilobytes; the chain is lengths -> sums ->
// page -> store.
constexpr int kTabThreads = 256;
constexpr int kTabWarps = kTabThreads / 32;
constexpr int kTabCols = 128;                // columns of a table row per warp and turn
constexpr int kTabSlots = 4 * kTabThreads;   // slot-map entries per CTA and turn

struct TablesArgs {
  const int32_t *len, *target, *table, *n_free;
  int32_t *free_pages, *table_out, *len_out, *new_start, *slot_map, *n_free_out;
  int* err;
  int B, P, max_pages, n_pages, max_new;
};

struct Sums {
  long long fresh, need, back;               // tokens, pages, pages
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
  int* after_s = len_s + a.B;                // [B] length after the call
  __shared__ Sums warp_sum_sh[kTabWarps];
  __shared__ long long used_sh[kTabWarps];
  grid_dependency_wait();

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long capacity = (long long)a.max_pages * a.P;
  const int per = (a.B + kTabThreads - 1) / kTabThreads;
  const int b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
  int n_free = a.n_free[0];
  bool bad_page = n_free < 0 || n_free > a.n_pages, bad_len = false;
  n_free = min(max(n_free, 0), a.n_pages);

  auto pages = [&](int n) { return n / a.P + (n % a.P != 0); };
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
  const long long avail = n_free + all.back;
  // Served: all of a request's pages and slots fit.  Both sums only grow, so
  // the requests that need pages and get them come before those that do not.
  long long used = 0;
  for (int b = b0; b < b1; ++b) {
    int l, t;
    request(b, &l, &t);
    const int fresh = max(t - l, 0), need = max(pages(t) - pages(l), 0);
    const bool served = (need == 0 || at.need + need <= avail) &&
                        (fresh == 0 || at.fresh + fresh <= a.max_new);
    fresh_at[b] = saturate(at.fresh);
    need_at[b] = saturate(at.need);
    back_at[b] = saturate(at.back);
    len_s[b] = l;
    after_s[b] = served ? t : l;
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
  const int n_back = saturate(all.back);

  // the i-th page released in this call
  auto released = [&](int i) {
    const int b = last_not_above(back_at, a.B, i);
    return a.table[(size_t)b * a.max_pages + pages(after_s[b]) + (i - back_at[b])];
  };
  // the page at column p of request b after the call
  auto page_at = [&](int b, int p) {
    const int held = pages(len_s[b]);
    if (p < held) return a.table[(size_t)b * a.max_pages + p];
    const int i = need_at[b] + p - held;
    return i < n_back ? released(i) : a.free_pages[n_free + n_back - 1 - i];
  };

  const int gwarp = blockIdx.x * kTabWarps + warp, gwarps = gridDim.x * kTabWarps;
  const int chunks = (a.max_pages + kTabCols - 1) / kTabCols;
  const long long units = (long long)a.B * chunks;
  for (long long u = gwarp; u < units; u += gwarps) {
    const int b = (int)(u / chunks), c0 = (int)(u % chunks) * kTabCols;
    const int keeps = pages(after_s[b]);
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
      const int pos = len_s[b] + (t - fresh_at[b]), p = pos / a.P;
      if (p != p_prev || b != b_prev) page = page_at(b, p);
      p_prev = p, b_prev = b;
      v[e] = page * a.P + pos % a.P;
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
  for (int i = blockIdx.x * kTabThreads + tid; i < n_back; i += gridDim.x * kTabThreads) {
    const int page = released(i);
    const long long j = (long long)n_free + n_back - 1 - i;
    if (page < 0 || page >= a.n_pages || j >= a.n_pages) bad_page = true;
    if (j < a.n_pages) a.free_pages[j] = page;
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
// That is why scales are powers of two: a page filled over many calls loses
// nothing each time its scale grows, and x / s is exact.
//
// One CTA per (chunk of tokens, head, K or V) finds the segments that begin in
// its chunk; its 8 warps form as many teams as there are segments, so that one
// long segment (a prompt's page) is eight warps' work and eight single tokens
// are one warp's each.  A thread keeps its share of the segment in registers
// between the maximum and the codes (kHold units of 8 elements).
// Bound: HBM, 3 bytes an element of bf16.
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
  int tokens, group, Hkv, P, chunk;
};

template <typename T>
struct Eight;                                // 8 consecutive elements
template <>
struct Eight<__nv_bfloat16> {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
};
template <>
struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
};

// |x| of a finite x, 0 of another
__device__ __forceinline__ float finite_size(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? __uint_as_float(u) : 0.f;
}

template <typename T, int D>
__global__ void __launch_bounds__(kAppThreads) append_q8_kernel(const AppendArgs a) {
  constexpr int kUnits = D / 8;              // units of a row
  __shared__ uint32_t joins[kAppThreads / 32];       // bit i: token t0 + i goes on with a segment
  __shared__ uint32_t starts[kAppThreads / 32];      // bit i: token t0 + i begins one
  __shared__ int start_at[kAppThreads];
  __shared__ float team_max[kAppWarps];
  grid_dependency_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int h = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  const int t0 = blockIdx.x * a.chunk;

  // ---- the segments that begin in this chunk; chunk + P <= kAppThreads tokens
  // are looked at, as far as the last of them can reach
  {
    const int t = t0 + tid;
    const int s = t < a.tokens ? a.slot_map[t] : -1;
    const int prev = t > 0 && t < a.tokens ? a.slot_map[t - 1] : -1;
    const bool valid = s >= 0 && s < a.n_slots;
    if (s >= a.n_slots && h == 0 && !is_v) record_error(a.err, SBD_DEVERR_PAGE);
    const bool join = valid && prev >= 0 && prev + 1 == s && s % a.P != 0;
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
    const int slot = a.slot_map[t], off = slot % a.P;
    const long long page = slot / a.P;
    const int units = n * kUnits;
    auto at = [&](int u) {
      const int tok = t + u / kUnits;
      return src + (tok / a.group) * group_stride + (tok % a.group) * token_stride + (u % kUnits) * 8;
    };
    Eight<T> hold[kHold];
#pragma unroll
    for (int e = 0; e < kHold; ++e)
      if (rank + e * team_threads < units) hold[e].load(at(rank + e * team_threads));
    const long long sc = page * a.Hkv + h;
    const float s_old = off > 0 ? scales[sc] : 0.f;
    float amax = 0.f;
    auto take_max = [&](const Eight<T>& v) {
      float x[8];
      v.get(x);
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, finite_size(x[e]));
    };
#pragma unroll
    for (int e = 0; e < kHold; ++e)
      if (rank + e * team_threads < units) take_max(hold[e]);
    for (int u = rank + kHold * team_threads; u < units; u += team_threads) {
      Eight<T> v;
      v.load(at(u));
      take_max(v);
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
    uint8_t* dst = cache + (page * a.Hkv + h) * (long long)(a.P * D);
    const float inv = 1.f / s;               // a power of two unless a caller's scale is kept
    const bool exact = (__float_as_uint(s) & 0x007fffffu) == 0;
    auto put = [&](int u, const Eight<T>& v) {
      float x[8];
      v.get(x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = exact ? x[e] * inv : x[e] / s;
      uint2 c;
      c.x = e4m3x4(x[0], x[1], x[2], x[3]);
      c.y = e4m3x4(x[4], x[5], x[6], x[7]);
      *reinterpret_cast<uint2*>(dst + (long long)off * D + 8 * u) = c;
    };
#pragma unroll
    for (int e = 0; e < kHold; ++e)
      if (rank + e * team_threads < units) put(rank + e * team_threads, hold[e]);
    for (int u = rank + kHold * team_threads; u < units; u += team_threads) {
      Eight<T> v;
      v.load(at(u));
      put(u, v);
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
               d.page_size, d.max_pages, d.n_pages, d.max_new};
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
  if (ctas > 2 * num_sms()) ctas = 2 * num_sms();
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
  a.P = d.page_size;
  // few tokens: short chunks, so that every SM has some of them
  const long long jobs = 2ll * d.n_kv_heads * ((d.tokens + 63) / 64);
  a.chunk = jobs < 4ll * num_sms() ? 16 : d.page_size > 64 ? d.page_size : 64;
  const bool f32 = d.dtype == SBD_DTYPE_F32;
  const void* fn = d.head_dim == 128
                       ? (f32 ? (const void*)append_q8_kernel<float, 128>
                              : (const void*)append_q8_kernel<__nv_bfloat16, 128>)
                       : (f32 ? (const void*)append_q8_kernel<float, 64>
                              : (const void*)append_q8_kernel<__nv_bfloat16, 64>);
  void* args[] = {(void*)&a};
  return launch_pdl(fn, dim3((unsigned)((d.tokens + a.chunk - 1) / a.chunk), d.n_kv_heads, 2),
                    dim3(kAppThreads), 0, st, args, "append_q8_kernel launch");
}

}  // namespace sbd
