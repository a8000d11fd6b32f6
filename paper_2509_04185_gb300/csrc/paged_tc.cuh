// What the kernels of block attention over the paged 8-bit cache on the tcgen05 tensor
// cores share: the instructions, the operands' layouts, the codes, the loads of pages
// and the merge of splits.
#pragma once

#include "paged.cuh"

namespace sbd_dev {

constexpr int kTile = 128;                   // keys of an MMA; a step is two tiles
constexpr int kMaxStages = 8;
constexpr int kBlkKeys = 32;                 // block keys, padded
constexpr int kMaxSplits = 16;
constexpr int kMaxOrder = 128;               // sequences that a launch sorts by length

// ------------------------------------------------------------ tcgen05 PTX
__device__ __forceinline__ void tc_alloc(uint32_t* dst_smem, uint32_t ncols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                   smem_u32(dst_smem)),
               "r"(ncols)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tc_dealloc(uint32_t taddr, uint32_t ncols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols)
               : "memory");
}
__device__ __forceinline__ void tc_fence_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_fence_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void tc_mma_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc,
                                          uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tc_mma_bf16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc,
                                            uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
          smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tc_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
                 "=r"(r[7])
               : "r"(taddr));
}
__device__ __forceinline__ void tc_wait_ld() {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint64_t* bar,
                                            int c0, int c1, int c2) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2)
      : "memory");
}
// The maximum over a warp (NaN only where every lane has it).
__device__ __forceinline__ float redux_max(float v) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}

// The same, NaN where any lane has it; and of two.
__device__ __forceinline__ float redux_max_nan(float v) {
  float r;
  asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float max_nan(float x, float y) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}

// Shared-memory operands of rows of `W` = 32, 64 or 128 bytes, swizzled over W:
// 16-byte pieces of a row permuted by the row's place, the pattern repeating every
// 8 rows (one 8 W-byte atom).
template <int W>
__device__ __forceinline__ uint32_t swz(uint32_t base, int row, int piece) {
  constexpr int kMask = W / 16 - 1;
  constexpr int kShift = W == 128 ? 0 : W == 64 ? 1 : 2;
  return base + row * W + ((piece ^ ((row >> kShift) & kMask)) << 4);
}
// Descriptor of such an operand: 8-row groups 8 W apart; `next` bytes from one
// atom to the next along a row (MN-major operands wider than an atom).
template <int W>
__device__ __forceinline__ uint64_t desc(uint32_t addr, uint32_t next = 16) {
  constexpr uint64_t kMode = W == 128 ? 2 : W == 64 ? 4 : 6;
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(next >> 4) << 16 |
         (uint64_t)(8 * W >> 4) << 32 | (uint64_t)1 << 46 | kMode << 61;
}
// e4m3 A and B, fp32 D.
__device__ __forceinline__ uint32_t idesc_f8(int M, int N, bool mn_major) {
  return 1u << 4 | (mn_major ? 1u : 0u) << 15 | (mn_major ? 1u : 0u) << 16 |
         (uint32_t)(N >> 3) << 17 | (uint32_t)(M >> 4) << 24;
}
// bf16 A and B, both MN-major, fp32 D.
__device__ __forceinline__ uint32_t idesc_bf16_mn(int M, int N) {
  return 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (uint32_t)(N >> 3) << 17 |
         (uint32_t)(M >> 4) << 24;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint4 v) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z),
               "r"(v.w)
               : "memory");
}
// The same without a branch (what it stores is the warp's, one lane does it).
__device__ __forceinline__ void st_shared_v4_if(bool p, uint32_t addr, float x, float y, float z, float w) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %5, 0;\n\t@q st.shared.v4.f32 [%0], {%1,%2,%3,%4};\n\t}"
               ::"r"(addr), "f"(x), "f"(y), "f"(z), "f"(w), "r"((uint32_t)p)
               : "memory");
}
__device__ __forceinline__ void bar_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// ------------------------------------------------------------ clusters
// (Every thread of the cluster comes to both, the wait as late as it can.)
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t mapa_shared(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
// Stores into a CTA of the cluster that count towards the bytes its barrier waits for.
__device__ __forceinline__ void st_async(uint32_t addr, float v, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.f32 [%0], %1, [%2];" ::"r"(addr), "f"(v), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void st_async(uint32_t addr, float4 v, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(addr),
               "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(bar)
               : "memory");
}
// Bytes that come to CTA `split` for the merge of `rows` rows of D floats and a sum.
template <int D>
__device__ __forceinline__ uint32_t merge_bytes(int rows, int split, int splits) {
  return split < rows ? (uint32_t)((rows - split + splits - 1) / splits * splits * (4 * D + 4)) : 0u;
}

// floor(x / d) for 0 <= x < 2^20 and inv = 1 / d to a few units in the last place: x + 1/2
// is half a unit of 1 / d away from where the quotient steps.  (A division of integers is
// 30 instructions, and what runs once waits for L2 to bring its code: 300 clocks for 8.)
__device__ __forceinline__ int whole_part(int x, float inv) { return __float2int_rz(((float)x + 0.5f) * inv); }

struct Args {
  const __nv_bfloat16 *q, *kb, *vb;
  const float *ks, *vs;
  const int32_t *table, *lens;
  __nv_bfloat16* out;
  int* err;
  int B, k, Hq, Hkv, G, M, max_pages, n_pages, n_causal, splits, chunks;
  int page_log2;
  int order;                 // blockIdx.z -> sequence by descending length
  float scale_log2;
  float inv_G, inv_chunks;   // 1 / G, 1 / chunks
  // The block position of packed row x.
  __device__ __forceinline__ int position(int x) const { return whole_part(x, inv_G); }
};

// A tile's page scales: of the keys; of the values over the largest of their step; that.
struct PageScales {
  float ks[kMaxStages][8], vw[kMaxStages][8], vref[kMaxStages];
};

__device__ __forceinline__ float finite_size(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? __uint_as_float(u) : 0.f;
}
// 16 consecutive bf16 values of a row; the D / 16 lanes of a row lie together.
template <int D>
struct Piece {
  uint4 w[2];
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    w[0] = reinterpret_cast<const uint4*>(p)[0];
    w[1] = reinterpret_cast<const uint4*>(p)[1];
  }
  __device__ __forceinline__ void zero() { w[0] = w[1] = make_uint4(0, 0, 0, 0); }
  // x = s (hi + lo) for the row's scale s, which it returns: the codes become
  // piece `c` of rows hi_row and lo_row of the operand at `base`.  What is not
  // finite becomes NaN.
  __device__ __forceinline__ float store(uint32_t base, int hi_row, int lo_row, int c) const {
    float x[16];
    const uint32_t u[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
    float amax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[2 * e] = __uint_as_float(u[e] << 16);
      x[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
      amax = fmaxf(amax, fmaxf(finite_size(x[2 * e]), finite_size(x[2 * e + 1])));
    }
#pragma unroll
    for (int o = 1; o < D / 16; o *= 2) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    const float s = scale_for(amax), inv = 1.f / s;
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float y[4], h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = x[4 * e + i];
        y[i] = (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u ? __int_as_float(0x7fffffff) : v * inv;
      }
      hi[e] = e4m3x4(y[0], y[1], y[2], y[3]);
      e4m3x4_values(hi[e], h);
      lo[e] = e4m3x4(y[0] - h[0], y[1] - h[1], y[2] - h[2], y[3] - h[3]);
    }
    st_shared_v4(swz<D>(base, hi_row, c), make_uint4(hi[0], hi[1], hi[2], hi[3]));
    st_shared_v4(swz<D>(base, lo_row, c), make_uint4(lo[0], lo[1], lo[2], lo[3]));
    return s;
  }
};

// The sequence of rank z in descending length (ties by index), for launches of more than
// one wave: the longest start first.  All threads come; B <= kMaxOrder, `sh` has room for
// as many.  (Lengths compared from shared memory, four at a time: from global memory one
// by one took a microsecond of a CTA's seven at 64 sequences.)
__device__ __forceinline__ int longest_first(const int32_t* lens, int B, int cap, int z, int* sh, int* pick) {
  const int t = threadIdx.x;
  if (t < kMaxOrder) sh[t] = t < B ? min(max(lens[t], 0), cap) : -1;
  __syncthreads();
  if (t < B) {
    const int mine = sh[t];
    int rank = 0;
    for (int j = 0; j < B; j += 4) {
      const int4 x = *reinterpret_cast<const int4*>(sh + j);
      rank += (x.x > mine || (x.x == mine && j < t)) + (x.y > mine || (x.y == mine && j + 1 < t)) +
              (x.z > mine || (x.z == mine && j + 2 < t)) + (x.w > mine || (x.w == mine && j + 3 < t));
    }
    if (rank == z) *pick = t;
  }
  __syncthreads();
  return *pick;
}

// One warp brings the tiles t_begin .. t_begin + nc - 1 of a sequence's cache into the
// ring of kStages stages (a tile of K, then of V) and their pages' scales to kSlots
// places; kStep tiles are a step.  No copy is in flight when it returns.
template <int D, int kStages, int kSlots, int kStep>
__device__ __forceinline__ void load_tiles(const CUtensorMap& tmap_k, const CUtensorMap& tmap_v, const Args& a, int b,
                                           int hkv, int len, int t_begin, int nc, uint32_t ring, PageScales& pages,
                                           uint64_t* kv_full, uint64_t* kv_empty, uint64_t* tail_bar) {
  const int lane = threadIdx.x & 31;
  const int P = 1 << a.page_log2, per_tile = kTile >> a.page_log2;
  const int p_first = t_begin * per_tile;
  const int p_end = (int)((min((t_begin + nc) * (long long)kTile, (long long)len) + P - 1) >> a.page_log2);
  const int32_t* table = a.table + (size_t)b * a.max_pages;
  // Pages come in windows of 32, one a lane: ids a window ahead, their scales a
  // tile into the window before.  A page out of range lies past the tensor's
  // end for the copy, which reads zeros there.
  auto id_at = [&](int p) {
    if (p >= p_end) return -1;
    const int id = table[p];
    if (id >= 0 && id < a.n_pages) return id;
    record_error(a.err, SBD_DEVERR_PAGE);
    return a.n_pages;
  };
  auto scale_at = [&](const float* s, int id) {
    return id >= 0 && id < a.n_pages ? s[(size_t)id * a.Hkv + hkv] : 0.f;
  };
  int id = id_at(p_first + lane), id_next = id_at(p_first + 32 + lane);
  float ks = scale_at(a.ks, id), vs = scale_at(a.vs, id), ks_next = 0.f, vs_next = 0.f;
  const int per_window = 32 / per_tile;
  int issued = 0;
  for (int j = 0; j < nc; ++j) {
    const int w = j % per_window;
    if (w == 0 && j > 0) {
      id = id_next, ks = ks_next, vs = vs_next;
      id_next = id_at(p_first + (j / per_window + 1) * 32 + lane);
    }
    if (w == 1) ks_next = scale_at(a.ks, id_next), vs_next = scale_at(a.vs, id_next);
    const int stage = j % kStages, slot = j % kSlots;
    const uint32_t at = ring + (uint32_t)stage * 2 * kTile * D;
    const bool freed = mbar_wait(&kv_empty[stage], ((j / kStages) & 1) ^ 1, a.err);
    if (!__all_sync(0xffffffffu, freed)) break;
    const int valid = max(0, min(kTile, len - (t_begin + j) * kTile)), n_pg = (valid + P - 1) >> a.page_log2;
    const int src = (w * per_tile + lane) & 31;      // lane i < n_pg: the tile's page i
    const int pg = __shfl_sync(0xffffffffu, id, src);
    // Values past the length may be anything (NaN); the products go on to the
    // next multiple of 32 keys, so those become zeros once the copy is there.
    const bool tail = (valid & 31) != 0;
    uint64_t* bar = tail ? tail_bar : &kv_full[stage];
    // The copies first; the scales (whose loads may still be on their way) are in
    // place before the barrier's one arrival.
    if (lane < n_pg) {
      const int row = pg < a.n_pages ? pg * a.Hkv + hkv : a.n_pages * a.Hkv;
      tma_load_3d(at + lane * P * D, &tmap_k, bar, 0, 0, row);
      tma_load_3d((at + kTile * D) + lane * P * D, &tmap_v, bar, 0, 0, row);
    }
    issued = j + 1;
    const float k_sc = __shfl_sync(0xffffffffu, ks, src);
    const float v_sc = __shfl_sync(0xffffffffu, vs, src);
    // the largest value scale of the step's pages (lanes without a page have 0)
    const int first = (w & ~(kStep - 1)) * per_tile;
    const float v_max = redux_max(lane >= first && lane < first + kStep * per_tile ? vs : 0.f);
    if (lane < 8) {                                  // (places without a page: weights of keys past the length)
      pages.ks[slot][lane] = lane < n_pg ? k_sc : 0.f;
      pages.vw[slot][lane] = lane >= n_pg ? 0.f : v_max > 0.f ? v_sc / v_max : v_sc * 0.f;
    }
    if (lane == 0) pages.vref[slot] = v_max;
    __syncwarp();
    if (lane == 0) mbar_arrive_expect_tx(bar, 2 * n_pg * P * D);
    if (tail) {
      mbar_wait(tail_bar, 0, a.err);
      const int end = (valid + 31) & ~31;
      for (int c = lane; c < (end - valid) * (D / 16); c += 32)
        st_shared_v4((at + kTile * D) + valid * D + 16 * c, make_uint4(0, 0, 0, 0));
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&kv_full[stage]);
    }
  }
  // no copy is in flight when the CTA ends, whatever became of its consumers
  for (int j = max(0, issued - kStages); j < issued; ++j)
    mbar_wait(&kv_full[j % kStages], (j / kStages) & 1, a.err);
}

// The CTAs of a cluster are the splits of one (sequence, KV head, chunk); CTA `split`
// has all splits' normalised rows split, split + splits, ... (`rows`, kPStride floats
// each) and their log2-sum-exps in its shared memory.  A warp a row.
template <int D, int R, int kWarps>
__device__ __forceinline__ void merge_rows(const Args& a, const float* rows, const float* lse, int b, int hkv, int chunk,
                                           int split) {
  constexpr int kPStride = D + 4;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kPer = D / 32;
#pragma unroll 1
  for (int slot = warp; slot * a.splits + split < R; slot += kWarps) {
    const int row = chunk * R + slot * a.splits + split;
    if (row >= a.M) break;
    const float l = lane < a.splits ? lse[slot * a.splits + lane] : -INFINITY;
    const float mx = redux_max(l);
    const float w = l == -INFINITY ? 0.f : ex2_ftz(l - mx);
    const float inv = __fdividef(1.f, warp_sum(w));
    const float* src = rows + slot * a.splits * kPStride + kPer * lane;
    float o[kPer];
#pragma unroll
    for (int c = 0; c < kPer; ++c) o[c] = 0.f;
#pragma unroll 2
    for (int s = 0; s < a.splits; ++s) {
      const float ws = __shfl_sync(0xffffffffu, w, s);
      if (!(ws == 0.f)) {
#pragma unroll
        for (int c = 0; c < kPer; ++c) o[c] = fmaf(ws, src[s * kPStride + c], o[c]);
      }
    }
    const int i = a.position(row);
    __nv_bfloat16* dst =
        a.out + (((size_t)b * a.k + i) * a.Hq + hkv * a.G + row - i * a.G) * D + kPer * lane;
#pragma unroll
    for (int c = 0; c < kPer; c += 2)
      *reinterpret_cast<__nv_bfloat162*>(dst + c) = __floats2bfloat162_rn(o[c] * inv, o[c + 1] * inv);
  }
}

// The end of a CTA of such a cluster, after its own pushes; every thread comes.  A CTA
// whose rows do not come in time writes none.  No CTA ends before all of the cluster have
// pushed: the barrier's arrival goes before the merge, its wait behind it.  Pushes issued
// may still be on their way then, and the one whose wait gave up has not seen them arrive:
// it waits again.
template <int D, int R, int kWarps>
__device__ __forceinline__ void merge_in_cluster(const Args& a, const float* rows, const float* lse, int b, int hkv, int chunk,
                                                 int split, uint64_t* merge_bar) {
  __syncwarp();
  cluster_arrive();
  const bool come = __all_sync(0xffffffffu, mbar_wait(merge_bar, 0, a.err));
  if (come) merge_rows<D, R, kWarps>(a, rows, lse, b, hkv, chunk, split);
  __syncwarp();
  cluster_wait();
  if (!come) mbar_wait(merge_bar, 0, a.err);
}

struct TcKernel {
  const void* fn;
  size_t smem;
  int threads;
};

}  // namespace sbd_dev

namespace sbd {

// The kernel with rows on the lanes, 128 packed rows a CTA.
sbd_dev::TcKernel paged_rows_kernel_for(int D);

}  // namespace sbd
