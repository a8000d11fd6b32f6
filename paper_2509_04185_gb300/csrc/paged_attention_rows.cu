// Block attention over the paged 8-bit cache on the tcgen05 tensor cores, rows on the
// lanes: bf16 activations with more than 32 packed rows (paged_attention_tc.cu has less).
//
//   S[row, key] = Q K^T     A = the rows' hi codes, then their lo codes (x / s = hi + lo,
//                           as there), B = K tile (128 keys, as the cache has it)
//   O[row, dim] = P V       A = P in fp16, from tensor memory, B = V tile in fp16
//
// A thread of the softmax owns a row: its maximum and sum are the thread's own, where
// with keys on the lanes each of them is a reduction over a warp and a trip through
// shared memory for every row.  V becomes fp16 once a tile (a code times its page's scale
// over the tile's largest; exact for powers of two down to 2^-15 of it): 1.5 instructions
// for a key and dimension, where P as code pairs took four for a key and row; and P is one
// number of 11 bits.  P is relative to the maximum of its own tile (so that weak keys next
// to one that takes all the weight keep their bits), every tile's product starts at zero,
// and the accumulators' warps add it to fp32 registers with the weight 2^(m_tile - m).
//
// Block keys (not cached, bf16) form the last step: the keys split into code pairs
// like the rows, the values as they are against P in bf16.
//
// Warp roles: 0 pages and TMA, 1 tensor memory and the products S, 2 the products O; 3 to
// 10 the softmax, two groups of four that take the tiles in turn; 11 to 18 the conversion
// of V and the accumulators, two warps to a quadrant of 32 rows.
//
// Bounds and figures.  16 requests of 8192 keys, 128 rows and dimensions: 81 us, 2,300
// clocks for a tile of 128 rows and keys, where memory would allow 41 us and the products
// 37 (16 a tile, 68 clocks each).  What sets the pace is a chain from tile to tile: the
// product O, the accumulators' warps that read and add it and convert the next V
// meanwhile.  At 128 dimensions there is one O: two S, two P in columns of their own and
// two O would be 640 columns of 512.  (P over the S it came from would leave room for a
// second; not built.)
// 19 x 4096 keys, 64 rows: 45 us, the same chain (24 us of bytes).  One request of 4096
// keys, 64 rows, 12 splits of three tiles: 11.5 us, of which 2 are the launch, 2.5 the
// way to the first scores (lengths -> table -> copies), 3 the merge of the splits.
// Registers matter more than instructions: shared memory leaves no L1, so a spill is a trip
// to L2; 150 bytes of them in the cold path of cut tiles cost 25 us.
#include <math.h>

#include "paged_tc.cuh"

namespace {

using namespace sbd_dev;

constexpr int kControl = 3;
constexpr int kTables = 8 * 1024;            // shared memory outside the operands
constexpr int kRows = 128;                   // packed rows of a CTA
constexpr int kSlots = 8;                    // tiles whose scales are kept

// A in tensor memory.
__device__ __forceinline__ void tc_mma_f16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                              uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tc_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tc_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// fp32 D, A K-major, B MN-major; A and B fp16 or bf16.
__device__ __forceinline__ uint32_t idesc_pv(bool bf16, int M, int N) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | 1u << 16 | (uint32_t)(N >> 3) << 17 | (uint32_t)(M >> 4) << 24;
}
__device__ __forceinline__ float max3_nan(float x, float y, float z) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
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
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
      "mul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
// The values of two codes (the low half of c) times w, in fp16.
__device__ __forceinline__ uint32_t half2_of(uint32_t c, __half2 w) {
  uint32_t x;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(x) : "h"((uint16_t)(c & 0xffffu)));
  const __half2 y = __hmul2(*reinterpret_cast<const __half2*>(&x), w);
  return *reinterpret_cast<const uint32_t*>(&y);
}

template <int D>
struct Shape {
  static constexpr int kSoftWarps = 8, kAccWarps = 8, kWorkWarps = kSoftWarps + kAccWarps;
  static constexpr int kDims = D / 2;                  // of an accumulators' thread
  static constexpr int kThreads = 32 * (kControl + kWorkWarps);
  // Tensor memory: two buffers of S, two of P (two keys a column), then O, in two
  // buffers where they fit.
  static constexpr int kPCol = 2 * kTile, kOCol = kPCol + kTile;
  static constexpr int kOBufs = kOCol + 2 * D <= 512 ? 2 : 1;
  static constexpr int kKV = kTile * D;
  static constexpr int kQ = 2 * kRows * D;
  static constexpr int kV16 = 2 * kKV, kV16Sub = kTile * 128;   // 64 dimensions a sub-tile
  static constexpr int kBlk = 2 * kBlkKeys * D, kBlkSub = kBlkKeys * 128;
  static constexpr int kFixed = 1024 + kQ + 2 * kV16 + 2 * kBlk;
  static constexpr int kLeft = 227 * 1024 - kTables - kFixed;
  // (a tile's scales are read until two tiles behind the last one that left the ring)
  static constexpr int kStages = kLeft / (2 * kKV) < kSlots - 2 ? kLeft / (2 * kKV) : kSlots - 2;
  static constexpr int kSmem = kFixed + kStages * 2 * kKV;
  static constexpr int kPStride = D + 4;
  static_assert(kStages >= 2, "a tile ahead");
  static_assert(kRows * kPStride * 4 <= kQ + 2 * kV16, "the partial rows fit the places of Q and V");
  static_assert((kRows + kMaxSplits) * kPStride * 4 <= kStages * 2 * kKV, "the partial rows fit the ring");
};

template <int D>
__global__ void __launch_bounds__(Shape<D>::kThreads, 1)
paged_rows_kernel(const __grid_constant__ CUtensorMap tmap_k,
                  const __grid_constant__ CUtensorMap tmap_v, const Args a) {
  using C = Shape<D>;
  constexpr int kStages = C::kStages, kDims = C::kDims, kOBufs = C::kOBufs;
  constexpr int kWorkWarps = C::kWorkWarps;

  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t kv_full[kMaxStages], kv_empty[kMaxStages];
  __shared__ __align__(8) uint64_t s_full[2], s_free[2], p_full[2], v_full[2], o_full[2], o_free[2];
  __shared__ __align__(8) uint64_t q_ready, blk_ready, tail_bar, merge_bar;
  __shared__ uint32_t tmem_base_sh;
  __shared__ int b_pick, blk_bad;
  __shared__ PageScales pages;
  __shared__ __align__(16) int order_sh[kMaxOrder];
  __shared__ __align__(16) float bks_sh[kBlkKeys];
  __shared__ float c_sh[kRows];                        // a row's score scale, log2 units
  __shared__ float2 stat_sh[4][kRows];                 // a step's maximum and sum of a row
  __shared__ float lse_sh[kRows + kMaxSplits];         // of the rows merged here, a row's splits together

  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_s = sbase, v16_s = q_s + C::kQ;
  const uint32_t bk_s = v16_s + 2 * C::kV16, bv_s = bk_s + C::kBlk;
  const uint32_t ring = bv_s + C::kBlk;
  auto k_tile = [&](int j) { return ring + (uint32_t)(j % kStages) * 2 * C::kKV; };
  auto v_tile = [&](int j) { return k_tile(j) + C::kKV; };

  float* const local = reinterpret_cast<float*>(smem_raw + (q_s - smem_u32(smem_raw)));   // partial rows, at the end

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = blockIdx.x, hkv = whole_part(blockIdx.y, a.inv_chunks), chunk = blockIdx.y - hkv * a.chunks;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&kv_full[s], 1);
      mbar_init(&kv_empty[s], 1 + C::kAccWarps);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], 2);              // the product, and its issuer's view of the scales
      mbar_init(&s_free[i], 4);
      mbar_init(&p_full[i], 4);
      mbar_init(&v_full[i], C::kAccWarps);
      mbar_init(&o_free[i], C::kAccWarps);
      mbar_init(&o_full[i], 2);              // the product, and its issuer's view of the statistics
    }
    mbar_init(&q_ready, kWorkWarps);
    mbar_init(&blk_ready, kWorkWarps);
    mbar_init(&tail_bar, 1);
    mbar_init(&merge_bar, 1);
    blk_bad = 0;
    fence_mbar_init();
    if (a.splits > 1) mbar_arrive_expect_tx(&merge_bar, merge_bytes<D>(min(kRows, a.M - chunk * kRows), split, a.splits));
  }
  __syncthreads();
  // What the previous grid may still write is read from here on.
  grid_dependency_wait();
  const int cap = a.max_pages << a.page_log2;
  const int b = a.order ? longest_first(a.lens, a.B, cap, blockIdx.z, order_sh, &b_pick) : (int)blockIdx.z;
  int len = a.lens[b];
  if (len < 0 || len > cap) {
    if (threadIdx.x == 0 && split == 0 && blockIdx.y == 0) record_error(a.err, SBD_DEVERR_CACHE_LEN);
    len = len < 0 ? 0 : cap;
  }
  const int n_tiles = (int)(((long long)len + kTile - 1) / kTile) + 1;
  const int t_begin = (int)((uint32_t)split * n_tiles / a.splits);
  const int t_end = (int)((uint32_t)(split + 1) * n_tiles / a.splits);
  const bool has_block = t_end == n_tiles && t_end > t_begin;
  // This CTA's cache tiles, a step each, and the block's keys as a last step.
  const int nc = t_end - t_begin - (has_block ? 1 : 0);
  const int n = nc + (has_block ? 1 : 0);
  auto keys_of = [&](int j) { return max(0, min(kTile, j < nc ? len - (t_begin + j) * kTile : 0)); };

  if (warp == 0) {
    // ------------------------------------------------ pages and TMA
    if (lane == 0) {
      tma_prefetch_desc(&tmap_k);
      tma_prefetch_desc(&tmap_v);
    }
    load_tiles<D, kStages, kSlots, 1>(tmap_k, tmap_v, a, b, hkv, len, t_begin, nc, ring, pages, kv_full, kv_empty, &tail_bar);
  } else if (warp == 1) {
    // ------------------------------------------------ S = Q K^T
    tc_alloc(&tmem_base_sh, 512);
    __syncwarp();
    if (n == 0) grid_dependents_launch();              // (nothing else here tells of the allocation)
    const uint32_t tmem = *(volatile uint32_t*)&tmem_base_sh;
    const bool leader = elect_one();
    bool ok = n > 0 && mbar_wait(&q_ready, 0, a.err);
    const uint64_t qd = desc<D>(q_s);
    constexpr int kLo = kRows * D / 16;                // from hi to lo codes
    for (int i = 0; i < n && ok; ++i) {
      const uint32_t d = tmem + (uint32_t)((i & 1) * kTile);
      ok = mbar_wait(&s_free[i & 1], ((i >> 1) & 1) ^ 1, a.err);
      if (has_block && i == n - 1) {
        ok = ok && mbar_wait(&blk_ready, 0, a.err);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t id = idesc_f8(kRows, kBlkKeys, false);
        const uint64_t kd = desc<D>(bk_s);
        if (leader) {                                  // the keys' hi codes, then their lo codes
#pragma unroll 1
          for (int h = 0; h < 4; ++h)
#pragma unroll 1
            for (int kk = 0; kk < D / 32; ++kk)
              tc_mma_f8(d, qd + ((h & 1) * kLo + 2 * kk), kd + ((h >> 1) * kBlkKeys * D / 16 + 2 * kk), id, h > 0 || kk > 0);
        }
      } else {
        ok = ok && mbar_wait(&kv_full[i % kStages], (i / kStages) & 1, a.err);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t id = idesc_f8(kRows, kTile, false);
        const uint64_t kd = desc<D>(k_tile(i));
        if (leader) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk)
              tc_mma_f8(d, qd + (h * kLo + 2 * kk), kd + 2 * kk, id, h > 0 || kk > 0);
          tc_commit(&kv_empty[i % kStages]);
        }
      }
      if (leader) {
        tc_commit(&s_full[i & 1]);
        mbar_arrive(&s_full[i & 1]);
      }
      __syncwarp();
    }
  } else if (warp == 2) {
    // ------------------------------------------------ O = P V
    const bool leader = elect_one();
    bool ok = true;
    for (int i = 0; i < n && ok; ++i) {
      const bool blk = has_block && i == n - 1;
      const int ob = i % kOBufs;
      ok = mbar_wait(&o_free[ob], (i / kOBufs & 1) ^ 1, a.err) && mbar_wait(&p_full[i & 1], (i >> 1) & 1, a.err) &&
           (blk || mbar_wait(&v_full[i & 1], (i >> 1) & 1, a.err));
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      const uint32_t tmem = *(volatile uint32_t*)&tmem_base_sh;
      const uint32_t o = tmem + C::kOCol + (uint32_t)(ob * D), p = tmem + C::kPCol + (uint32_t)((i & 1) * (kTile / 2));
      const uint64_t vd = blk ? desc<128>(bv_s, C::kBlkSub) : desc<128>(v16_s + (uint32_t)(i & 1) * C::kV16, C::kV16Sub);
      const int steps = blk ? kBlkKeys / 16 : (keys_of(i) + 31) / 32 * 2;
      const uint32_t id = idesc_pv(blk, kRows, D);
      if (leader) {
#pragma unroll
        for (int kk = 0; kk < kTile / 16; ++kk)
          if (kk < steps) tc_mma_f16_ta(o, p + 8 * kk, vd + kk * 128, id, kk > 0);
        tc_commit(&o_full[i & 1]);
        mbar_arrive(&o_full[i & 1]);
      }
      __syncwarp();
    }
    // A kernel that takes tensor memory before it waits for this grid may follow, and what it
    // holds it keeps until this grid is done: it starts only where this CTA has its own, as
    // the products show (a CTA without any leaves it to warp 1, one that gave up to its end).
    // (The accumulators' warps have no register to spare for the condition.)
    if (n > 0 && ok) grid_dependents_launch();
  } else {
    const int sw = warp - kControl, quad = warp & 3;
    const int r = quad * 32 + lane, row = chunk * kRows + r;   // lane of tensor memory, packed row
    const int at = sw * 32 + lane;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    // The chunk's rows become code pairs, then the block's keys; the block's values stay
    // as they are.  All loads first, and one loop for rows and keys: its code comes
    // from L2 once (a copy of its own for the keys took 2,700 clocks of one user's
    // 25,000).  What lies behind the last row is left as it is: rows of the products
    // that nothing reads.
    constexpr int kTurn = 32 * kWorkWarps / (D / 16);  // rows of a turn
    constexpr int kQTurns = kRows / kTurn;
    static_assert(kQTurns * kTurn == kRows && kBlkKeys <= kTurn, "rows in whole turns, keys in one");
    const int c = at % (D / 16), r0 = at / (D / 16);
    const int q_turns = min(kQTurns, (a.M - chunk * kRows + kTurn - 1) / kTurn);
    Piece<D> piece[kQTurns + 1], value;
    const bool key_here = has_block && r0 < a.k;
    const size_t key_off = (((size_t)b * a.k + r0) * a.Hkv + hkv) * D + 16 * c;
#pragma unroll
    for (int e = 0; e < kQTurns; ++e) {
      const int x = chunk * kRows + r0 + e * kTurn, i = a.position(x);
      piece[e].zero();
      if (x < a.M) piece[e].load(a.q + (((size_t)b * a.k + i) * a.Hq + hkv * a.G + x - i * a.G) * D + 16 * c);
    }
    piece[kQTurns].zero(), value.zero();
    if (key_here) {
      piece[kQTurns].load(a.kb + key_off);
      value.load(a.vb + key_off);
    }
#pragma unroll 1
    for (int e = 0; e <= kQTurns; ++e) {
      const bool keys = e == kQTurns;
      if (keys ? has_block && r0 < kBlkKeys : e < q_turns) {   // (whole warps)
        const int to = keys ? r0 : r0 + e * kTurn;
        const float s = piece[0].store(keys ? bk_s : q_s, to, to + (keys ? kBlkKeys : kRows), c);
        if (c == 0) *(keys ? &bks_sh[to] : &c_sh[to]) = keys ? s : s * a.scale_log2;
      }
#pragma unroll
      for (int x = 0; x < kQTurns; ++x) piece[x] = piece[x + 1];
      if (e == kQTurns - 1) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_ready);
      }
    }
    if (has_block) {
      bool bad = false;
      // Values that are not finite stay out of the product (a row that does not
      // see them would multiply them by 0) and are added at the end.
      auto finite2 = [&](uint32_t w) {
        const bool lo_bad = (w & 0x7f80u) == 0x7f80u, hi_bad = (w & 0x7f800000u) == 0x7f800000u;
        bad |= lo_bad || hi_bad;
        return (lo_bad ? 0u : w & 0xffffu) | (hi_bad ? 0u : w & 0xffff0000u);
      };
      if (r0 < kBlkKeys) {
#pragma unroll 1
        for (int e = 0; e < 2; ++e) {                  // 8 dimensions each
          const uint4 v = value.w[0];
          st_shared_v4(swz<128>(bv_s + (2 * c + e) / 8 * C::kBlkSub, r0, (2 * c + e) % 8),
                       make_uint4(finite2(v.x), finite2(v.y), finite2(v.z), finite2(v.w)));
          value.w[0] = value.w[1];
        }
      }
      if (bad) blk_bad = 1;
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&blk_ready);
    }
    bar_sync(5, 32 * kWorkWarps);                      // c of all rows
    const int pos = a.position(row), vis = pos < a.n_causal ? pos + 1 : a.k;
    const bool rows_here = chunk * kRows + quad * 32 < a.M;   // whole warps without rows only keep step
    bool ok = true;
    if (sw < C::kSoftWarps) {
      // ---------------------------------------------- softmax
      // Each step by itself: what its P is relative to is its own maximum, and the
      // statistics go to the accumulators' warps.
      const float c_row = c_sh[r];
      const int group = sw / 4;
      for (int i = group; i < n; i += 2) {
        const bool blk = has_block && i == n - 1;
        const int st = i % kSlots, valid = !rows_here ? 0 : blk ? a.k : keys_of(i);   // (uniform over the warp)
        if (!mbar_wait(&s_full[group], (i >> 1) & 1, a.err)) ok = false;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t tmem = *(volatile uint32_t*)&tmem_base_sh + lane_addr;
        const uint32_t sa = tmem + (uint32_t)(group * kTile), pa = tmem + C::kPCol + (uint32_t)(group * (kTile / 2));
        // 16 keys are a piece, which lies in one page.  Pieces are read twice, for the
        // maximum and for the probabilities, in pairs a pair ahead; one by one where the
        // length or the row's view of the block may cut them.
        auto score_scale = [&](int c) {                // > 0: masked scores stay -inf
          return max_nan(c_row * (blk ? 1.f : pages.ks[st][16 * c >> a.page_log2]), 1.17549435e-38f);
        };
        auto cut_scores = [&](int c, float (&z)[16]) {
          uint32_t x[16];
          tc_ld16(sa + 16 * c, x);
          tc_wait_ld();
          const int seen = (blk ? vis : valid) - 16 * c;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float y = blk ? __uint_as_float(x[e]) * bks_sh[(16 * c + e) & (kBlkKeys - 1)] : __uint_as_float(x[e]);
            z[e] = e < seen ? y : -INFINITY;
          }
        };
        auto top = [](const float (&z)[16]) {          // NaN propagates
          float m = max_nan(z[0], z[1]);
#pragma unroll
          for (int e = 2; e < 16; e += 2) m = max3_nan(m, z[e], z[e + 1]);
          return m;
        };
        uint32_t x0[16], x1[16];
        float my = -INFINITY;
        const bool all = !blk && valid == kTile;       // (the case that the time goes to)
        if (all) {
          tc_ld16(sa, x0);
          tc_ld16(sa + 16, x1);
#pragma unroll 2
          for (int c = 0; c < kTile / 16; c += 2) {
            float z[2][16];
            tc_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) z[0][e] = __uint_as_float(x0[e]), z[1][e] = __uint_as_float(x1[e]);
            const int next = (16 * c + 32) % kTile;
            tc_ld16(sa + next, x0);
            tc_ld16(sa + next + 16, x1);
            my = max3_nan(my, top(z[0]) * score_scale(c), top(z[1]) * score_scale(c + 1));
          }
        } else {
#pragma unroll 1
          for (int c = 0; 16 * c < valid; ++c) {
            float z[16];
            cut_scores(c, z);
            my = max_nan(my, top(z) * score_scale(c));
          }
        }
        const float neg = my == -INFINITY ? 0.f : -my;
        // P's place is free once the product before last is done
        if (i >= 2) ok = mbar_wait(&o_full[group], ((i >> 1) & 1) ^ 1, a.err);
        float2 sum = make_float2(0.f, 0.f);
        auto probabilities = [&](int c, bool bf16, const float (&z)[16]) {
          const float cs = score_scale(c);
          const float2 c2 = make_float2(cs, cs), n2 = make_float2(neg, neg);
          uint32_t w[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float2 p = fma2(make_float2(z[2 * e], z[2 * e + 1]), c2, n2);
            p.x = ex2_ftz(p.x), p.y = ex2_ftz(p.y);
            sum = add2(sum, p);
            const __half2 x = __floats2half2_rn(p.x, p.y);
            w[e] = bf16 ? pack_bf16(p.x, p.y) : *reinterpret_cast<const uint32_t*>(&x);
          }
          tc_st8(pa + 8 * c, w);
        };
        if (all) {
#pragma unroll 2
          for (int c = 0; c < kTile / 16; c += 2) {
            float z[2][16];
            tc_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) z[0][e] = __uint_as_float(x0[e]), z[1][e] = __uint_as_float(x1[e]);
            if (c + 2 < kTile / 16) {
              tc_ld16(sa + 16 * c + 32, x0);
              tc_ld16(sa + 16 * c + 48, x1);
            }
            probabilities(c, false, z[0]);
            probabilities(c + 1, false, z[1]);
          }
        } else {
          // as far as the product goes: 32 keys at a time
#pragma unroll 1
          for (int c = 0; c < (valid + 31) / 32 * 2; ++c) {
            float z[16];
            cut_scores(c, z);
            probabilities(c, blk, z);
          }
        }
        tc_wait_st();
        stat_sh[i & 3][r] = make_float2(my, sum.x + sum.y);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&s_free[group]);
          mbar_arrive(&p_full[group]);
        }
      }
    } else {
      // ---------------------------------------------- accumulators
      // A thread keeps its row's maximum and the sum of probabilities against it, and
      // the accumulators of kDims dimensions, against it too.
      const int part = (sw - C::kSoftWarps) / 4;
      float m_ref = -INFINITY, l = 0.f;
      float2 acc[kDims / 2];
#pragma unroll
      for (int e = 0; e < kDims / 2; ++e) acc[e] = make_float2(0.f, 0.f);
      // Of V this thread converts 16 dimensions of the keys v_key, v_key + kKeyStep, ...
      // Eight lanes have four pieces of two keys k and k ^ 5, so that they read and
      // write eight different places of a swizzled row.
      const int ct = (sw - C::kSoftWarps) * 32 + lane;
      constexpr int kC = D / 16, kKeyStep = 32 * C::kAccWarps / kC;
      static_assert(kKeyStep % 8 == 0, "the swizzle repeats");
      const int v_c = (ct & 3) + (ct >> 3) % (kC / 4) * 4;
      const int v_pair = (ct >> 3) / (kC / 4);          // keys 0, 5 / 1, 4 / 2, 7 / 3, 6 of eight
      const int v_key = v_pair / 4 * 8 + (v_pair % 4 ^ ((ct >> 2 & 1) * 5));
      const uint32_t v_src = swz<D>(0, v_key, v_c), v_dst = swz<128>(v_c / 4 * C::kV16Sub, v_key, 2 * v_c % 8);
      for (int s = 0; s <= n; ++s) {
        // V of tile s, a tile ahead of the accumulators: its place is free, since the
        // product before last is done.
        if (s < nc) {
          ok = mbar_wait(&kv_full[s % kStages], (s / kStages) & 1, a.err);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          const uint32_t src = v_tile(s) + v_src, dst = v16_s + (uint32_t)(s & 1) * C::kV16 + v_dst;
#pragma unroll
          for (int e = 0; e < kTile / kKeyStep; ++e) {
            const __half2 w = __float2half2_rn(pages.vw[s % kSlots][(v_key + e * kKeyStep) >> a.page_log2]);
            const uint4 x = ld_shared_v4(src + e * kKeyStep * D);
            st_shared_v4(dst + e * kKeyStep * 128, make_uint4(half2_of(x.x, w), half2_of(x.x >> 16, w), half2_of(x.y, w), half2_of(x.y >> 16, w)));
            st_shared_v4((dst ^ 16) + e * kKeyStep * 128, make_uint4(half2_of(x.z, w), half2_of(x.z >> 16, w), half2_of(x.w, w), half2_of(x.w >> 16, w)));
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&kv_empty[s % kStages]);
            mbar_arrive(&v_full[s & 1]);
          }
        }
        const int i = s - 1;
        if (i < 0) continue;
        if (!mbar_wait(&o_full[i & 1], (i >> 1) & 1, a.err)) ok = false;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t oa = *(volatile uint32_t*)&tmem_base_sh + lane_addr + C::kOCol + (uint32_t)(i % kOBufs * D + part * kDims);
        if (rows_here) {
          const bool blk = has_block && i == n - 1;
          const float2 ms = stat_sh[i & 3][r];
          const float m_new = max_nan(m_ref, ms.x);
          const float keep = m_ref == -INFINITY ? 0.f : ex2_ftz(m_ref - m_new);
          const float g = ms.x == -INFINITY ? 0.f : ex2_ftz(ms.x - m_new);
          l = fmaf(l, keep, ms.y * g);
          const float fp = g * (blk ? 1.f : pages.vref[i % kSlots]);
          const bool moved = __any_sync(0xffffffffu, m_new != m_ref && m_ref != -INFINITY);
          m_ref = m_new;
          const float2 f = make_float2(fp, fp);
          if (moved) {
#pragma unroll
            for (int e = 0; e < kDims / 2; ++e) acc[e] = mul2(acc[e], make_float2(keep, keep));
          }
#pragma unroll
          for (int c = 0; c < kDims; c += 16) {
            uint32_t x[16];
            tc_ld16(oa + c, x);
            tc_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; e += 2)
              acc[(c + e) / 2] = fma2(make_float2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), f, acc[(c + e) / 2]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&o_free[i % kOBufs]);
      }
      if (a.splits > 1) cluster_arrive();
      // ------------------------------------------------ epilogue
      const float inv = m_ref == -INFINITY ? 0.f : __fdividef(1.f, l);
#pragma unroll
      for (int e = 0; e < kDims / 2; ++e) acc[e].x *= inv, acc[e].y *= inv;
      const bool mine = row < a.M;
      const int i = pos;
      if (has_block && blk_bad && mine) {
#pragma unroll 1
        for (int e = 0; e < vis; ++e) {
          const __nv_bfloat16* v = a.vb + (((size_t)b * a.k + e) * a.Hkv + hkv) * D + part * kDims;
#pragma unroll
          for (int d = 0; d < kDims / 2; ++d) {
            const float x = __bfloat162float(v[2 * d]), y = __bfloat162float(v[2 * d + 1]);
            if (!(fabsf(x) < INFINITY)) acc[d].x += x;
            if (!(fabsf(y) < INFINITY)) acc[d].y += y;
          }
        }
      }
      if (a.splits == 1) {
        if (mine) {
          __nv_bfloat16* dst = a.out + (((size_t)b * a.k + i) * a.Hq + hkv * a.G + row - i * a.G) * D + part * kDims;
#pragma unroll
          for (int e = 0; e < kDims / 2; e += 4)
            *reinterpret_cast<uint4*>(dst + 2 * e) =
                make_uint4(pack_bf16(acc[e].x, acc[e].y), pack_bf16(acc[e + 1].x, acc[e + 1].y),
                           pack_bf16(acc[e + 2].x, acc[e + 2].y), pack_bf16(acc[e + 3].x, acc[e + 3].y));
        }
      } else {
        // The places of Q and V are idle, the ring may not be yet in other CTAs.
        float* dst = local + r * C::kPStride + part * kDims;
#pragma unroll
        for (int e = 0; e < kDims / 2; e += 2)
          *reinterpret_cast<float4*>(dst + 2 * e) = make_float4(acc[e].x, acc[e].y, acc[e + 1].x, acc[e + 1].y);
        if (part == 0) c_sh[r] = n > 0 && ok ? m_ref + __log2f(l) : -INFINITY;
      }
    }
  }
  if (a.splits > 1 && warp < kControl + C::kSoftWarps) cluster_arrive();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tc_dealloc(*(volatile uint32_t*)&tmem_base_sh, 512);
  }
  if (a.splits == 1) return;
  // Row r is merged in CTA r mod splits of the cluster: its partial rows go into that
  // one's ring, which is idle there once every CTA has come here.  A warp a row (every
  // lane a row of its own took 4,000 clocks: 16 bytes a packet).
  cluster_wait();
  const int rows = min(kRows, a.M - chunk * kRows);
  const float inv_splits = __fdividef(1.f, (float)a.splits);
#pragma unroll 1
  for (int r = warp; r < rows; r += C::kThreads / 32) {
    const int slot = whole_part(r, inv_splits), to = r - slot * a.splits, at = slot * a.splits + split;
    const uint32_t bar = mapa_shared(smem_u32(&merge_bar), to);
    if (lane < D / 4)
      st_async(mapa_shared(ring + 4u * (at * C::kPStride + 4 * lane), to),
               *reinterpret_cast<const float4*>(local + r * C::kPStride + 4 * lane), bar);
    if (lane == 0) st_async(mapa_shared(smem_u32(&lse_sh[at]), to), c_sh[r], bar);
  }
  merge_in_cluster<D, kRows, C::kThreads / 32>(a, reinterpret_cast<const float*>(smem_raw + (ring - smem_u32(smem_raw))), lse_sh,
                                           b, hkv, chunk, split, &merge_bar);
}

}  // namespace

namespace sbd {

sbd_dev::TcKernel paged_rows_kernel_for(int D) {
  if (D == 128) return {(const void*)paged_rows_kernel<128>, Shape<128>::kSmem, Shape<128>::kThreads};
  return {(const void*)paged_rows_kernel<64>, Shape<64>::kSmem, Shape<64>::kThreads};
}

}  // namespace sbd
