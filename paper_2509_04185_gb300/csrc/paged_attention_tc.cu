// Block attention over the paged 8-bit cache on the tcgen05 tensor cores, for
// bf16 activations with up to 32 packed rows of a KV head (r = i*G + g: block
// position i, query head g of the group); and the plan and launch of all of them.
//
// The codes are what the tensor cores read (kind::f8f6f4): no conversion of the
// cache anywhere.  Activations carry 8 significant bits and a code 4, so every
// activation enters as a pair of codes, x / s = hi + lo: the rounding of x / s to
// e4m3 and the rounding of what that leaves, s a power of two that brings the
// row's largest element to 224 .. 448.  Keys are the M side of both products:
//
//   S[key, (hi|lo) row]  = K Q^T      A = K tile (128 keys, K-major),
//                                     B = the rows' hi codes, then their lo codes
//   O[dim, (hi|lo) row] += V^T P^T    A = V tile (MN-major), B = P (MN-major)
//
// so that N follows the rows of the call (R = 16 or 32 a CTA, 8 of 16 computed on for up
// to 8) and a thread of the softmax owns one key: its page's scales are scalars of the thread, masks a
// comparison, a row's maximum and sum one redux a warp.  Above 32 rows those
// reductions cost more than the tile's loads, and rows are on the lanes
// (paged_attention_rows.cu): at 64 rows over 19 x 4096 keys, 128 dimensions, 45 us
// instead of the 50.4 that this kernel took, at 128 rows over 16 x 8192 81 instead of 177.
//
// Tiles go in steps of two (256 keys): what a step costs by row and not by key --
// redux, the row's scale and maximum from shared memory, the accumulators.
//
// P.  Probabilities span more octaves than two codes: next to a key that takes all
// the weight, a thousand weak ones would vanish.  So P is relative to the maximum
// of its own step (times the value scale over the step's largest, and 2^8), every
// step's product starts at zero, and the softmax warps add the product of the step
// before to fp32 accumulators in registers (8 rows, a dimension a thread), weighted
// 2^(m_step - m).  No accumulator in tensor memory is ever rescaled, and no warp
// waits for a product that has just been asked for.
//
// Block keys (not cached, bf16) form the last step: the keys split into code pairs
// like the rows, two products for S; the values as they are against P in bf16
// (kind::f16), since a row may see a single small value of a key.
//
// Bounds and figures (8 KV heads, 128 dimensions; floor: the cache's bytes at the
// measured copy rate).  One query a request, 4 rows: 4 x 32768 keys 45.5 us, 5.9 TB/s of
// 6.8 on 128 of 152 SMs; 19 x 4096 keys 30 us, 5.3 TB/s, of which the start, before any
// copy is under way, is 4.  Eight queries, 32 rows, 19 x 4096: 34 us, the softmax warps'
// instructions.  One request of 4096 keys in 12 splits: 7.2 us, of which launch, lengths ->
// table -> copies, tensor memory and the merge are 5.
//
// Warp roles: 0 pages and TMA, 1 tensor memory and the products S, 2 the products O (1
// too, where two CTAs of 32 rows share an SM); then the softmax and the accumulators, four
// warps for 8 rows of a step: with 16 rows a warp's instructions were the longer part of
// a step (51 us instead of 45.5 for 4 rows of 16, 31.1 instead of 30.2 for 16).
#include <math.h>

#include "paged_tc.cuh"

namespace {

using namespace sbd_dev;

constexpr int kTables = 8 * 1024;            // shared memory outside the operands
constexpr float kPScale = 256.f;             // P = 2^8 p
constexpr float kLoScale = 32.f;             // lo codes of P hold 2^5 of the rest

template <int D, int R, int kUse, int kCtas>
struct Shape {
  // The rows' hi and lo codes lie side by side along N.  (An MMA of M = 128 takes 53
  // clocks up to N = 64: one after the other into the same columns costs twice.)
  static constexpr int kNS = 2 * R;                    // columns of a tile's S
  static constexpr int kNO = 2 * R;                    // columns of O, bytes of a key's row of P
  // Two buffers of S (of two tiles), or one for each of two CTAs that share an SM.
  static constexpr int kSBufs = 2 / kCtas;
  static constexpr int kOCol = kSBufs * 2 * kNS;
  static constexpr int kTmemCols = kOCol + 2 * kNO <= 128 ? 128 : kOCol + 2 * kNO <= 256 ? 256 : 512;
  static_assert(kCtas * kTmemCols <= 512, "tensor memory holds them");
  // Four softmax warps take 8 rows of a step, of the first kUse (what the others' columns
  // hold reaches no column that is read); 16 where two CTAs of 32 rows share an SM, with
  // one warp less for the products: five warps a scheduler leave 96 registers each (and
  // a dozen more are spilled, 64 bytes at 64 dimensions, 52 at 128).
  static constexpr bool kFew = R == 32 && kCtas == 2;
  static constexpr int kRT = kFew ? 16 : 8;
  static constexpr int kControl = kFew ? 2 : 3;        // warps: pages and TMA, products S, products O
  static constexpr int kParts = kUse / kRT;
  static constexpr int kSoftWarps = 4 * kParts;
  static constexpr int kThreads = 32 * (kControl + kSoftWarps);
  static constexpr int kKV = kTile * D;                // a K or V tile
  static constexpr int kQ = 2 * R * D;
  // P of a tile takes the place of its K, which is dead by then.
  static_assert(kTile * kNO <= kKV, "P fits there");
  static constexpr int kPBlk = kBlkKeys * kNO;         // the block's P
  // The block's keys (hi rows, then lo rows), or its values (bf16, 64 dimensions
  // a sub-tile).
  static constexpr int kBlk = 2 * kBlkKeys * D;
  static constexpr int kBlkSub = kBlkKeys * 128;
  static constexpr int kFixed = 1024 + kQ + kPBlk + 2 * kBlk;
  static constexpr int kLeft = (228 / kCtas - 1) * 1024 - kTables - kFixed;
  static constexpr int kStages = kLeft / (2 * kKV) < kMaxStages ? kLeft / (2 * kKV) : kMaxStages;
  static constexpr int kSmem = kFixed + kStages * 2 * kKV;
  static constexpr int kPStride = D + 4;               // floats of a partial row
  static_assert(kStages >= 4 / kCtas, "two steps of two tiles");
  static_assert(kPBlk % 1024 == 0, "operands begin on 1 KB");
  static_assert((R + kMaxSplits) * kPStride * 4 <= kStages * 2 * kKV, "the partial rows fit the ring");
  static_assert(kBlk + kTile * D <= 2 * kBlk + kStages * 2 * kKV, "reads past the block's keys stay inside");
};

// Four probabilities as code pairs.  The fp16 pattern of p in [0, 1], shifted right
// by 7, is the e4m3 pattern of 2^8 p (the exponents are 8 apart, and so are the
// subnormal steps), so hi, p to 4 bits, is a rounded shift; lo = 2^5 (p - hi), exact in
// fp16, to 4 more.  Together they hold p to 2^-9, and to 2^-23 of the step's largest.
__device__ __forceinline__ void p_codes(__half2 p01, __half2 p23, uint32_t* hi, uint32_t* lo) {
  auto bits = [](__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); };
  auto half2 = [](uint32_t x) { return *reinterpret_cast<const __half2*>(&x); };
  const uint32_t a = bits(p01), b = bits(p23);         // p <= 1: bits 14, 15 and 30, 31 are 0
  *hi = __byte_perm(a + a + 0x00800080u, b + b + 0x00800080u, 0x7531);
  const uint32_t na = ((a + 0x00400040u) & 0xff80ff80u) ^ 0x80008000u;   // -hi
  const uint32_t nb = ((b + 0x00400040u) & 0xff80ff80u) ^ 0x80008000u;
  const __half2 up = __float2half2_rn(kPScale * kLoScale);
  const uint32_t c = bits(__hmul2(__hadd2(p01, half2(na)), up));
  const uint32_t d = bits(__hmul2(__hadd2(p23, half2(nb)), up));
  uint16_t x, y;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(x) : "r"(c));
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(y) : "r"(d));
  *lo = (uint32_t)x | (uint32_t)y << 16;
}

__device__ __forceinline__ void tc_ld(uint32_t taddr, uint32_t (&r)[8]) { tc_ld8(taddr, r); }
__device__ __forceinline__ void tc_ld(uint32_t taddr, uint32_t (&r)[16]) { tc_ld16(taddr, r); }
__device__ __forceinline__ void st_shared_v2(uint32_t addr, const uint32_t (&x)[2]) {
  asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(x[0]), "r"(x[1]) : "memory");
}

template <int D, int R, int kUse, int kCtas>
__global__ void __launch_bounds__(Shape<D, R, kUse, kCtas>::kThreads, kCtas)
paged_tc_kernel(const __grid_constant__ CUtensorMap tmap_k,
                const __grid_constant__ CUtensorMap tmap_v, const Args a) {
  using C = Shape<D, R, kUse, kCtas>;
  constexpr int kSBufs = C::kSBufs, kRT = C::kRT, kControl = C::kControl;
  constexpr int kStages = C::kStages, kNS = C::kNS, kNO = C::kNO;
  constexpr int kParts = C::kParts, kSoftWarps = C::kSoftWarps;
  static_assert(R == 16 || R == 32, "a key's row of P is one swizzle atom");

  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t kv_full[kMaxStages], kv_empty[kMaxStages];
  __shared__ __align__(8) uint64_t s_full[2], s_free[2], p_full[4], o_full[2], o_free[2];
  __shared__ __align__(8) uint64_t q_ready, blk_ready, tail_bar, merge_bar;
  __shared__ uint32_t tmem_base_sh;
  __shared__ int b_pick, blk_bad;
  __shared__ PageScales pages;
  __shared__ __align__(16) int order_sh[kMaxOrder];
  __shared__ float bks_sh[kBlkKeys];
  __shared__ __align__(16) float c_sh[R];              // a row's score scale, log2 units
  __shared__ int vis_sh[R];                            // block keys that it sees
  __shared__ __align__(16) float red_sh[kParts][2][4][kRT];  // maxima of a part's warps, two steps
  __shared__ __align__(16) float sum_sh[kSoftWarps][kRT];    // a warp's sums of probabilities
  __shared__ __align__(16) float mq_sh[kSoftWarps][kRT];     // a warp's copy of the step's maxima, negated
  __shared__ __align__(16) float f_sh[kSoftWarps][2][kRT];   // its rows' weights: of a step's product, of what was before
  __shared__ float lse_sh[R + kMaxSplits];                   // of the rows merged here, a row's splits together

  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_s = sbase, pblk_s = q_s + C::kQ;
  const uint32_t bk_s = pblk_s + C::kPBlk, bv_s = bk_s + C::kBlk;
  const uint32_t ring = bv_s + C::kBlk;
  auto k_tile = [&](int j) { return ring + (uint32_t)(j % kStages) * 2 * C::kKV; };
  auto v_tile = [&](int j) { return k_tile(j) + C::kKV; };

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = blockIdx.x, hkv = whole_part(blockIdx.y, a.inv_chunks), chunk = blockIdx.y - hkv * a.chunks;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&kv_full[s], 1);
      mbar_init(&kv_empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s_full[i], 2);              // the product, and its issuer's view of the scales
      mbar_init(&s_free[i], kSoftWarps);
      mbar_init(&o_full[i], 1);
      mbar_init(&o_free[i], kSoftWarps);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&p_full[i], kSoftWarps);
    mbar_init(&q_ready, kSoftWarps);
    mbar_init(&blk_ready, kSoftWarps);
    mbar_init(&tail_bar, 1);
    mbar_init(&merge_bar, 1);
    blk_bad = 0;
    fence_mbar_init();
    if (a.splits > 1) mbar_arrive_expect_tx(&merge_bar, merge_bytes<D>(min(R, a.M - chunk * R), split, a.splits));
  }
  __syncthreads();
  // What the previous grid may still write is read from here on.  There is no
  // barrier of the block any more before the work begins: tensor memory, the table
  // and the first copies, and the rows are fetched side by side.
  grid_dependency_wait();
  const int cap = a.max_pages << a.page_log2;
  const int b = a.order ? longest_first(a.lens, a.B, cap, blockIdx.z, order_sh, &b_pick) : (int)blockIdx.z;
  int len = a.lens[b];
  if (len < 0 || len > cap) {
    if (threadIdx.x == 0 && split == 0 && blockIdx.y == 0) record_error(a.err, SBD_DEVERR_CACHE_LEN);
    len = len < 0 ? 0 : cap;
  }
  const int n_cache = (int)(((long long)len + kTile - 1) / kTile);
  const int n_tiles = n_cache + 1;
  const int t_begin = (int)((uint32_t)split * n_tiles / a.splits);
  const int t_end = (int)((uint32_t)(split + 1) * n_tiles / a.splits);
  const bool has_block = t_end == n_tiles && t_end > t_begin;
  // This CTA's cache tiles, two a step, and the block's keys as a last step.
  const int nc = t_end - t_begin - (has_block ? 1 : 0);
  const int n = (nc + 1) / 2 + (has_block ? 1 : 0);
  // keys of local cache tile j
  auto keys_of = [&](int j) { return max(0, min(kTile, j < nc ? len - (t_begin + j) * kTile : 0)); };

  // O = V^T P^T of step i, from uniform code of one warp.
  auto output = [&](int i, bool leader) {
    const uint32_t id_pv = idesc_f8(D, kNO, true);
    bool ok = mbar_wait(&o_free[i & 1], ((i >> 1) & 1) ^ 1, a.err) &&
         mbar_wait(&p_full[i & 3], (i >> 2) & 1, a.err);
    ok = __all_sync(0xffffffffu, ok);
    if (!ok) return false;
    tc_fence_after();
    const uint32_t o = *(volatile uint32_t*)&tmem_base_sh + C::kOCol + (uint32_t)((i & 1) * kNO);
    if (has_block && i == n - 1) {
      const uint64_t vd = desc<128>(bv_s, C::kBlkSub), pd = desc<kNO>(pblk_s);
      if (leader) {
#pragma unroll
        for (int kk = 0; kk < kBlkKeys / 16; ++kk)
          tc_mma_bf16(o, vd + kk * 128, pd + kk * kNO, idesc_bf16_mn(D, R), kk > 0);
      }
    } else {
      for (int j = 2 * i; j < min(nc, 2 * i + 2); ++j) {
        const uint64_t vd = desc<D>(v_tile(j)), pd = desc<kNO>(k_tile(j));
        const int steps = (keys_of(j) + 31) / 32;
        if (leader) {
#pragma unroll
          for (int kk = 0; kk < kTile / 32; ++kk)
            if (kk < steps) tc_mma_f8(o, vd + kk * 2 * D, pd + kk * 2 * kNO, id_pv, (j & 1) || kk > 0);
          tc_commit(&kv_empty[j % kStages]);
        }
      }
    }
    if (leader) tc_commit(&o_full[i & 1]);
    __syncwarp();
    return true;
  };

  if (warp == 0) {
    // ------------------------------------------------ pages and TMA
    if (lane == 0) {
      tma_prefetch_desc(&tmap_k);
      tma_prefetch_desc(&tmap_v);
    }
    load_tiles<D, kStages, kStages, 2>(tmap_k, tmap_v, a, b, hkv, len, t_begin, nc, ring, pages, kv_full, kv_empty, &tail_bar);
  } else if (warp == 1) {
    // ------------------------------------------------ S = K Q^T
    // Ahead of the softmax by the second buffer (with one, after the step's product O,
    // whose tiles leave the ring for the next ones).  The whole warp runs the loop
    // (descriptors stay in uniform registers) and one lane issues.
    // Tensor memory is taken only after the previous grid is done, so that no CTA of
    // it can be left waiting for it.  Its address reaches the other warps with the
    // first scores.
    tc_alloc(&tmem_base_sh, C::kTmemCols);
    __syncwarp();
    if (n == 0) grid_dependents_launch();              // (nothing else here tells of the allocation)
    const uint32_t tmem = *(volatile uint32_t*)&tmem_base_sh;
    const bool leader = elect_one();
    const bool ready = n > 0 && mbar_wait(&q_ready, 0, a.err);
    const uint32_t id_s = idesc_f8(kTile, kNS, false);
    const uint64_t qd = desc<D>(q_s);
    auto product = [&](uint32_t d, uint64_t kd, bool add) {
#pragma unroll
      for (int kk = 0; kk < D / 32; ++kk) tc_mma_f8(d, kd + 2 * kk, qd + 2 * kk, id_s, add || kk > 0);
    };
    auto scores = [&](int i) {
      const int buf = i % kSBufs;
      const uint32_t d = tmem + (uint32_t)(buf * 2 * kNS);
      bool ok = mbar_wait(&s_free[buf], (i / kSBufs & 1) ^ 1, a.err);
      if (has_block && i == n - 1) {
        ok = ok && mbar_wait(&blk_ready, 0, a.err);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) return false;
        tc_fence_after();
        if (leader) {                                  // the keys' hi codes, then their lo codes
          product(d, desc<D>(bk_s), false);
          product(d, desc<D>(bk_s + kBlkKeys * D), true);
        }
      } else {
        for (int j = 2 * i; j < min(nc, 2 * i + 2) && ok; ++j) {
          ok = mbar_wait(&kv_full[j % kStages], (j / kStages) & 1, a.err);
          ok = __all_sync(0xffffffffu, ok);
          tc_fence_after();
          if (leader && ok) product(d + (uint32_t)((j & 1) * kNS), desc<D>(k_tile(j)), false);
        }
        if (!ok) return false;
      }
      if (leader) {
        tc_commit(&s_full[buf]);
        mbar_arrive(&s_full[buf]);
      }
      __syncwarp();
      return true;
    };
    if (ready) {
      for (int i = 0; i <= n; ++i) {
        if (C::kFew && i > 0 && !output(i - 1, leader)) break;
        if (i == n || !scores(i)) break;
      }
    }
  } else if (!C::kFew && warp == 2) {
    // ------------------------------------------------ O = V^T P^T
    const bool leader = elect_one();
    for (int i = 0; i < n; ++i)
      if (!output(i, leader)) break;
  } else {
    // ------------------------------------------------ softmax and accumulators
    const int sw = warp - kControl, quad = warp & 3, part = sw / 4;
    const int r0 = part * kRT;                         // its rows: r0 .. r0 + kRT - 1
    uint32_t tmem = 0;
    const int key = quad * 32 + lane;                  // of both tiles
    const int at = sw * 32 + lane;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    constexpr int kRowsTurn = 32 * kSoftWarps / (D / 16);
    {
      const int c = at % (D / 16);
#pragma unroll 1
      for (int r = at / (D / 16); r < R; r += kRowsTurn) {
        const int row = chunk * R + r, i = a.position(row);
        Piece<D> x;
        x.zero();
        if (row < a.M) x.load(a.q + (((size_t)b * a.k + i) * a.Hq + hkv * a.G + row - i * a.G) * D + 16 * c);
        const float s = x.store(q_s, r, R + r, c);
        if (c == 0) {
          c_sh[r] = fmaxf(s * a.scale_log2, 1.17549435e-38f);   // > 0: masked scores stay -inf
          vis_sh[r] = i < a.n_causal ? i + 1 : a.k;
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_ready);
      bar_sync(5, 32 * kSoftWarps);                    // c and vis of all rows
    }
    if (has_block) {
      const int c = at % (D / 16);
      bool bad = false;
#pragma unroll 1
      for (int key = at / (D / 16); key < kBlkKeys; key += kRowsTurn) {
        Piece<D> x, y;
        x.zero(), y.zero();
        if (key < a.k) {
          const size_t off = (((size_t)b * a.k + key) * a.Hkv + hkv) * D + 16 * c;
          x.load(a.kb + off);
          y.load(a.vb + off);
        }
        const float s = x.store(bk_s, key, kBlkKeys + key, c);
        if (c == 0) bks_sh[key] = s;
        // Values that are not finite stay out of the product (a row that does not
        // see them would multiply them by 0) and are added at the end.
        auto finite2 = [&](uint32_t w) {
          const bool lo_bad = (w & 0x7f80u) == 0x7f80u, hi_bad = (w & 0x7f800000u) == 0x7f800000u;
          bad |= lo_bad || hi_bad;
          return (lo_bad ? 0u : w & 0xffffu) | (hi_bad ? 0u : w & 0xffff0000u);
        };
#pragma unroll
        for (int e = 0; e < 2; ++e)                    // 8 dimensions each
          st_shared_v4(swz<128>(bv_s + (2 * c + e) / 8 * C::kBlkSub, key, (2 * c + e) % 8),
                       make_uint4(finite2(y.w[e].x), finite2(y.w[e].y), finite2(y.w[e].z), finite2(y.w[e].w)));
      }
      if (bad) blk_bad = 1;
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&blk_ready);
    }
    // A lane keeps the statistics of one row (32 / kRT lanes a row) over its warp's keys:
    // the running maximum (the same in the four warps of a part) and the sum of
    // probabilities against it.  A thread also keeps the accumulators of its warp's
    // rows for one dimension, against the same maximum.
    const int own = lane % kRT;
    const float c_own = c_sh[r0 + own];
    float m_ref = -INFINITY, l = 0.f;
    float acc[kRT];
#pragma unroll
    for (int r = 0; r < kRT; ++r) acc[r] = 0.f;
    bool ok = true, moved = false;
    // Adds the product of step i, whose weights f_sh holds.
    auto add_product = [&](int i) {
      if (ok && !mbar_wait(&o_full[i & 1], (i >> 1) & 1, a.err)) ok = false;
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) return;
      tc_fence_after();
      const uint32_t oa = tmem + lane_addr + C::kOCol + (uint32_t)((i & 1) * kNO + r0);
      const bool blk = has_block && i == n - 1;
      if (moved) {
#pragma unroll
        for (int r = 0; r < kRT; r += 4) {
          const float4 x = *reinterpret_cast<const float4*>(&f_sh[sw][1][r]);
          acc[r] *= x.x, acc[r + 1] *= x.y, acc[r + 2] *= x.z, acc[r + 3] *= x.w;
        }
      }
#pragma unroll
      for (int c = 0; c < kRT; c += 8) {
        uint32_t h[8], lo[8];
        tc_ld8(oa + c, h);
        tc_ld8(oa + R + c, lo);
        tc_wait_ld();
        if (blk) {                                     // the block's product has no lo columns
#pragma unroll
          for (int e = 0; e < 8; ++e) lo[e] = 0;
        }
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
          const float4 f4 = *reinterpret_cast<const float4*>(&f_sh[sw][0][c + e]);
          const float f[4] = {f4.x, f4.y, f4.z, f4.w};
#pragma unroll
          for (int q = 0; q < 4; ++q)
            acc[c + e + q] = fmaf(fmaf(__uint_as_float(lo[e + q]), 1.f / kLoScale, __uint_as_float(h[e + q])), f[q],
                                  acc[c + e + q]);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&o_free[i & 1]);
    };
    for (int i = 0; i < n; ++i) {
      const int buf = i % kSBufs, phase = i / kSBufs & 1;
      const bool blk = has_block && i == n - 1;
      const int j0 = 2 * i, st0 = j0 % kStages, st1 = (j0 + 1) % kStages;
      const int valid0 = blk ? a.k : keys_of(j0), valid1 = blk ? 0 : keys_of(j0 + 1);
      const bool has0 = quad * 32 < valid0, has1 = quad * 32 < valid1;
      if (ok && !mbar_wait(&s_full[buf], phase, a.err)) ok = false;
      ok = __all_sync(0xffffffffu, ok);
      float z0[kRT], z1[kRT];
      float vw0 = 1.f, vw1 = 1.f, vref = 1.f;
      if (ok) {
        tc_fence_after();
        tmem = *(volatile uint32_t*)&tmem_base_sh;
        if (has0) {
          // (the scales come with the stages, which stay until P is handed in)
          float kf0 = 0.f, kf1 = 0.f;
          if (blk) {
            kf0 = bks_sh[key & (kBlkKeys - 1)];
          } else {
            const int pg = key >> a.page_log2;
            kf0 = pages.ks[st0][pg], vw0 = pages.vw[st0][pg], vref = pages.vref[st0];
            if (has1) kf1 = pages.ks[st1][pg], vw1 = pages.vw[st1][pg];
          }
          // Both tiles' columns are read, also where the second has no keys.
          const uint32_t sa = tmem + lane_addr + (uint32_t)(buf * 2 * kNS + r0);
          uint32_t h[kRT], lo[kRT];
          tc_ld(sa, h);
          tc_ld(sa + R, lo);
          tc_wait_ld();
#pragma unroll
          for (int r = 0; r < kRT; ++r) z0[r] = (__uint_as_float(h[r]) + __uint_as_float(lo[r])) * kf0;
          tc_ld(sa + kNS, h);
          tc_ld(sa + kNS + R, lo);
          tc_wait_ld();
#pragma unroll
          for (int r = 0; r < kRT; ++r) z1[r] = (__uint_as_float(h[r]) + __uint_as_float(lo[r])) * kf1;
          if (blk) {
#pragma unroll
            for (int r = 0; r < kRT; ++r) z0[r] = key < vis_sh[r0 + r] ? z0[r] : -INFINITY;
          } else if (valid0 < quad * 32 + 32) {
#pragma unroll
            for (int r = 0; r < kRT; ++r) z0[r] = key < valid0 ? z0[r] : -INFINITY;
          }
          if (valid1 < quad * 32 + 32) {
#pragma unroll
            for (int r = 0; r < kRT; ++r) z1[r] = key < valid1 ? z1[r] : -INFINITY;
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s_free[buf]);
        // NaN propagates: a row with one has NaN statistics from here on
        if (has0) {
#pragma unroll
          for (int r = 0; r < kRT; r += 4)
            st_shared_v4_if(lane == 0, smem_u32(&red_sh[part][i & 1][quad][r]),
                            redux_max_nan(max_nan(z0[r], z1[r])), redux_max_nan(max_nan(z0[r + 1], z1[r + 1])),
                            redux_max_nan(max_nan(z0[r + 2], z1[r + 2])),
                            redux_max_nan(max_nan(z0[r + 3], z1[r + 3])));
        } else {
          red_sh[part][i & 1][quad][own] = -INFINITY;
        }
      }
      bar_sync(1 + part, 128);
      if (!ok) continue;
      const float(*x)[kRT] = red_sh[part][i & 1];
      const float my = max_nan(max_nan(x[0][own], x[1][own]), max_nan(x[2][own], x[3][own])) * c_own;   // c > 0
      mq_sh[sw][own] = my == -INFINITY ? 0.f : -my;
      __syncwarp();
      if (has0) {
        // p of four rows, and their sums over the warp's keys in fixed point: the
        // pattern of 1 + x counts x in steps of 2^-23, 32 of them stay below 2^28
        // (modulo the patterns of 1).
        auto probs = [&](int r, float (&p)[4], float (&q)[4]) {
          const float4 c4 = *reinterpret_cast<const float4*>(&c_sh[r0 + r]);
          const float4 m4 = *reinterpret_cast<const float4*>(&mq_sh[sw][r]);
          const float cc[4] = {c4.x, c4.y, c4.z, c4.w}, mq[4] = {m4.x, m4.y, m4.z, m4.w};
          uint32_t n1[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            p[e] = ex2_ftz(fmaf(z0[r + e], cc[e], mq[e]));
            q[e] = ex2_ftz(fmaf(z1[r + e], cc[e], mq[e]));
            n1[e] = __reduce_add_sync(0xffffffffu, __float_as_uint(fmaf(p[e] + q[e], 0.5f, 1.f)));
          }
          st_shared_v4_if(lane == 0, smem_u32(&sum_sh[sw][r]), __uint_as_float(n1[0]),
                          __uint_as_float(n1[1]), __uint_as_float(n1[2]), __uint_as_float(n1[3]));
        };
        if (!blk) {
          const __half2 w0 = __float2half2_rn(vw0), w1 = __float2half2_rn(vw1);
          const uint32_t p0 = k_tile(j0) + r0 % 16, p1 = k_tile(j0 + 1) + r0 % 16;
#pragma unroll
          for (int g = 0; g < kRT; g += 8) {           // 8 rows, half a piece
            uint32_t hi0[2], lo0[2], hi1[2], lo1[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float p[4], q[4];
              probs(g + 4 * e, p, q);
              p_codes(__hmul2(__floats2half2_rn(p[0], p[1]), w0), __hmul2(__floats2half2_rn(p[2], p[3]), w0), &hi0[e], &lo0[e]);
              p_codes(__hmul2(__floats2half2_rn(q[0], q[1]), w1), __hmul2(__floats2half2_rn(q[2], q[3]), w1), &hi1[e], &lo1[e]);
            }
            st_shared_v2(swz<kNO>(p0, key, r0 / 16) + g, hi0);
            st_shared_v2(swz<kNO>(p0, key, (R + r0) / 16) + g, lo0);
            if (has1) {
              st_shared_v2(swz<kNO>(p1, key, r0 / 16) + g, hi1);
              st_shared_v2(swz<kNO>(p1, key, (R + r0) / 16) + g, lo1);
            }
          }
        } else {
#pragma unroll
          for (int r = 0; r < kRT; r += 8) {
            float p[4], q[4], zero[4];
            probs(r, p, zero);
            probs(r + 4, q, zero);
            st_shared_v4(swz<kNO>(pblk_s, key, (r0 + r) / 8),
                         make_uint4(pack_bf16(p[0] * kPScale, p[1] * kPScale), pack_bf16(p[2] * kPScale, p[3] * kPScale),
                                    pack_bf16(q[0] * kPScale, q[1] * kPScale), pack_bf16(q[2] * kPScale, q[3] * kPScale)));
          }
        }
        fence_proxy_async_smem();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_full[i & 3]);
      // The step before's product, done by now.  (A warp is past it before it hands
      // in its next P but one, so no phase of p_full is ever two behind.)
      if (i > 0) add_product(i - 1);
      const float m_new = max_nan(m_ref, my);
      const float keep = m_ref == -INFINITY ? 0.f : ex2_ftz(m_ref - m_new);
      const float g = my == -INFINITY ? 0.f : ex2_ftz(my - m_new);
      const uint32_t steps = __float_as_uint(sum_sh[sw][own]) - 32u * 0x3f800000u;
      l = fmaf(l, keep, has0 ? (float)steps * (1.f / (1 << 22)) * g : 0.f);
      __syncwarp();                                    // f of the step before is read
      if (!has0) vref = blk ? 1.f : pages.vref[st0];
      f_sh[sw][0][own] = g * vref * (1.f / kPScale);
      f_sh[sw][1][own] = keep;
      moved = __any_sync(0xffffffffu, m_new != m_ref && m_ref != -INFINITY);
      m_ref = m_new;
      __syncwarp();
    }
    if (n > 0) add_product(n - 1);
    // A kernel that takes tensor memory before it waits for this grid may follow, and what
    // it holds it keeps until this grid is done: it starts only where this CTA has its own,
    // as the products show (a CTA without any leaves it to warp 1, one that gave up to its end).
    if (n > 0 && ok) grid_dependents_launch();
    if (a.splits > 1) cluster_arrive();
    // ------------------------------------------------ epilogue
    sum_sh[sw][own] = l;
    bar_sync(1 + part, 128);
    const float sum = (sum_sh[4 * part][own] + sum_sh[4 * part + 1][own]) +
                      (sum_sh[4 * part + 2][own] + sum_sh[4 * part + 3][own]);
    f_sh[sw][0][own] = m_ref == -INFINITY ? 0.f : __fdividef(1.f, sum);
    __syncwarp();
#pragma unroll
    for (int r = 0; r < kRT; r += 4) {
      const float4 f4 = *reinterpret_cast<const float4*>(&f_sh[sw][0][r]);
      acc[r] *= f4.x, acc[r + 1] *= f4.y, acc[r + 2] *= f4.z, acc[r + 3] *= f4.w;
    }
    // M = 64 leaves 16 dimensions in the first half of every quadrant's lanes
    const int d = D == 128 ? quad * 32 + lane : quad * 16 + (lane & 15);
    const bool has_d = D == 128 || lane < 16;
    const int row = chunk * R + r0;                    // packed rows row .. row + kRT - 1
    if (has_block && blk_bad && has_d) {
#pragma unroll
      for (int r = 0; r < kRT; ++r) {
#pragma unroll 1
        for (int e = 0; e < vis_sh[r0 + r]; ++e) {
          const float v = __bfloat162float(a.vb[(((size_t)b * a.k + e) * a.Hkv + hkv) * D + d]);
          if (!(fabsf(v) < INFINITY)) acc[r] += v;
        }
      }
    }
    if (a.splits == 1) {
      int i = a.position(row), q = row - i * a.G;      // block position, query head of the group
      __nv_bfloat16* dst = a.out + (((size_t)b * a.k + i) * a.Hq + hkv * a.G + q) * D + d;
#pragma unroll
      for (int r = 0; r < kRT; ++r) {
        if (has_d && row + r < a.M) *dst = __float2bfloat16(acc[r]);
        dst += D;
        if (++q == a.G) q = 0, dst += (size_t)(a.Hq - a.G) * D;
      }
    } else {
      // Row r is merged in CTA r mod splits of the cluster: its partial rows go into
      // that one's ring, which is idle there once every CTA has come here.
      const float lse = n > 0 && ok ? m_ref + __log2f(sum) : -INFINITY;
      const float inv_splits = __fdividef(1.f, (float)a.splits);
      cluster_wait();
      if (quad == 0 && lane < kRT && row + own < a.M) {
        const int slot = whole_part(r0 + own, inv_splits), to = r0 + own - slot * a.splits;
        st_async(mapa_shared(smem_u32(&lse_sh[slot * a.splits + split]), to), lse, mapa_shared(smem_u32(&merge_bar), to));
      }
      int slot = whole_part(r0, inv_splits), to = r0 - slot * a.splits;
#pragma unroll
      for (int r = 0; r < kRT; ++r) {
        if (has_d && row + r < a.M)
          st_async(mapa_shared(ring + 4u * ((slot * a.splits + split) * C::kPStride + d), to), n > 0 ? acc[r] : 0.f,
                   mapa_shared(smem_u32(&merge_bar), to));
        if (++to == a.splits) to = 0, ++slot;
      }
    }
  }
  if (a.splits > 1 && warp < kControl) {
    cluster_arrive();
    cluster_wait();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tc_dealloc(*(volatile uint32_t*)&tmem_base_sh, C::kTmemCols);
  }
  if (a.splits == 1) return;
  // ------------------------------------------------ merge in the cluster
  // The CTAs of a cluster are the splits of one (sequence, KV head, chunk); CTA
  // `split` has all splits' normalised rows split, split + splits, ... and their
  // log2-sum-exps in its own shared memory once as many bytes have come as they make, a
  // warp a row.  (Rows read from the other CTAs, all splits of a row requested at once,
  // took 3.5 us of one user's 15: the requests were 250 instructions that run once.
  // Pushed between two barriers of the cluster they took 0.5 us longer.)
  merge_in_cluster<D, R, C::kThreads / 32>(a, reinterpret_cast<const float*>(smem_raw + (ring - smem_u32(smem_raw))), lse_sh, b,
                                           hkv, chunk, split, &merge_bar);
}

template <int D, int R, int kUse, int kCtas>
TcKernel instance() {
  using C = Shape<D, R, kUse, kCtas>;
  return {(const void*)paged_tc_kernel<D, R, kUse, kCtas>, C::kSmem, C::kThreads};
}
template <int D>
TcKernel kernel_of(int M, int ctas) {
  if (M > 16) return ctas == 1 ? instance<D, 32, 32, 1>() : instance<D, 32, 32, 2>();
  if (M > 8) return ctas == 1 ? instance<D, 16, 16, 1>() : instance<D, 16, 16, 2>();
  return ctas == 1 ? instance<D, 16, 8, 1>() : instance<D, 16, 8, 2>();
}
TcKernel kernel_for(int D, int M, int ctas) {
  if (M > 32) return sbd::paged_rows_kernel_for(D);
  return D == 128 ? kernel_of<128>(M, ctas) : kernel_of<64>(M, ctas);
}

}  // namespace

namespace sbd {

void paged_tc_plan(AttnQ8Plan* p, int num_splits) {
  // Up to 32 rows keys are on the lanes, above them rows, 128 a CTA (less than 128 leaves
  // lanes idle, and is faster all the same: see the head of this file).
  p->rows = p->M <= 16 ? 16 : p->M <= 32 ? 32 : 128;
  p->chunks = (p->M + p->rows - 1) / p->rows;
  const long long jobs = (long long)p->B * p->Hkv * p->chunks, sms = num_sms();
  const long long tiles = ((long long)p->max_pages * p->P + kTile - 1) / kTile + 1;
  // Splits.  The host knows the capacity and not the lengths, so it splits while one wave
  // holds all CTAs, and never into a second: 16 requests of 4096 keys on 128 CTAs take
  // 29 us whole and 38 in halves, of 100 to 8000 keys 48 whole and 36 in halves, of 200
  // to 600 keys in a cache for many more 10 and 18.
  const auto fill = [&](long long slots) {
    const long long most = jobs > 0 ? slots / jobs : 1;
    return (int)(most > kMaxSplits ? kMaxSplits : most > tiles ? tiles : most);
  };
  int s = num_splits > 0 ? num_splits : fill(sms);
  // Up to 32 rows two CTAs may share an SM, with half of the ring each.  More CTAs than
  // a wave: the start of one hides behind the other (64 requests, one query each, 500
  // keys: 33 -> 21 us; eight queries, 40 -> 31).  At 128 dimensions the ring is short for
  // that, so only with a capacity of 1024 keys, or up to 16 rows from three waves on (64
  // requests of 0 .. 4000 keys 68 -> 60 us, of 4000 118 -> 124, 32 rows 73 -> 84; 26 of 0 ..
  // 4000 29 -> 51); at 64 dimensions always (32 rows: 64 requests of 4000 keys 126 -> 115
  // us, 32 of 1000 26 -> 21, of 0 .. 2000 25 -> 27).
  p->ctas = 1;
  if (p->rows <= 32 && jobs * (s < 1 ? 1 : s) > sms && (p->D == 64 || tiles <= 9 || (p->rows == 16 && jobs > 3 * sms)))
    p->ctas = 2;
  // At 64 dimensions up to 16 rows also in one wave, where five tiles and more are left to a split (19
  // requests of 4096 keys 28 -> 22 us, 4 of 32000 49 -> 43; 8 of 500 keys 9.1 -> 10.5).
  if (p->rows == 16 && p->D == 64 && num_splits == 0 && fill(2 * sms) > s && tiles >= 5 * fill(2 * sms)) {
    p->ctas = 2;
    s = fill(2 * sms);
  }
  if (s > kMaxSplits) s = kMaxSplits;
  // (Asked for two CTAs an SM, the driver still answers for one.)
  const TcKernel kern = kernel_for(p->D, p->M, p->ctas), one = kernel_for(p->D, p->M, 1);
  for (; s > 1; --s)
    if (cluster_slots(kern.fn, kern.threads, kern.smem, s) > 0 &&
        p->ctas * cluster_slots(one.fn, one.threads, one.smem, s) >= (num_splits > 0 ? 1 : jobs))
      break;
  p->splits = s < 1 ? 1 : s;
}

sbd_status paged_tc_launch(const AttnQ8Plan& p, const AttnQ8Tensors& t, cudaStream_t st) {
  const TcKernel kern = kernel_for(p.D, p.M, p.ctas);
  // Codes as bytes: (D, tokens of a page, page and head); a copy is a page.
  CUtensorMap tk, tv;
  const uint64_t dims[3] = {(uint64_t)p.D, (uint64_t)p.P, (uint64_t)p.n_pages * p.Hkv};
  const uint64_t strides[2] = {(uint64_t)p.D, (uint64_t)p.D * p.P};
  const uint32_t box[3] = {(uint32_t)p.D, (uint32_t)p.P, 1};
  const CUtensorMapSwizzle swizzle = p.D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B;
  sbd_status s = encode_tensor_map(&tk, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, (void*)t.k_cache, dims,
                                   strides, box, swizzle);
  if (s != SBD_OK) return s;
  s = encode_tensor_map(&tv, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, (void*)t.v_cache, dims, strides, box,
                        swizzle);
  if (s != SBD_OK) return s;
  Args a;
  a.q = (const __nv_bfloat16*)t.q;
  a.kb = (const __nv_bfloat16*)t.kb;
  a.vb = (const __nv_bfloat16*)t.vb;
  a.ks = t.k_scale;
  a.vs = t.v_scale;
  a.table = t.table;
  a.lens = t.lens;
  a.out = (__nv_bfloat16*)t.out;
  a.err = device_error_word();
  a.B = p.B;
  a.k = p.k;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.G = p.G;
  a.M = p.M;
  a.max_pages = p.max_pages;
  a.n_pages = p.n_pages;
  a.n_causal = p.n_causal;
  a.splits = p.splits;
  a.chunks = p.chunks;
  a.page_log2 = log2_page(p.P);
  // more CTAs than one wave: the longest sequences first (the pick costs B^2
  // comparisons a CTA, hence the limit)
  a.order = p.B > 1 && p.B <= kMaxOrder &&
            (long long)p.B * p.Hkv * p.chunks * p.splits > num_sms();
  a.scale_log2 = p.scale_log2;
  a.inv_G = 1.f / (float)p.G;
  a.inv_chunks = 1.f / (float)p.chunks;
  s = allow_smem(kern.fn, kern.smem, "cudaFuncSetAttribute(paged_tc_kernel)");
  if (s != SBD_OK) return s;
  void* args[] = {(void*)&tk, (void*)&tv, (void*)&a};
  return launch_pdl(kern.fn, dim3(p.splits, p.Hkv * p.chunks, p.B), dim3(kern.threads), kern.smem, st,
                    args, "paged_tc_kernel launch", p.splits);
}

}  // namespace sbd
