// Causal attention of packed prompts on the 5th-generation tensor cores (see tova_packed.cuh for the operation): bf16.
//
// Work.  An item is two tiles of 128 tokens that share their K and V tiles: two query heads of one KV head and the same tokens
// where a KV head has an even number of query heads (both tiles then see the same columns), else 256 tokens of one head.  One
// resident block per SM walks through the list of items, those with the most columns first, so that the blocks end together; a
// call with fewer items than SMs has no list, and every block finds its own.
//
// Roles in a block.  They meet through mbarriers only and run ahead of one another across items.
//   1 copying thread    Q, then K and V tiles of 128 tokens by tiled TMA into a ring of slots (128-byte swizzle)
//   1 issuing warp      S_t = Q_t K^T (128 x 128, fp32 in TMEM) and O_t += P_t V of the two tiles in turn, PV_0(j) S_0(j+1)
//                       PV_1(j) S_1(j+1): one tile's contractions run while the other's soft-max does
//   4 warps a tile      a thread per row: logits from TMEM, weights as bf16 back over them, where they are the A operand of
//                       O += P V.  The weights' reference is a whole number, 0 at first and hardly ever moved (see tova_tree_tc.cuh): a
//                       tile needs no maximum, only where a row's weights sum to more than 2^32, its first ones to less than
//                       2^-32, or its reference is beyond 2^22, is it done over.  The sum is over the rounded weights, so that the weights that multiply V add up
//                       to one.  At the end the row of O, divided by its sum.
//   2 checking warps    V tiles on the diagonal hold values of later tokens, and of other sequences, under weights of 0; where
//                       one is not finite it becomes 0, and the rows that do see it get it added in the end.
// TMEM: 256 columns a tile (S 128, O 128).  Every wait is bounded; one that runs out leaves NaN in the rows that the block had
// yet to write.
//
// Measured (GPU time, in a captured graph): seven prompts from 8191 tokens down, 32 query over 8 KV heads x 128 (875 GFLOP) 750 us,
// 1160 TFLOP/s, 0.70 of the measured bf16 rate (call after call, at the clocks of the power cap, 884 us); one prompt of 1024 / 2048 /
// 4096 tokens 23 / 42 / 127 us; nine prompts of up to 200 tokens, 8 over 2 heads x 64, 8.6 us.  What bounds the
// first: a round of both tiles takes 3500 cycles, its contractions 2050 of them.  The soft-max of a tile takes 2100 (exponentials
// 1024 of them, TMEM loads and stores 700) and overlaps the other's contractions, not its own.  Not kept: two threads a row (2 %,
// with a protocol for moving a reference that two warps share), an issuing warp for each tile (1.35 times as long: their
// contractions interleave), exponentials by polynomials (1.05 times), all of a row's logits loaded at once (spills, 1.05 times).
#pragma once

#include "tova_packed.cuh"
#include "tova_tree_tc.cuh"

namespace tova {

// Two bf16 values, each added to a fp32 sum.
__device__ __forceinline__ void add_bf16x2(uint32_t u, float& lo, float& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tadd.rn.f32.bf16 %0, a, %0;\n\tadd.rn.f32.bf16 %1, b, %1;\n\t}" : "+f"(lo), "+f"(hi) : "r"(u));
}

constexpr float PACKED_TC_FAR = 4194304.f;      // 2^22: up to here a rounded product of a logit is off by a quarter at most

template <int D>
struct PackedTcShape {
  static constexpr int ROWS = 128, COLS = 128;
  static constexpr int TILE = ROWS * D * 2;                    // bytes of a tile of Q, K or V
  static constexpr int SLOTS = D == 128 ? 5 : 8;
  static constexpr int SOFT_WARPS = 8, COPIER = 8, ISSUER = 9, CHECKER = 10, CHECK_WARPS = 2;      // first warp of each role
  static constexpr int THREADS = 32 * (CHECKER + CHECK_WARPS);
  static constexpr int SMEM = (2 + SLOTS) * TILE + 1024;
};

// Where a block's copies lie: copy x of the present item has place at + x in the order of all of the block's, in a ring of SLOTS.
// The count starts anew a whole number of turns back before it grows large (a long sequence with many heads has more than 2^31).
template <int SLOTS>
struct PackedRing {
  int at = 0;
  __host__ __device__ __forceinline__ int slot(int x) const { return (at + x) % SLOTS; }
  __host__ __device__ __forceinline__ uint32_t phase(int x) const { return (uint32_t)((at + x) / SLOTS) & 1u; }
  __host__ __device__ __forceinline__ bool again(int x) const { return at + x >= SLOTS; }        // another copy was there before
  __host__ __device__ __forceinline__ void pass(int copies) {
    at += copies;
    if (at >= 4 * SLOTS) at = 2 * SLOTS + at % (2 * SLOTS);
  }
};

// An item: tokens and heads of its two tiles, columns in tiles of 128.
struct PackedItem {
  int t0, t1;                  // first token of the sequence, the first behind it
  int q0[2], head[2];          // first token of each tile, counted in the sequence; its query head
  int n[2], most;              // column tiles of each (0: there is no such tile), of both
  int checked;                 // the first column tile with masked columns
};

// The items of a block: every grid-th of the list, up and down in turn, so that no block has the longer one each time.  (The
// list's next entry is fetched an item early.)
struct PackedWalk {
  int round, total, heads, x;
  int4 e;
  __device__ __forceinline__ int place() const { return round * gridDim.x + ((round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x); }
  __device__ __forceinline__ void start(const PackedParams& p, const int4& own) {
    heads = p.pairs ? p.H / 2 : p.H;
    round = 0;
    if (p.list) {
      total = *p.n_list * heads;
      x = blockIdx.x;
      if (x < total) e = __ldg(p.list + x / heads);
    } else {                               // the one item that the block has found itself
      total = own.w ? 1 : 0;
      x = 0;
      e = own;
    }
  }
  __device__ __forceinline__ bool next(const PackedParams& p, PackedItem& it) {
    if (x >= total) return false;
    const int hd = (p.list ? x : blockIdx.x) % heads, tile = e.z;
    it.t0 = e.x;
    it.t1 = e.y;
    if (p.pairs) {
      it.q0[0] = it.q0[1] = tile * 128;
      it.head[0] = 2 * hd;
      it.head[1] = 2 * hd + 1;
      it.n[0] = it.n[1] = it.most = tile + 1;
      it.checked = tile;
    } else {
      it.q0[0] = tile * 256;
      it.q0[1] = it.q0[0] + 128;
      it.head[0] = it.head[1] = hd;
      it.n[0] = 2 * tile + 1;
      it.n[1] = it.q0[1] < e.y - e.x ? 2 * tile + 2 : 0;
      it.most = max(it.n[0], it.n[1]);
      it.checked = 2 * tile;
    }
    ++round;
    x = p.list ? place() : 1;
    if (x < total) e = __ldg(p.list + x / heads);
    return true;
  }
};

template <int D>
__global__ void __launch_bounds__(PackedTcShape<D>::THREADS, 1)
    tova_packed_tc_kernel(const __grid_constant__ PackedParams p, const __grid_constant__ CUtensorMap map_q,
                          const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using S = PackedTcShape<D>;
  constexpr int R = S::ROWS, C = S::COLS;
  extern __shared__ unsigned char packed_tc_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(packed_tc_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char *q_s = smem, *slot_s = smem + 2 * S::TILE;     // boxes of [128 rows][128 bytes]
  // landed and free again: Q of a tile, a slot; S computed, weights written, O complete; diagonal tiles checked, an item's rows
  // written (by items of even and odd number)
  __shared__ __align__(8) uint64_t q_full[2], q_free[2], full[S::SLOTS], empty[S::SLOTS], bar_s[2], bar_p[2], bar_o[2], bar_odd[2], bar_done[2];
  __shared__ uint32_t tmem_base_s;
  __shared__ int odd_s[2][S::CHECK_WARPS];
  __shared__ int4 own_s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int i = 0; i < S::SLOTS; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1 + S::CHECK_WARPS);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(&q_full[t], 1);
      mbar_init(&q_free[t], 1);
      mbar_init(&bar_s[t], 1);
      mbar_init(&bar_p[t], 4);
      mbar_init(&bar_o[t], 1);
      mbar_init(&bar_odd[t], S::CHECK_WARPS);
      mbar_init(&bar_done[t], S::SOFT_WARPS);
    }
    mbar_fence_init();
  }
  if (warp == S::ISSUER) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base_s)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();                                                  // (the list; without one nothing is waited for)
  if (warp == S::CHECKER && !p.list) {
    const int heads = p.pairs ? p.H / 2 : p.H;
    int b, tile, t0 = 0, t1 = 0;
    const bool have = packed_find(p, p.pairs ? 128 : 256, blockIdx.x / heads, lane, b, tile);
    if (have) packed_bounds(p, b, t0, t1);
    if (lane == 0) own_s = make_int4(t0, t1, tile, have);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  const int4 own = own_s;
  bool ok = true;
  PackedWalk walk;
  walk.start(p, own);
  PackedItem it;
  // Copies are made and consumed in the order K0 V0 K1 V1 ...; the ring's positions go on from item to item.
  PackedRing<S::SLOTS> ring;

  if (warp == S::COPIER) {
    // ============================== copying thread ==============================
    if (lane == 0) {
      uint32_t used[2] = {0, 0};                               // Q tiles so far
      auto box = [&](unsigned char* dst, const CUtensorMap* map, int head, int token, uint64_t* bar) {
        mbar_expect_tx(bar, S::TILE);
#pragma unroll
        for (int c = 0; c < D / 64; ++c) tma_load_3d_tile(dst + c * (R * 128), map, c * 64, head, token, bar);
      };
      while (ok && walk.next(p, it)) {
        const int hk = it.head[0] / p.G;
        for (int x = 0; x < 2 * it.most && ok; ++x) {
          const int slot = ring.slot(x);
          if (ring.again(x)) ok = mbar_wait_bounded(&empty[slot], ring.phase(x) ^ 1u);
          if (!ok) break;
          box(slot_s + slot * S::TILE, (x & 1) ? &map_v : &map_k, hk, it.t0 + (x >> 1) * C, &full[slot]);
          if (x == 0) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              if (it.n[t] == 0) continue;
              if (used[t] > 0) ok = ok && mbar_wait_bounded(&q_free[t], (used[t] - 1) & 1);
              if (!ok) break;
              box(q_s + t * S::TILE, &map_q, it.head[t], it.t0 + it.q0[t], &q_full[t]);
              ++used[t];
            }
          }
        }
        ring.pass(2 * it.most);
      }
      // (Where a wait ran out it took two seconds, and whatever was on its way has landed since.)
    }
  } else if (warp == S::ISSUER) {
    // ============================== issuing warp ==============================
    // The whole warp walks through the items, so that descriptors are formed in the warp's own registers; one lane of it
    // issues.  (By a single thread the address arithmetic between the contractions left the tensor cores idle.)
    uint32_t leader;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(leader));
    const uint32_t idesc_s = umma_idesc_bf16(R, C, false), idesc_o = umma_idesc_bf16(R, D, true);
    const uint64_t q_d = umma_desc_sw128(smem_addr(q_s), 16, 1024);
    const uint64_t k_d = umma_desc_sw128(smem_addr(slot_s), 16, 1024), v_d = umma_desc_sw128(smem_addr(slot_s), C * 128, 1024);
    auto at = [](uint64_t d, uint32_t bytes) { return (d & 0xffffffff00000000ull) | (uint32_t)((uint32_t)d + (bytes >> 4)); };
    // Positions in the ring: where K and V of the next columns are, as (slot, phase).
    int k_slot = 0, v_slot = 1;
    uint32_t k_phase = 0, v_phase = 0;
    auto step2 = [](int& slot, uint32_t& phase) {
      slot += 2;
      if (slot >= S::SLOTS) {
        slot -= S::SLOTS;
        phase ^= 1u;
      }
    };
    uint32_t used[2] = {0, 0}, weights[2] = {0, 0};
    for (int item = 0; ok && walk.next(p, it); ++item) {
      // S of tile t over the columns in slot k_slot.
      auto issue_s = [&](int t, bool last) {
        const uint64_t k_t = at(k_d, k_slot * S::TILE);
        if (leader) {
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
            umma_bf16(tmem + 256 * t, at(q_d, t * S::TILE + (ks >> 2) * (R * 128) + (ks & 3) * 32), at(k_t, (ks >> 2) * (C * 128) + (ks & 3) * 32),
                      idesc_s, ks > 0 ? 1u : 0u);
          umma_commit(&bar_s[t]);
          if (last) umma_commit(&q_free[t]);
        }
        __syncwarp();
      };
      ok = warp_wait(&full[k_slot], k_phase);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (it.n[t] == 0) continue;
        ok = ok && warp_wait(&q_full[t], used[t] & 1);
        if (!ok) break;
        ++used[t];
        tc_fence_after();
        issue_s(t, it.n[t] == 1);
      }
      if (!ok) break;
      if (leader) umma_commit(&empty[k_slot]);
      __syncwarp();
      step2(k_slot, k_phase);
      for (int j = 0; j < it.most && ok; ++j) {
        const uint64_t v_t = at(v_d, v_slot * S::TILE);
        ok = warp_wait(&full[v_slot], v_phase);
        if (j + 1 < it.most) ok = ok && warp_wait(&full[k_slot], k_phase);
        if (j == it.checked) ok = ok && warp_wait(&bar_odd[item & 1], (uint32_t)((item >> 1) & 1));
        if (!ok) break;
        const int last = j < it.n[1] ? 1 : 0;                  // the last tile that takes these columns
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (j >= it.n[t]) continue;
          ok = warp_wait(&bar_p[t], weights[t] & 1);
          if (!ok) break;
          ++weights[t];
          tc_fence_after();
          if (leader) {
#pragma unroll
            for (int kk = 0; kk < C / 16; ++kk)
              umma_bf16_a_tmem(tmem + 256 * t + 128, tmem + 256 * t + kk * 8, at(v_t, kk * 2048), idesc_o, (j > 0 || kk > 0) ? 1u : 0u);
            if (j + 1 == it.n[t]) umma_commit(&bar_o[t]);
            if (t == last) umma_commit(&empty[v_slot]);
          }
          __syncwarp();
          if (j + 1 < it.n[t]) issue_s(t, j + 2 == it.n[t]);
        }
        if (!ok) break;
        step2(v_slot, v_phase);
        if (j + 1 < it.most) {             // (the last tile of all to take the next columns has been issued: all have)
          if (leader) umma_commit(&empty[k_slot]);
          __syncwarp();
          step2(k_slot, k_phase);
        }
      }
    }
  } else if (warp >= S::CHECKER) {
    // ============================== checking warps ==============================
    const int w = warp - S::CHECKER;
    for (int item = 0; ok && walk.next(p, it); ++item) {
      if (item >= 2) ok = warp_wait(&bar_done[item & 1], (uint32_t)(((item >> 1) - 1) & 1));     // its flag has been read
      bool odd = false;
      // They follow every copy, and a slot is free again only when they have seen what was in it: a wait by parity must be
      // neither ahead of its barrier by a phase nor behind by two.
      for (int x = 0; x < 2 * it.most && ok; ++x) {
        const int slot = ring.slot(x);
        ok = warp_wait(&full[slot], ring.phase(x));
        if (!ok) break;
        if ((x & 1) && (x >> 1) >= it.checked) {
          unsigned char* v_t = slot_s + slot * S::TILE;
          // Zero times a value is a NaN where it is not finite.
          const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
          __nv_bfloat162 found[2] = {zero, zero};
          auto h = [](uint32_t x) { return *reinterpret_cast<const __nv_bfloat162*>(&x); };
          for (int r = w * 32 + lane; r < C; r += 32 * S::CHECK_WARPS) {
#pragma unroll
            for (int ch = 0; ch < D / 8; ++ch) {
              const uint4 v = *reinterpret_cast<const uint4*>(v_t + (ch >> 3) * (C * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4));
              found[0] = __hfma2(h(v.x), zero, found[0]);
              found[1] = __hfma2(h(v.y), zero, found[1]);
              found[0] = __hfma2(h(v.z), zero, found[0]);
              found[1] = __hfma2(h(v.w), zero, found[1]);
            }
          }
          found[0] = __hadd2(found[0], found[1]);
          if (__low2float(found[0]) != 0.f || __high2float(found[0]) != 0.f) {        // (NaN)
            for (int r = w * 32 + lane; r < C; r += 32 * S::CHECK_WARPS)
#pragma unroll 1
              for (int ch = 0; ch < D / 8; ++ch) {
                uint4* at = reinterpret_cast<uint4*>(v_t + (ch >> 3) * (C * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4));
                uint4 v = *at;
                if (tree_drop_odd(v)) *at = v;
              }
            odd = true;
          }
        }
        warp_arrive(&empty[slot], lane);
      }
      if (odd) fence_proxy_async_smem();
      odd = __any_sync(0xffffffffu, odd) != 0;
      if (lane == 0) odd_s[item & 1][w] = odd;
      warp_arrive(&bar_odd[item & 1], lane);
      ring.pass(2 * it.most);
    }
  } else {
    // ============================== soft-max: a thread per row ==============================
    const int t = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t base = tmem + 256 * t + ((uint32_t)((warp & 3) * 32) << 16);
    const uint64_t scale_2 = pack_f2(p.scale2, p.scale2);
    uint32_t tiles = 0, outs = 0;
    for (int item = 0; walk.next(p, it); ++item) {
      const int n = t ? it.n[1] : it.n[0], q0 = t ? it.q0[1] : it.q0[0], head = t ? it.head[1] : it.head[0];
      float m_ref = 0.f, l = 0.f;
      for (int j = 0; j < n && ok; ++j) {
        ok = warp_wait(&bar_s[t], tiles & 1);
        if (!ok) break;
        ++tiles;
        tc_fence_after();
        const bool masked = j * C >= q0;                       // the diagonal
        uint32_t w[C / 2];                                     // packed weights
        float sum;
        auto mask = [&](int c, uint32_t (&s)[32]) {
          if (masked) {
            const uint32_t see = row >= 32 * c + 31 ? 0xffffffffu : row >= 32 * c ? (2u << (row - 32 * c)) - 1u : 0u;
#pragma unroll
            for (int x = 0; x < 32; ++x) s[x] = ((see >> x) & 1u) ? s[x] : 0xff800000u;
          }
        };
        // `far`: a logit's product with the scale is rounded by itself where the reference, which is a logit's rounded product too,
        // is so large that the two would not meet otherwise.
        auto weights = [&](bool far) {
          const float ref = m_ref == -INFINITY ? 0.f : m_ref;
          const uint64_t neg_2 = pack_f2(-ref, -ref), mul_2 = far ? pack_f2(1.f, 1.f) : scale_2;
          float sums[2] = {0.f, 0.f};
          uint32_t s[2][32];
          tmem_ld32_start(base, s[0]);
#pragma unroll
          for (int c = 0; c < C / 32; ++c) {
            tmem_ld32_wait(s[c & 1]);
            if (c + 1 < C / 32) tmem_ld32_start(base + 32 * (c + 1), s[(c + 1) & 1]);
            mask(c, s[c & 1]);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float x0, x1;
              uint64_t x = pack_f2(__uint_as_float(s[c & 1][2 * e]), __uint_as_float(s[c & 1][2 * e + 1]));
              if (far) x = mul_f2(x, scale_2);
              unpack_f2(fma_f2(x, mul_2, neg_2), x0, x1);
              const uint32_t u = pack_bf16(ex2_approx(x0), ex2_approx(x1));
              add_bf16x2(u, sums[0], sums[1]);
              w[16 * c + e] = u;
            }
          }
          sum = sums[0] + sums[1];
        };
        weights(false);
        // A row's reference is moved where its weights grow too large, or where its first ones are all very small (below 2^-32 of a
        // weight of 1: later ones might lose their smallest).  The warp's other rows form theirs anew against the reference that they
        // have: the same bits, so that a row's result does not depend on what later tokens, or other sequences, ask for.
        const bool ask = !(sum <= TREE_TC_MOST) || fabsf(m_ref) > PACKED_TC_FAR || (j == 0 && sum < 1.f / TREE_TC_MOST);
        if (__any_sync(0xffffffffu, ask)) {
          float top = -INFINITY;
#pragma unroll
          for (int c = 0; c < C / 32; ++c) {
            uint32_t s[32];
            tmem_ld32_start(base + 32 * c, s);
            tmem_ld32_wait(s);
            mask(c, s);
#pragma unroll
            for (int x = 0; x < 32; ++x) top = fmaxf(top, __uint_as_float(s[x]));
          }
          top *= p.scale2;
          // (without a finite logit so far, or with a NaN among them, there may be none to move to)
          const bool beyond = ask && (top > m_ref + 16.f || j == 0 || (m_ref == -INFINITY && top > -INFINITY));
          const float m_new = beyond ? ceilf(top) : m_ref;
          const float corr = beyond && j > 0 ? ex2_approx(m_ref - m_new) : 1.f;       // a power of two, or 0
          m_ref = m_new;
          l *= corr;
          // (S of this tile was issued behind O of the one before, which is complete therefore)
          if (j > 0) {
#pragma unroll
            for (int c = 0; c < D; c += 16) tree_tc_scale16(base + 128 + c, corr);
          }
          weights(fabsf(m_ref) > PACKED_TC_FAR && m_ref != -INFINITY);
        }
        l += sum;
#pragma unroll
        for (int c = 0; c < C / 32; ++c) {
          uint32_t (&wc)[16] = *reinterpret_cast<uint32_t (*)[16]>(&w[16 * c]);
          tmem_st16(base + 16 * c, wc);                        // over logits that have been read
        }
        tmem_st_wait();
        tc_fence_before();
        warp_arrive(&bar_p[t], lane);
      }
      // (Also by warps without a tile: else they could report several items written while the others are still at the first.)
      ok = ok && warp_wait(&bar_odd[item & 1], (uint32_t)((item >> 1) & 1));
      if (n > 0) {
        ok = ok && warp_wait(&bar_o[t], outs & 1);
        if (ok) ++outs;
        tc_fence_after();
        const bool odd = ok && (odd_s[item & 1][0] | odd_s[item & 1][1]) != 0;
        const int tok = it.t0 + q0 + row;
        const bool in = tok < it.t1;
        const float r = 1.f / l;
        const int first = tok - (lane & 3);                    // of the four rows whose pieces this lane stores
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + ((long long)first * p.H + head) * D;
#pragma unroll
        for (int c = 0; c < D; c += 32) {
          float o[32];
          if (ok) {
            tmem_ld32(base + 128 + c, o);
          } else {
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = __uint_as_float(0x7fc00000u);
          }
          if (odd && in) {
#pragma unroll 1
            for (int x = it.t0 + it.checked * C; x <= tok; ++x) {
              const uint4* v = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.v) + x * p.v_stride + (long long)(head / p.G) * D + c);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                float f[8];
                Vec16<__nv_bfloat16>::unpack(__ldg(v + k), f);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  if (!(fabsf(f[e]) < INFINITY)) o[8 * k + e] += f[e];
              }
            }
          }
          // Four lanes transpose their four 16-byte pieces, so that each store writes 64 bytes of a row: eight rows an
          // instruction, not 32.
          uint4 w[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            w[k] = make_uint4(pack_bf16(o[8 * k] * r, o[8 * k + 1] * r), pack_bf16(o[8 * k + 2] * r, o[8 * k + 3] * r),
                              pack_bf16(o[8 * k + 4] * r, o[8 * k + 5] * r), pack_bf16(o[8 * k + 6] * r, o[8 * k + 7] * r));
#pragma unroll
          for (int bit = 1; bit <= 2; bit <<= 1)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              if (k & bit) continue;
              const bool up = (lane & bit) != 0;
              const uint4 send = up ? w[k] : w[k | bit], keep = up ? w[k | bit] : w[k];
              const uint4 got = make_uint4(__shfl_xor_sync(0xffffffffu, send.x, bit), __shfl_xor_sync(0xffffffffu, send.y, bit),
                                           __shfl_xor_sync(0xffffffffu, send.z, bit), __shfl_xor_sync(0xffffffffu, send.w, bit));
              w[k] = up ? got : keep;
              w[k | bit] = up ? keep : got;
            }
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (first + k < it.t1) *reinterpret_cast<uint4*>(out + (long long)k * p.H * D + c + (lane & 3) * 8) = w[k];
          __syncwarp();
        }
        tc_fence_before();                 // O has been read: the next item's first weights are reported behind this
      }
      warp_arrive(&bar_done[item & 1], lane);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == S::ISSUER) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

}  // namespace tova
