// Attention of drafted tokens over a state on the 5th-generation tensor cores (see tova_tree.cuh for the operation):
// bf16 queries, more than 64 rows of the product (nodes x query heads of a KV head).
//
// A block takes NT tiles of 128 rows and runs down its columns in tiles of 128; row i of a tile is TMEM lane i.  Roles:
//   4 producer warps    K and V tiles into a ring of shared-memory slots in the 128-byte-swizzled layout the tensor cores
//                       read: bf16 states by cp.async, as far ahead as there are slots; 8-bit states through registers,
//                       converted exactly (see tova_tree_mma.cuh); drafts, the last tiles, by plain loads that take out
//                       infinities and NaN.  Columns behind the run are zeros, whatever lies there.
//   1 issuing thread    S = Q K^T (128 x 128, fp32 in TMEM) and O += P V in the order PV_0(i) S_0(i+1) PV_1(i) S_1(i+1):
//                       the tensor cores work on one row tile while the other's soft-max runs (two row tiles in a block,
//                       or two blocks on an SM)
//   4 warps a row tile  one thread per row: logits from TMEM, mask, running maximum, weights as bf16 back over the logits,
//                       where they are the A operand of O += P V.  The sum is taken over the rounded weights, so that the
//                       weights that multiply V add up to one.  The reference maximum moves only when a tile's exceeds it
//                       by more than 2^8: weights up to 256 lose nothing in floating point, and O is almost never rescaled.
// A tile of 128 columns, not 64, because S = Q K^T reads both operands from shared memory: 8 KiB per 64 cycles of math
// (128 x 128 x 16) are what shared memory delivers, 6 KiB per 32 cycles (128 x 64 x 16) are not.  TMEM: 256 columns per row
// tile (S 128, O 128).  One row tile: two blocks per SM; two row tiles (more than 128 rows): one block per SM, and every K
// and V tile feeds both.  Every wait is bounded; one that runs out leaves NaN in the block's rows.
#pragma once

#include "tova_tree_mma.cuh"

namespace tova {

constexpr int TREE_TC_ROWS = 128;      // rows of a tile
constexpr int TREE_TC_COLS = 128;      // columns of a tile
constexpr float TREE_TC_SLACK = 8.f;   // log2 of how far weights may exceed 1 before O is rescaled

template <int D, int FMT, int NT>
struct TreeTcShape {
  static constexpr int SOFT_WARPS = 4 * NT;
  static constexpr int THREADS = 32 * (SOFT_WARPS + 4 + 1);
  static constexpr int Q_BYTES = TREE_TC_ROWS * D * 2;            // per row tile
  static constexpr int SLOT = TREE_TC_COLS * D * 2;
  static constexpr int SLOTS = (NT == 1 ? 2 : 4) * (128 / D);
  // Tiles whose scales are kept.  K of tile i takes the slot of K of tile i - SLOTS/2; S of that tile is complete then, so
  // the soft-max of all tiles before it has passed: their scales may go.
  static constexpr int SCALE_TILES = SLOTS / 2 + 2;
  static constexpr int SCALES = FMT == FORMAT_PLAIN ? 0 : SCALE_TILES * 2 * TREE_TC_COLS * 4;
  static constexpr int SMEM = NT * Q_BYTES + SLOTS * SLOT + SCALES + 1024;
  static constexpr int TMEM_COLS = 256 * NT;
  static constexpr int NODES = NT == 1 ? TREE_TC_ROWS : TREE_MAX_NODES;   // one row tile: M <= 128, so N <= 128
  static constexpr int WORDS = NODES / 32;
  // after the last contraction Q and the ring hold the rows of O on their way out
  static_assert(NT * TREE_TC_ROWS * D * 4 <= NT * Q_BYTES + SLOTS * SLOT, "O fits");
};

// The mbarrier receives this thread's arrival (counted in its initial count) once its cp.async so far have landed.
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
}

template <int D, int FMT, int NT>
__global__ void __launch_bounds__(TreeTcShape<D, FMT, NT>::THREADS, NT == 1 ? 2 : 1)
    tova_tree_tc_kernel(const __grid_constant__ TreeParams p) {
  using S = TreeTcShape<D, FMT, NT>;
  constexpr bool PLAIN = FMT == FORMAT_PLAIN;
  constexpr int C = TREE_TC_COLS, R = TREE_TC_ROWS;
  constexpr int PRODUCER = S::SOFT_WARPS, ISSUER = S::SOFT_WARPS + 4;      // first warp of each role
  extern __shared__ unsigned char tree_tc_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(tree_tc_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* q_s = smem;                               // per row tile: boxes of [128 rows][128 bytes]
  unsigned char* slot_s = q_s + NT * S::Q_BYTES;           // per slot: boxes of [128 rows][128 bytes]
  float* scale_s = reinterpret_cast<float*>(slot_s + S::SLOTS * S::SLOT);   // [tile % SCALE_TILES][k, v][128]
  __shared__ __align__(8) uint64_t full[S::SLOTS], empty[S::SLOTS], bar_q, bar_s[NT], bar_p[NT], bar_o[NT], bar_sc[S::SCALE_TILES];
  __shared__ uint32_t tmem_base_s;
  __shared__ int odd_s;
  __shared__ int par_s[S::NODES];
  __shared__ __align__(16) uint32_t anc_s[S::NODES][S::WORDS];     // ancestor bits of every node

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.z / p.Hkv, hk = blockIdx.z % p.Hkv;
  const int split = blockIdx.y, row0 = blockIdx.x * (R * NT);
  const int len = tree_len(p, b);
  const bool last = split == p.splits - 1;
  const int c0 = split * p.split_cols;
  const int c1 = last ? len : min(len, c0 + p.split_cols);
  const int n_state = c1 > c0 ? (c1 - c0 + C - 1) / C : 0;
  const int n = n_state + (last ? (p.N + C - 1) / C : 0);  // tiles of this block

  if (tid == 0) {
    for (int i = 0; i < S::SLOTS; ++i) {
      mbar_init(&full[i], 128);
      mbar_init(&empty[i], 1);
    }
    mbar_init(&bar_q, R * NT);
    for (int t = 0; t < NT; ++t) {
      mbar_init(&bar_s[t], 1);
      mbar_init(&bar_p[t], R);
      mbar_init(&bar_o[t], 1);
    }
    for (int i = 0; i < S::SCALE_TILES; ++i) mbar_init(&bar_sc[i], 128);
    mbar_fence_init();
    odd_s = 0;
  }
  if (warp == ISSUER) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base_s)), "r"(S::TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  bool ok = true;
  // Copies are made and consumed in the order K0 V0 K1 V1 ...: position 2 i is K of tile i, 2 i + 1 its V.

  if (warp >= PRODUCER && warp < ISSUER) {
    // ============================== producers ==============================
    const int pt = tid - PRODUCER * 32;
    auto slot_free = [&](int pos) {
      return pos < S::SLOTS || mbar_wait_bounded(&empty[pos % S::SLOTS], (uint32_t)((pos / S::SLOTS - 1) & 1));
    };
    // Where 16-byte chunk ch of row `row` lies in a slot.
    auto place = [&](int row, int ch) { return (ch >> 3) * (C * 128) + row * 128 + (((ch & 7) ^ (row & 7)) << 4); };
    auto draft = [&](int pos) {
      const bool is_k = !(pos & 1);
      unsigned char* dst = slot_s + (pos % S::SLOTS) * S::SLOT;
      const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(is_k ? p.k_new : p.v_new);
      bool odd = false;
#pragma unroll 4
      for (int e = pt; e < C * (D / 8); e += 128) {
        const int row = e / (D / 8), ch = e % (D / 8), j = (pos / 2 - n_state) * C + row;
        uint4 w = make_uint4(0, 0, 0, 0);
        if (j < p.N) {
          w = *reinterpret_cast<const uint4*>(src + (((long long)j * p.B + b) * p.Hkv + hk) * D + ch * 8);
          if (!is_k) odd |= tree_drop_odd(w);
        }
        *reinterpret_cast<uint4*>(dst + place(row, ch)) = w;
      }
      if (odd) odd_s = 1;
      fence_proxy_async_smem();
      mbar_arrive(&full[pos % S::SLOTS]);
    };
    if constexpr (PLAIN) {
      const unsigned char* g[2] = {static_cast<const unsigned char*>(p.K) + (long long)blockIdx.z * p.cap * (2 * D),
                                   static_cast<const unsigned char*>(p.V) + (long long)blockIdx.z * p.cap * (2 * D)};
      constexpr int CH = D / 8, STEP = 128 / CH;           // a thread's chunks: one column, every STEP-th row
      const int row_t = pt / CH, ch_t = pt % CH;
      for (int pos = 0; pos < 2 * n && ok; ++pos) {
        ok = slot_free(pos);
        if (!ok) break;
        if (pos / 2 < n_state) {
          const int j0 = c0 + (pos / 2) * C;
          const uint32_t dst = smem_addr(slot_s + (pos % S::SLOTS) * S::SLOT);
          const unsigned char* src = ((pos & 1) ? g[1] : g[0]) + ch_t * 16;
#pragma unroll
          for (int x = 0; x < C / STEP; ++x) {
            const int row = x * STEP + row_t;
            const bool in = j0 + row < c1;
            cp_async16(dst + place(row, ch_t), src + (long long)(in ? j0 + row : c0) * (2 * D), in ? 16u : 0u);
          }
          cp_async_arrive(&full[pos % S::SLOTS]);
        } else {
          draft(pos);
        }
      }
      cp_async_commit();
      cp_async_wait<0>();
    } else {
      const unsigned char* g[2] = {static_cast<const unsigned char*>(p.K) + (long long)blockIdx.z * p.cap * D,
                                   static_cast<const unsigned char*>(p.V) + (long long)blockIdx.z * p.cap * D};
      constexpr int CH = D / 16, STEP = 128 / CH, PER = C / STEP;
      const int row_t = pt / CH, ch_t = pt % CH;
      uint4 raw[PER];                  // this thread's chunks of the position that comes next
      auto fetch = [&](int pos) {
        const int j0 = c0 + (pos / 2) * C;
        const unsigned char* src = ((pos & 1) ? g[1] : g[0]) + ch_t * 16;
#pragma unroll
        for (int x = 0; x < PER; ++x) {
          const int j = j0 + x * STEP + row_t;
          raw[x] = pos / 2 < n_state && j < c1 ? *reinterpret_cast<const uint4*>(src + (long long)j * D) : make_uint4(0, 0, 0, 0);
        }
      };
      // Two scales a thread and tile, fetched a tile early and stored with the tile's K.
      float next_k, next_v;
      auto fetch_scales = [&](int tile) {
        const int j = c0 + tile * C + pt;
        const bool in = j < c1;
        next_k = tile < n_state ? (in ? p.k_scale[(long long)blockIdx.z * p.cap + j] : 0.f) : 1.f;
        next_v = tile < n_state ? (in ? p.v_scale[(long long)blockIdx.z * p.cap + j] : 0.f) : 1.f;
      };
      fetch(0);
      fetch_scales(0);
      for (int pos = 0; pos < 2 * n; ++pos) {
        const int tile = pos / 2;
        ok = slot_free(pos);
        if (!ok) break;
        if (!(pos & 1)) {
          float* sc = scale_s + (tile % S::SCALE_TILES) * 2 * C;
          sc[pt] = next_k;
          sc[C + pt] = next_v;
          mbar_arrive(&bar_sc[tile % S::SCALE_TILES]);
          fetch_scales(tile + 1);
        }
        if (tile >= n_state) {
          draft(pos);
          continue;
        }
        unsigned char* dst = slot_s + (pos % S::SLOTS) * S::SLOT;
        uint4 now[PER];
#pragma unroll
        for (int x = 0; x < PER; ++x) now[x] = raw[x];
        fetch(pos + 1);
#pragma unroll
        for (int x = 0; x < PER; ++x) {
          const int row = x * STEP + row_t;
          const uint4 w = now[x];
          *reinterpret_cast<uint4*>(dst + place(row, 2 * ch_t)) =
              make_uint4(tree_codes2<FMT>(w.x, w.x, 0, 1), tree_codes2<FMT>(w.x, w.x, 2, 3),
                         tree_codes2<FMT>(w.y, w.y, 0, 1), tree_codes2<FMT>(w.y, w.y, 2, 3));
          *reinterpret_cast<uint4*>(dst + place(row, 2 * ch_t + 1)) =
              make_uint4(tree_codes2<FMT>(w.z, w.z, 0, 1), tree_codes2<FMT>(w.z, w.z, 2, 3),
                         tree_codes2<FMT>(w.w, w.w, 0, 1), tree_codes2<FMT>(w.w, w.w, 2, 3));
        }
        fence_proxy_async_smem();
        mbar_arrive(&full[pos % S::SLOTS]);
      }
    }
    named_barrier_sync(1, 32 * ISSUER);          // odd_s is final
  } else if (warp == ISSUER) {
    // ============================== issuing thread ==============================
    if (lane == 0 && n > 0) {
      const uint32_t idesc_s = umma_idesc_bf16(R, C, false);
      const uint32_t idesc_o = umma_idesc_bf16(R, D, true);
      const uint32_t q_a = smem_addr(q_s), slot_a = smem_addr(slot_s);
      // cp.async writes through the generic proxy: a tile that has landed is ordered before the tensor cores' reads by a
      // proxy fence here, behind the wait.
      auto landed = [&](int pos) {
        if (!mbar_wait_bounded(&full[pos % S::SLOTS], (uint32_t)((pos / S::SLOTS) & 1))) return false;
        fence_proxy_async_smem();
        return true;
      };
      auto issue_s = [&](int t, int i) {
        const uint32_t k_a = slot_a + ((2 * i) % S::SLOTS) * S::SLOT;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const uint64_t a = umma_desc_sw128(q_a + t * S::Q_BYTES + (ks >> 2) * (R * 128) + (ks & 3) * 32, 16, 1024);
          const uint64_t bd = umma_desc_sw128(k_a + (ks >> 2) * (C * 128) + (ks & 3) * 32, 16, 1024);
          umma_bf16(tmem + 256 * t, a, bd, idesc_s, ks > 0 ? 1u : 0u);
        }
        umma_commit(&bar_s[t]);
        if (t == NT - 1) umma_commit(&empty[(2 * i) % S::SLOTS]);
      };
      ok = mbar_wait_bounded(&bar_q, 0u) && landed(0);
      if (ok) {
        tc_fence_after();
#pragma unroll
        for (int t = 0; t < NT; ++t) issue_s(t, 0);
      }
      for (int i = 0; i < n && ok; ++i) {
        const uint32_t v_a = slot_a + ((2 * i + 1) % S::SLOTS) * S::SLOT;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (t == 0) ok = landed(2 * i + 1);
          ok = ok && mbar_wait_bounded(&bar_p[t], (uint32_t)(i & 1));
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int kk = 0; kk < C / 16; ++kk)
            umma_bf16_a_tmem(tmem + 256 * t + 128, tmem + 256 * t + kk * 8, umma_desc_sw128(v_a + kk * 2048, C * 128, 1024), idesc_o,
                             (i > 0 || kk > 0) ? 1u : 0u);
          if (t == NT - 1) umma_commit(&empty[(2 * i + 1) % S::SLOTS]);
          if (i + 1 < n) {
            if (t == 0) ok = landed(2 * i + 2);
            if (!ok) break;
            tc_fence_after();
            issue_s(t, i + 1);
          } else {
            umma_commit(&bar_o[t]);
          }
        }
      }
    }
  } else {
    // ============================== soft-max: one thread per row ==============================
    const int t = warp >> 2;
    const uint32_t base = tmem + 256 * t + ((uint32_t)((warp & 3) * 32) << 16);
    const int m0 = row0 + t * R + (warp & 3) * 32;       // the warp's first row
    const int node = m0 + lane < p.M ? (m0 + lane) / p.G : -1;
    // Q rows of the row tile, K-major with the 128-byte swizzle; rows past the product are zeros.
    {
      constexpr int CH = D / 8, STEP = 128 / CH;
      const int x = tid & 127, row_t = x / CH, ch = x % CH;
      const uint32_t dst = smem_addr(q_s + t * S::Q_BYTES) + (ch >> 3) * (R * 128);
#pragma unroll 4
      for (int k = 0; k < R / STEP; ++k) {
        const int r = k * STEP + row_t, m = row0 + t * R + r;
        const int nd = min(m, p.M - 1) / p.G, g = min(m, p.M - 1) - nd * p.G;
        cp_async16(dst + r * 128 + (((ch & 7) ^ (r & 7)) << 4),
                   static_cast<const __nv_bfloat16*>(p.q) + (((long long)nd * p.B + b) * p.H + hk * p.G + g) * D + ch * 8, m < p.M ? 16u : 0u);
      }
      cp_async_commit();
    }
    if (last) {
      for (int i = tid; i < p.N; i += 32 * S::SOFT_WARPS) par_s[i] = p.parents ? p.parents[(long long)i * p.B + b] : i - 1;
      named_barrier_sync(2, 32 * S::SOFT_WARPS);
      for (int i = tid; i < p.N; i += 32 * S::SOFT_WARPS) tree_ancestor_bits<S::WORDS>(i, p.parents == nullptr, par_s, anc_s[i]);
    }
    cp_async_wait<0>();
    fence_proxy_async_smem();
    mbar_arrive(&bar_q);
    named_barrier_sync(2, 32 * S::SOFT_WARPS);
    const uint32_t* anc = anc_s[max(node, 0)];
    bool real = false;               // a node's row, not padding's or one behind the product
    if (last && node >= 0) {
#pragma unroll
      for (int k = 0; k < S::WORDS; ++k) real |= anc[k] != 0;
    }
    float m_ref = -INFINITY, l = 0.f;
    const uint64_t scale_2 = pack_f2(p.scale2, p.scale2);
    for (int i = 0; i < n; ++i) {
      const float* sc = scale_s + (i % S::SCALE_TILES) * 2 * C;
      ok = mbar_wait_bounded(&bar_s[t], (uint32_t)(i & 1));
      if constexpr (!PLAIN) ok = ok && mbar_wait_bounded(&bar_sc[i % S::SCALE_TILES], (uint32_t)((i / S::SCALE_TILES) & 1));
      ok = __all_sync(0xffffffffu, ok) != 0;
      if (!ok) break;
      tc_fence_after();
      // A quarter of a row's logits at a time, read once for the maximum and again for the weights: that costs less than 128
      // registers a thread would.
      const int left = i < n_state ? c1 - (c0 + i * C) : C;
      float s[32];
      auto logits = [&](int h) {
        tmem_ld32(base + 32 * h, s);
        if constexpr (!PLAIN) {
#pragma unroll
          for (int c = 0; c < 32; c += 4) {
            const float4 f = *reinterpret_cast<const float4*>(sc + 32 * h + c);
            s[c] *= f.x; s[c + 1] *= f.y; s[c + 2] *= f.z; s[c + 3] *= f.w;
          }
        }
        if (i >= n_state) {
          const int w = 4 * (i - n_state) + h;
          const uint32_t see = real && w < S::WORDS ? anc[w] : 0u;
#pragma unroll
          for (int c = 0; c < 32; ++c) s[c] = ((see >> c) & 1u) ? s[c] : -INFINITY;
        } else if (left < C) {
#pragma unroll
          for (int c = 0; c < 32; ++c) s[c] = 32 * h + c < left ? s[c] : -INFINITY;
        }
      };
      float top = -INFINITY;
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        logits(h);
        float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int c = 4; c < 32; c += 4)
#pragma unroll
          for (int k = 0; k < 4; ++k) mx[k] = fmaxf(mx[k], s[c + k]);
        top = fmaxf(top, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])));
      }
      top *= p.scale2;
      float corr = 1.f;
      if (top > m_ref + TREE_TC_SLACK || (m_ref == -INFINITY && top > -INFINITY)) {
        corr = ex2_approx(m_ref - top);
        m_ref = top;
        l *= corr;
      }
      __syncwarp();
      // O of the tiles so far was summed against the old reference.  (The last of them is complete: S of this tile was
      // issued behind it.)
      if (i > 0 && __any_sync(0xffffffffu, corr != 1.f)) {
#pragma unroll
        for (int c = 0; c < D; c += 32) {
          tmem_ld32(base + 128 + c, s);
#pragma unroll
          for (int k = 0; k < 32; ++k) s[k] *= corr;
          tmem_st32(base + 128 + c, s);
        }
      }
      const float ref = m_ref == -INFINITY ? 0.f : m_ref;
      const uint64_t mneg_2 = pack_f2(-ref, -ref);
      uint64_t sum2[2] = {pack_f2(0.f, 0.f), pack_f2(0.f, 0.f)};
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        logits(h);
        uint32_t w[16];            // packed weights, two bf16 each
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float x0, x1;
          unpack_f2(fma_f2(pack_f2(s[2 * e], s[2 * e + 1]), scale_2, mneg_2), x0, x1);
          const float e0 = ex2_approx(x0), e1 = ex2_approx(x1);
          if constexpr (PLAIN) {
            w[e] = pack_bf16(e0, e1);
            sum2[e & 1] = add_f2(sum2[e & 1], pack_f2(__uint_as_float(w[e] << 16), __uint_as_float(w[e] & 0xffff0000u)));
          } else {
            // (the sum is over the weights as they were before the value scale went in: to divide it out again costs
            //  more than it gives)
            sum2[e & 1] = add_f2(sum2[e & 1], pack_f2(e0, e1));
            const float2 f = *reinterpret_cast<const float2*>(sc + C + 32 * h + 2 * e);
            w[e] = pack_bf16(e0 * f.x, e1 * f.y);
          }
        }
        tmem_st16(base + 16 * h, w);       // over logits that have been read
      }
      float s0, s1;
      unpack_f2(add_f2(sum2[0], sum2[1]), s0, s1);
      l += s0 + s1;
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(&bar_p[t]);
    }
    // Every row tile's last contraction: Q and the ring are then free for O's way out.
    if (ok && n > 0) {
#pragma unroll
      for (int x = 0; x < NT; ++x) ok = ok && mbar_wait_bounded(&bar_o[x], 0u);
      ok = __all_sync(0xffffffffu, ok) != 0;
      tc_fence_after();
    }
    named_barrier_sync(1, 32 * ISSUER);          // odd_s is final; no thread is still copying
    pdl_launch_dependents();
    if (last && !real) l = TREE_PADDING;
    if (!ok) l = __uint_as_float(0x7fc00000u);
    const bool zero = n == 0 || l == TREE_PADDING || l == 0.f;
    const float r = p.splits > 1 ? 1.f : (zero ? 0.f : 1.f / l);
    const long long at0 = ((long long)split * gridDim.z + blockIdx.z) * p.M + m0;
    if (p.splits > 1 && node >= 0) p.part_ml[at0 + lane] = make_float2(m_ref, l);
    constexpr int OCH = D / 4;                   // 16-byte chunks of a row of O, turned with the row: no bank conflicts
    unsigned char* stage = smem + (t * R + (warp & 3) * 32) * (D * 4);
#pragma unroll
    for (int c = 0; c < D; c += 32) {
      float o[32];
      tmem_ld32(base + 128 + c, o);              // (nothing was written there in a block without columns: not used then)
      if (last && odd_s && real) tree_add_odd<S::WORDS, 32>(p, b, hk, anc, D, c, o);
#pragma unroll
      for (int k = 0; k < 32; k += 4)
        *reinterpret_cast<float4*>(stage + lane * (D * 4) + ((((c + k) / 4) ^ (lane & (OCH - 1))) << 4)) =
            zero ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o[k] * r, o[k + 1] * r, o[k + 2] * r, o[k + 3] * r);
      __syncwarp();
    }
    constexpr int AT_ONCE = 32 / OCH;            // rows a warp writes at a time
#pragma unroll 4
    for (int x = 0; x < 32; x += AT_ONCE) {
      const int rr = x + lane / OCH, m = m0 + rr, ch = lane % OCH;
      if (m >= p.M) break;
      const float4 v = *reinterpret_cast<const float4*>(stage + rr * (D * 4) + ((ch ^ (rr & (OCH - 1))) << 4));
      if (p.splits == 1) {
        const int nd = m / p.G, g = m - nd * p.G;
        tree_store4<__nv_bfloat16>(static_cast<__nv_bfloat16*>(p.out) + (((long long)nd * p.B + b) * p.H + hk * p.G + g) * D + ch * 4,
                                   v.x, v.y, v.z, v.w);
      } else {
        *reinterpret_cast<float4*>(p.part_acc + (at0 + rr) * D + ch * 4) = v;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == ISSUER)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::TMEM_COLS) : "memory");
}

}  // namespace tova
