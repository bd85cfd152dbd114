// Attention of drafted tokens over a state on the 5th-generation tensor cores (see tova_tree.cuh for the operation):
// bf16 queries, more than 64 rows of the product (nodes x query heads of a KV head).
//
// A block takes NT tiles of 128 rows and runs down its columns in tiles of 64; row i of a tile is TMEM lane i.  Roles:
//   4 producer warps    K and V tiles into a ring of shared-memory slots in the 128-byte-swizzled layout the tensor cores
//                       read: bf16 states by cp.async several slots ahead; 8-bit states through a raw ring (every thread
//                       converts the chunks it copied itself, exactly, see tova_tree_mma.cuh); drafts, the last tiles,
//                       by plain loads that take out infinities and NaN.  Columns behind the run are zeros.
//   1 issuing thread    S = Q K^T (128 x 64, fp32 in TMEM, two buffers a row tile) one tile ahead of O += P V
//   4 warps a row tile  one thread per row: logits from TMEM, mask, running maximum, weights as bf16 back into the logits'
//                       columns as the A operand of O += P V.  The sum is taken over the rounded weights, so that the
//                       weights that multiply V add up to one.  The reference maximum moves only when a tile's exceeds it
//                       by more than 2^8: weights up to 256 lose nothing in floating point, and O is almost never rescaled.
// The roles meet through mbarriers.  One row tile: 256 TMEM columns and 113 KiB, two blocks per SM; two row tiles (more
// than 128 rows): all 512 columns, one block per SM, and every K and V tile feeds both.  A barrier per S buffer and kind:
// a waiter can then never be two phases behind.  Every wait is bounded; one that runs out leaves NaN in the block's rows.
#pragma once

#include "tova_tree_mma.cuh"

namespace tova {

constexpr int TREE_TC_ROWS = 128;      // rows of a tile
constexpr int TREE_TC_COLS = 64;
constexpr int TREE_TC_SCALE_TILES = 8; // tiles whose scales are kept: more than the ring reaches ahead
constexpr float TREE_TC_SLACK = 8.f;   // log2 of how far weights may exceed 1 before O is rescaled

template <int D, int FMT, int NT>
struct TreeTcShape {
  static constexpr int SOFT_WARPS = 4 * NT;
  static constexpr int THREADS = 32 * (SOFT_WARPS + 4 + 1);
  static constexpr int Q_BYTES = TREE_TC_ROWS * D * 2;            // per row tile
  static constexpr int SLOT = TREE_TC_COLS * D * 2;
  static constexpr int RAW = FMT == FORMAT_PLAIN ? 0 : TREE_TC_COLS * D;
  static constexpr int RAW_SLOTS = FMT == FORMAT_PLAIN ? 0 : (NT == 1 ? 3 : 6);
  static constexpr int SCALES = FMT == FORMAT_PLAIN ? 0 : TREE_TC_SCALE_TILES * 2 * TREE_TC_COLS * 4;
  static constexpr int SLOTS = NT == 1 ? (FMT == FORMAT_PLAIN ? 4 : 3) : (FMT == FORMAT_PLAIN ? 9 : 6);
  static constexpr int SMEM = NT * Q_BYTES + SLOTS * SLOT + RAW_SLOTS * RAW + SCALES + 1024;
  static constexpr int TMEM_COLS = 256 * NT;
  static constexpr int NODES = NT == 1 ? TREE_TC_ROWS : TREE_MAX_NODES;   // one row tile: M <= 128, so N <= 128
  static constexpr int WORDS = NODES / 32;
};

template <int D, int FMT, int NT>
__global__ void __launch_bounds__(TreeTcShape<D, FMT, NT>::THREADS, NT == 1 ? 2 : 1)
    tova_tree_tc_kernel(const __grid_constant__ TreeParams p) {
  using S = TreeTcShape<D, FMT, NT>;
  constexpr bool PLAIN = FMT == FORMAT_PLAIN;
  constexpr int C = TREE_TC_COLS, R = TREE_TC_ROWS;
  extern __shared__ unsigned char tree_tc_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(tree_tc_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* q_s = smem;                               // per row tile: boxes of [128 rows][128 bytes]
  unsigned char* slot_s = q_s + NT * S::Q_BYTES;           // per slot: boxes of [64 rows][128 bytes]
  unsigned char* raw_s = slot_s + S::SLOTS * S::SLOT;
  float* scale_s = reinterpret_cast<float*>(raw_s + S::RAW_SLOTS * S::RAW);   // [tile % 8][k, v][64]
  __shared__ __align__(8) uint64_t full[S::SLOTS], empty[S::SLOTS], bar_s[NT][2], bar_p[NT][2], bar_o[NT][2], bar_sc[TREE_TC_SCALE_TILES];
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
    for (int t = 0; t < NT; ++t)
      for (int i = 0; i < 2; ++i) {
        mbar_init(&bar_s[t][i], 1);
        mbar_init(&bar_p[t][i], R);
        mbar_init(&bar_o[t][i], 1);
      }
    for (int i = 0; i < TREE_TC_SCALE_TILES; ++i) mbar_init(&bar_sc[i], 128);
    mbar_fence_init();
    odd_s = 0;
  }
  if (warp == S::SOFT_WARPS + 4) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base_s)), "r"(S::TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (last)
    for (int i = tid; i < p.N; i += S::THREADS) par_s[i] = p.parents ? p.parents[(long long)i * p.B + b] : i - 1;
  // Q rows, K-major with the 128-byte swizzle; rows past the product are zeros.
  for (int e = tid; e < NT * R * (D / 8); e += S::THREADS) {
    const int r = e / (D / 8), ch = e % (D / 8);
    const int m = row0 + r;
    uint4 w = make_uint4(0, 0, 0, 0);
    if (m < p.M) {
      const int nd = m / p.G, g = m - nd * p.G;
      w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + (((long long)nd * p.B + b) * p.H + hk * p.G + g) * D + ch * 8);
    }
    *reinterpret_cast<uint4*>(q_s + (r / R) * S::Q_BYTES + (ch >> 3) * (R * 128) + (r % R) * 128 + (((ch & 7) ^ (r & 7)) << 4)) = w;
  }
  fence_proxy_async_smem();      // the tensor cores read Q through the asynchronous proxy
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;

  // Order in which the tiles are copied and consumed: K0 | K1 V0 | K2 V1 | ... | K(n-1) V(n-2) | V(n-1).
  auto pos_k = [&](int i) { return i == 0 ? 0 : 2 * i - 1; };
  auto pos_v = [&](int i) { return i == n - 1 ? 2 * n - 1 : 2 * i + 2; };
  bool ok = true;

  if (warp >= S::SOFT_WARPS && warp < S::SOFT_WARPS + 4) {
    // ============================== producers ==============================
    const int pt = tid - S::SOFT_WARPS * 32;
    const unsigned char* Kg = static_cast<const unsigned char*>(p.K) + (long long)blockIdx.z * p.cap * (PLAIN ? 2 * D : D);
    const unsigned char* Vg = static_cast<const unsigned char*>(p.V) + (long long)blockIdx.z * p.cap * (PLAIN ? 2 * D : D);
    auto decode = [&](int pos, bool& is_k, int& tile) {
      if (pos == 0) { is_k = true; tile = 0; }
      else if (pos == 2 * n - 1) { is_k = false; tile = n - 1; }
      else { is_k = pos & 1; tile = is_k ? (pos + 1) / 2 : pos / 2 - 1; }
    };
    auto slot_free = [&](int pos) {
      return pos < S::SLOTS || mbar_wait_bounded(&empty[pos % S::SLOTS], (uint32_t)((pos / S::SLOTS - 1) & 1));
    };
    // One scale a thread and tile, fetched a tile early and stored with the tile's K (the slot that K goes to was freed
    // by a tile less than TREE_TC_SCALE_TILES back, whose scales and all before them are used up).
    auto scale_of = [&](int tile) {
      const int j = c0 + tile * C + (pt & 63);
      const float* src = (pt < 64 ? p.k_scale : p.v_scale) + (long long)blockIdx.z * p.cap;
      return tile < n_state ? (j < c1 ? src[j] : 0.f) : 1.f;
    };
    float next_scale = PLAIN ? 0.f : scale_of(0);
    auto scales = [&](int tile) {
      scale_s[((tile % TREE_TC_SCALE_TILES) * 2 + (pt >> 6)) * C + (pt & 63)] = next_scale;
      mbar_arrive(&bar_sc[tile % TREE_TC_SCALE_TILES]);
      next_scale = scale_of(tile + 1);
    };
    auto draft = [&](int pos, bool is_k, int tile) {
      unsigned char* dst = slot_s + (pos % S::SLOTS) * S::SLOT;
      const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(is_k ? p.k_new : p.v_new);
      bool odd = false;
#pragma unroll 4
      for (int e = pt; e < C * (D / 8); e += 128) {
        const int row = e / (D / 8), ch = e % (D / 8), j = (tile - n_state) * C + row;
        uint4 w = make_uint4(0, 0, 0, 0);
        if (j < p.N) {
          w = *reinterpret_cast<const uint4*>(src + (((long long)j * p.B + b) * p.Hkv + hk) * D + ch * 8);
          if (!is_k) odd |= tree_drop_odd(w);
        }
        *reinterpret_cast<uint4*>(dst + (ch >> 3) * (C * 128) + row * 128 + (((ch & 7) ^ (row & 7)) << 4)) = w;
      }
      if (odd) odd_s = 1;
    };
    if constexpr (PLAIN) {
      constexpr int AHEAD = S::SLOTS - 2;
      for (int pos = 0; pos < 2 * n + AHEAD && ok; ++pos) {
        if (pos < 2 * n) {
          bool is_k;
          int tile;
          decode(pos, is_k, tile);
          ok = slot_free(pos);
          if (!ok) break;
          if (tile < n_state) {
            const int j0 = c0 + tile * C;
            const uint32_t dst = smem_addr(slot_s + (pos % S::SLOTS) * S::SLOT);
            const unsigned char* g = is_k ? Kg : Vg;
#pragma unroll
            for (int x = 0; x < C * (D / 8) / 128; ++x) {
              const int e = x * 128 + pt;
              const int row = e / (D / 8), ch = e % (D / 8);
              const bool in = j0 + row < c1;
              cp_async16(dst + (ch >> 3) * (C * 128) + row * 128 + (((ch & 7) ^ (row & 7)) << 4),
                         g + (long long)(in ? j0 + row : c0) * (2 * D) + ch * 16, in ? 16u : 0u);
            }
          } else {
            draft(pos, is_k, tile);
          }
        }
        cp_async_commit();
        if (pos >= AHEAD) {
          cp_async_wait<AHEAD>();
          fence_proxy_async_smem();
          mbar_arrive(&full[(pos - AHEAD) % S::SLOTS]);
        }
      }
      cp_async_wait<0>();
    } else {
      constexpr int AHEAD = S::RAW_SLOTS - 1;
      constexpr int CHR = D / 16;                    // 16-byte chunks of a row of codes
      constexpr int PER = C * CHR / 128;             // chunks of a thread
      auto fetch = [&](int pos) {
        bool is_k;
        int tile;
        decode(pos, is_k, tile);
        if (tile >= n_state) return;
        const int j0 = c0 + tile * C;
        const unsigned char* g = is_k ? Kg : Vg;
        const uint32_t dst = smem_addr(raw_s + (pos % S::RAW_SLOTS) * S::RAW);
#pragma unroll
        for (int x = 0; x < PER; ++x) {
          const int e = x * 128 + pt;
          const int row = e / CHR, ch = e % CHR;
          const bool in = j0 + row < c1;
          cp_async16(dst + e * 16, g + (long long)(in ? j0 + row : c0) * D + ch * 16, in ? 16u : 0u);
        }
      };
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (i < 2 * n) fetch(i);
        cp_async_commit();
      }
      for (int pos = 0; pos < 2 * n; ++pos) {
        bool is_k;
        int tile;
        decode(pos, is_k, tile);
        if (pos + AHEAD < 2 * n) fetch(pos + AHEAD);
        cp_async_commit();
        ok = slot_free(pos);
        if (!ok) break;
        if (is_k) scales(tile);
        if (tile < n_state) {
          cp_async_wait<AHEAD>();
          unsigned char* dst = slot_s + (pos % S::SLOTS) * S::SLOT;
          const unsigned char* src = raw_s + (pos % S::RAW_SLOTS) * S::RAW;
#pragma unroll
          for (int x = 0; x < PER; ++x) {
            const int e = x * 128 + pt;
            const int row = e / CHR, ch = (e % CHR) * 2;
            const uint4 w = *reinterpret_cast<const uint4*>(src + e * 16);
            const uint4 lo = make_uint4(tree_codes2<FMT>(w.x, w.x, 0, 1), tree_codes2<FMT>(w.x, w.x, 2, 3),
                                        tree_codes2<FMT>(w.y, w.y, 0, 1), tree_codes2<FMT>(w.y, w.y, 2, 3));
            const uint4 hi = make_uint4(tree_codes2<FMT>(w.z, w.z, 0, 1), tree_codes2<FMT>(w.z, w.z, 2, 3),
                                        tree_codes2<FMT>(w.w, w.w, 0, 1), tree_codes2<FMT>(w.w, w.w, 2, 3));
            unsigned char* line = dst + (ch >> 3) * (C * 128) + row * 128;
            *reinterpret_cast<uint4*>(line + (((ch & 7) ^ (row & 7)) << 4)) = lo;
            *reinterpret_cast<uint4*>(line + ((((ch & 7) + 1) ^ (row & 7)) << 4)) = hi;
          }
        } else {
          draft(pos, is_k, tile);
        }
        fence_proxy_async_smem();
        mbar_arrive(&full[pos % S::SLOTS]);
      }
      cp_async_wait<0>();
    }
  } else if (warp == S::SOFT_WARPS + 4) {
    // ============================== issuing thread ==============================
    if (lane == 0 && n > 0) {
      const uint32_t idesc_s = umma_idesc_bf16(R, C, false);
      const uint32_t idesc_o = umma_idesc_bf16(R, D, true);
      const uint32_t q_a = smem_addr(q_s), slot_a = smem_addr(slot_s);
      auto issue_s = [&](int i) {
        const int pos = pos_k(i);
        if (!mbar_wait_bounded(&full[pos % S::SLOTS], (uint32_t)((pos / S::SLOTS) & 1))) return false;
        tc_fence_after();
        const uint32_t k_a = slot_a + (pos % S::SLOTS) * S::SLOT;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint64_t a = umma_desc_sw128(q_a + t * S::Q_BYTES + (ks >> 2) * (R * 128) + (ks & 3) * 32, 16, 1024);
            const uint64_t bd = umma_desc_sw128(k_a + (ks >> 2) * (C * 128) + (ks & 3) * 32, 16, 1024);
            umma_bf16(tmem + 256 * t + 64 * (i & 1), a, bd, idesc_s, ks > 0 ? 1u : 0u);
          }
          umma_commit(&bar_s[t][i & 1]);
        }
        umma_commit(&empty[pos % S::SLOTS]);
        return true;
      };
      ok = issue_s(0);
      for (int i = 0; i < n && ok; ++i) {
        if (i + 1 < n && !(ok = issue_s(i + 1))) break;
        const int pos = pos_v(i);
        ok = mbar_wait_bounded(&full[pos % S::SLOTS], (uint32_t)((pos / S::SLOTS) & 1));
        const uint32_t v_a = slot_a + (pos % S::SLOTS) * S::SLOT;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          ok = ok && mbar_wait_bounded(&bar_p[t][i & 1], (uint32_t)((i >> 1) & 1));
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int kk = 0; kk < C / 16; ++kk)
            umma_bf16_a_tmem(tmem + 256 * t + 128, tmem + 256 * t + 64 * (i & 1) + kk * 8, umma_desc_sw128(v_a + kk * 2048, C * 128, 1024),
                             idesc_o, (i > 0 || kk > 0) ? 1u : 0u);
          umma_commit(&bar_o[t][i & 1]);
        }
        if (ok) umma_commit(&empty[pos % S::SLOTS]);
      }
    }
  } else {
    // ============================== soft-max: one thread per row ==============================
    const int t = warp >> 2;
    const uint32_t base = tmem + 256 * t + ((uint32_t)((warp & 3) * 32) << 16);
    const int m = row0 + t * R + (warp & 3) * 32 + lane;
    const int node = m < p.M ? m / p.G : -1;
    if (last) {
      for (int i = tid; i < p.N; i += 32 * S::SOFT_WARPS) tree_ancestor_bits<S::WORDS>(i, p.parents == nullptr, par_s, anc_s[i]);
      named_barrier_sync(2, 32 * S::SOFT_WARPS);
    }
    const uint32_t* anc = anc_s[max(node, 0)];
    bool real = false;               // a node's row, not padding's or one behind the product
    if (last && node >= 0) {
#pragma unroll
      for (int k = 0; k < S::WORDS; ++k) real |= anc[k] != 0;       // (words past N's are zero: bits only go down from i)
    }
    float m_ref = -INFINITY, l = 0.f;
    for (int i = 0; i < n; ++i) {
      const uint32_t tm_s = base + 64 * (i & 1);
      const float* sc = scale_s + (i % TREE_TC_SCALE_TILES) * 2 * C;
      ok = mbar_wait_bounded(&bar_s[t][i & 1], (uint32_t)((i >> 1) & 1));
      if constexpr (!PLAIN) ok = ok && mbar_wait_bounded(&bar_sc[i % TREE_TC_SCALE_TILES], (uint32_t)((i / TREE_TC_SCALE_TILES) & 1));
      ok = __all_sync(0xffffffffu, ok) != 0;
      if (!ok) break;
      tc_fence_after();
      // Half a row's logits at a time; the first half is read again after the maximum is known, which costs less than 32
      // more registers a thread would.
      const int left = i < n_state ? c1 - (c0 + i * C) : C;
      float s[32];
      auto logits = [&](int h) {
        tmem_ld32(tm_s + 32 * h, s);
        if constexpr (!PLAIN) {
#pragma unroll
          for (int c = 0; c < 32; c += 4) {
            const float4 f = *reinterpret_cast<const float4*>(sc + 32 * h + c);
            s[c] *= f.x; s[c + 1] *= f.y; s[c + 2] *= f.z; s[c + 3] *= f.w;
          }
        }
        if (i >= n_state) {
          const int w = 2 * (i - n_state) + h;
          const uint32_t see = real && w < S::WORDS ? anc[w] : 0u;
#pragma unroll
          for (int c = 0; c < 32; ++c) s[c] = ((see >> c) & 1u) ? s[c] : -INFINITY;
        } else if (left < C) {
#pragma unroll
          for (int c = 0; c < 32; ++c) s[c] = 32 * h + c < left ? s[c] : -INFINITY;
        }
      };
      auto top_of = [&]() {
        float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int c = 4; c < 32; c += 4)
#pragma unroll
          for (int k = 0; k < 4; ++k) mx[k] = fmaxf(mx[k], s[c + k]);
        return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
      };
      logits(0);
      float top = top_of();
      logits(1);
      top = fmaxf(top, top_of()) * p.scale2;
      float corr = 1.f;
      if (top > m_ref + TREE_TC_SLACK || (m_ref == -INFINITY && top > -INFINITY)) {
        corr = ex2_approx(m_ref - top);
        m_ref = top;
        l *= corr;
      }
      const float ref = m_ref == -INFINITY ? 0.f : m_ref;
      const uint64_t scale_2 = pack_f2(p.scale2, p.scale2), mneg_2 = pack_f2(-ref, -ref);
      uint64_t sum2[2] = {pack_f2(0.f, 0.f), pack_f2(0.f, 0.f)};
      float w[32];            // packed weights, two bf16 each
      auto weights = [&](int h) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float x0, x1;
          unpack_f2(fma_f2(pack_f2(s[2 * e], s[2 * e + 1]), scale_2, mneg_2), x0, x1);
          const float e0 = ex2_approx(x0), e1 = ex2_approx(x1);
          uint32_t u;
          if constexpr (PLAIN) {
            u = pack_bf16(e0, e1);
            sum2[e & 1] = add_f2(sum2[e & 1], pack_f2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)));
          } else {
            // (the sum is over the weights as they were before the value scale went in: to divide it out again costs
            //  more than it gives)
            sum2[e & 1] = add_f2(sum2[e & 1], pack_f2(e0, e1));
            const float2 f = *reinterpret_cast<const float2*>(sc + C + 32 * h + 2 * e);
            u = pack_bf16(e0 * f.x, e1 * f.y);
          }
          w[16 * h + e] = __uint_as_float(u);
        }
      };
      weights(1);
      logits(0);
      weights(0);
      float s0, s1;
      unpack_f2(add_f2(sum2[0], sum2[1]), s0, s1);
      l += s0 + s1;
      if (i > 0 && __any_sync(0xffffffffu, corr != 1.f)) {
        // O of the tiles so far was summed against the old reference; the last of them has to be complete
        ok = __all_sync(0xffffffffu, mbar_wait_bounded(&bar_o[t][(i - 1) & 1], (uint32_t)(((i - 1) >> 1) & 1))) != 0;
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < D; c += 32) {
          float o[32];
          tmem_ld32(base + 128 + c, o);
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] *= corr;
          tmem_st32(base + 128 + c, o);
        }
      }
      tmem_st32(tm_s, w);
      tmem_st_wait();
      tc_fence_before();
      mbar_arrive(&bar_p[t][i & 1]);
    }
    if (ok && n > 0) {
      ok = __all_sync(0xffffffffu, mbar_wait_bounded(&bar_o[t][(n - 1) & 1], (uint32_t)(((n - 1) >> 1) & 1))) != 0;
      tc_fence_after();
    }
    named_barrier_sync(1, 32 * (S::SOFT_WARPS + 4));       // the producers' word on odd values
    pdl_launch_dependents();
    if (last && !real) l = TREE_PADDING;
    const bool in = node >= 0;
    const int g = in ? m - node * p.G : 0;
    const float r = ok ? (l == TREE_PADDING || l == 0.f ? 0.f : 1.f / l) : __uint_as_float(0x7fc00000u);
    const long long at = ((long long)split * gridDim.z + blockIdx.z) * p.M + m;
    if (p.splits > 1 && in) p.part_ml[at] = make_float2(m_ref, ok ? l : __uint_as_float(0x7fc00000u));
#pragma unroll
    for (int c = 0; c < D; c += 32) {
      float o[32];
      tmem_ld32(base + 128 + c, o);      // (nothing was written there in a block without columns: o is not used then)
      if (n == 0 || (l == TREE_PADDING && ok)) {
#pragma unroll
        for (int k = 0; k < 32; ++k) o[k] = 0.f;
      }
      if (last && odd_s && real) tree_add_odd<S::WORDS, 32>(p, b, hk, anc, D, c, o);
      if (in && p.splits == 1) {
        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(p.out) + (((long long)node * p.B + b) * p.H + hk * p.G + g) * D + c;
#pragma unroll
        for (int k = 0; k < 32; k += 8)
          *reinterpret_cast<uint4*>(dst + k) = make_uint4(pack_bf16(o[k] * r, o[k + 1] * r), pack_bf16(o[k + 2] * r, o[k + 3] * r),
                                                          pack_bf16(o[k + 4] * r, o[k + 5] * r), pack_bf16(o[k + 6] * r, o[k + 7] * r));
      } else if (in) {
        float* dst = p.part_acc + at * D + c;
#pragma unroll
        for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(dst + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
      }
      __syncwarp();
    }
  }
  if (warp >= S::SOFT_WARPS && warp < S::SOFT_WARPS + 4) named_barrier_sync(1, 32 * (S::SOFT_WARPS + 4));
  tc_fence_before();
  __syncthreads();
  if (warp == S::SOFT_WARPS + 4)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::TMEM_COLS) : "memory");
}

}  // namespace tova
