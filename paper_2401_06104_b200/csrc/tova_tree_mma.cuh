// Attention of drafted tokens over a state on warp-level matrix instructions (see tova_tree.cuh for the operation):
// bf16 queries, up to 64 rows of the product (nodes x query heads of a KV head), states in bf16, int8 or e4m3.
//
// With few rows the kernel's only hard limit is the state's bytes, so everything else hides behind their copies: a
// block of four warps runs down its columns in tiles of 64, copied ahead (cp.async, several stages) into swizzled
// shared memory.  WR groups of warps share out the rows, the 4 / WR warps of a group the tile's columns; every warp
// keeps a running maximum, sum and O of its own over the columns it has seen, and the warps are joined once, at the
// end, through shared memory.  Where the columns of a (sequence, KV head) are cut into at most eight runs, the blocks of the
// runs form a cluster and join through distributed shared memory: a second kernel would cost a small call as much again.
// O is rescaled only when some row's maximum moved.  The drafts are one more tile, copied
// ahead like the others.  The weights are summed as they were rounded to bf16, so that what multiplies V adds up to one.
// Measured (GPU time, in a captured graph): 8 chained drafts of 64 sequences over up to 1024 rows of 32 heads x 128 (738 MB) 139
// us, 5.3 TB/s, DRAM bound; one token over 1000 int8 rows of 8 KV heads 8.2 us, the latency of one cluster.  Single steps of 64
// sequences over 1024 rows of 32 heads: bf16 168 us (6.4 TB/s), int8 203, e4m3 206; over 32 x 4096 rows of 8 heads 108, 138,
// 139: an 8-bit state's bytes would take half, the conversion of its codes takes longer.
//
// 8-bit states are converted on the way from shared memory to the matrix instructions' operands, each code once per
// row group: int8 by pasting its 7 low bits and its sign bit behind the exponent of 128 (two bf16 numbers whose
// difference is the code), e4m3 by shifting exponent and mantissa into bf16's and multiplying by 2^120; both exact.
// A key with one of e4m3's two NaN codes gets the scale NaN where it lies, a value's component is noted and made NaN at the end.
// The row's scale goes onto the logit and onto the weight, never onto a converted operand.  So that a thread's operand
// elements are neighbouring bytes, the order of the contraction index (over D for the logits) and of O's columns is a
// permutation of the natural one - the sums do not care, the operands of the other side follow it.
#pragma once

#include <cooperative_groups.h>

#include "tova_mma.cuh"
#include "tova_tc.cuh"     // ex2_approx
#include "tova_tree.cuh"

namespace tova {

constexpr int TREE_MMA_NODES = 64;     // M <= 64, so there are no more nodes than that: the drafts are one tile

// W warps a block, tiles of 16 W columns.  Four warps and two blocks per SM where there are blocks enough to fill the GPU;
// eight warps a block where there are not, so that fewer tiles follow one another and two warps share a scheduler.
template <int D, int FMT, int MT, int WR, int W>
struct TreeMmaShape {
  static constexpr int THREADS = 32 * W;
  static constexpr int COLS = 16 * W;                   // columns of a tile
  static constexpr int WK = W / WR;                     // warps that share out a tile's columns
  static constexpr int KS = COLS / WK;                  // columns of a warp
  static constexpr int NB = KS / 8;
  static constexpr int ROWS = 16 * MT * WR;             // rows of the product per block
  static constexpr int ROW_BYTES = D * (FMT == FORMAT_PLAIN ? 2 : 1);
  static constexpr int TILE = COLS * ROW_BYTES;
  static constexpr int STAGE = 2 * TILE + (FMT == FORMAT_PLAIN ? 0 : 2 * COLS * 4);
  // 48 to 100 KiB a block and two blocks per SM, or twice that and one: about twice what the memory's latency asks for
  static constexpr int STAGES = FMT == FORMAT_PLAIN ? 3 : (D == 128 ? 5 : 8);
  static constexpr int Q_BYTES = ROWS * D * 2;
  static constexpr int SMEM = STAGES * STAGE + Q_BYTES;
  // the drafts take one stage (bf16 states), or one for their keys and one for their values (8-bit states)
  static constexpr int DRAFT_STAGES = FMT == FORMAT_PLAIN ? 1 : 2;
  static_assert(COLS * D * 2 * (FMT == FORMAT_PLAIN ? 2 : 1) <= STAGE && STAGES > DRAFT_STAGES, "drafts fit the ring");
  // the ring's room is taken over by the joining of the warps
  static_assert(WK * ROWS * (D * 4 + 8) <= STAGES * STAGE, "partial results fit the ring");
  static_assert(ROWS * 8 <= Q_BYTES, "a block's maxima and sums fit Q's room");
};

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Bytes ia and ib of the eight bytes (a, b) as two bf16 numbers, ia in the low half.
template <int FMT>
__device__ __forceinline__ uint32_t tree_codes2(uint32_t a, uint32_t b, int ia, int ib) {
  if constexpr (FMT == FORMAT_INT8) {
    const uint32_t x = __byte_perm(a, b, (uint32_t)(ia | (ib << 8)));            // code in the low byte of each half
    const uint32_t lo = (x & 0x007f007fu) | 0x43004300u;                         // 128 + low seven bits
    const uint32_t hi = (x & 0x00800080u) | 0x43004300u;                         // 128, or 256 for a negative code
    const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&lo), *reinterpret_cast<const __nv_bfloat162*>(&hi));
    return *reinterpret_cast<const uint32_t*>(&d);
  } else {
    const uint32_t x = __byte_perm(a, b, (uint32_t)((ia << 4) | (ib << 12)));    // code in the high byte of each half
    const uint32_t w = (x & 0x80008000u) | ((x >> 4) & 0x07f007f0u);
    const uint32_t up = 0x7b807b80u;                                             // 2^120: from exponent bias 7 to 127
    const __nv_bfloat162 d = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&w), *reinterpret_cast<const __nv_bfloat162*>(&up));
    return *reinterpret_cast<const uint32_t*>(&d);
  }
}

// e4m3 has no infinities, and NaN for the codes 0x7f and 0xff, which tree_codes2 turns into 480 and -480.  A state may hold them
// (tova_quant_write stores none, but codes converted elsewhere can), so all that is converted is looked at: adding one to a
// byte changes its top bit only where the seven others are ones.  (A carry out of 0xff reaches the next byte, beside a
// code that has been found.)  Two instructions for four codes, beside ten that convert them: single steps over 64 x 32 heads x
// 1024 rows take 206 us where 191 without, trees of 25 over 4 x 16001 rows (tcgen05 kernel) 93 where 90.
// Here: the top bits of w's NaN codes | what has been found before.
__device__ __forceinline__ uint32_t tree_nan_codes(uint32_t w, uint32_t found) { return found | (w ^ (w + 0x01010101u)); }
__device__ __forceinline__ uint32_t tree_nan_codes(const uint4& w, uint32_t found) {
  return tree_nan_codes(w.w, tree_nan_codes(w.z, tree_nan_codes(w.y, tree_nan_codes(w.x, found))));
}
constexpr uint32_t TREE_NAN_FOUND = 0x80808080u;
// The bytes of four codes that are NaN, as bits 0..3.
__device__ __forceinline__ uint32_t tree_which_nan(uint32_t w) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m |= (uint32_t)(((w >> (8 * i)) & 0x7fu) == 0x7fu) << i;
  return m;
}
// tree_codes2's results where a NaN may be among the codes: nothing else gives 480.
__device__ __forceinline__ uint32_t tree_mark_nan(uint32_t d) {
  if ((d & 0x00007fffu) == 0x000043f0u) d |= 0x00007fffu;
  if ((d & 0x7fff0000u) == 0x43f00000u) d |= 0x7fff0000u;
  return d;
}

// Byte offset of 16-byte chunk `ch` of row `row` in a tile.  bf16 rows: the low three chunk bits turn with the row, so
// that eight rows' chunks (one ldmatrix) fall into different banks.  8-bit rows: both readers below - eight lanes on two
// neighbouring rows x four chunks, or on four rows two apart x two chunks - find eight different chunks of a 128-byte line.
template <int ROW_BYTES>
__device__ __forceinline__ uint32_t tree_off16(int row, int ch) {
  return (uint32_t)(row * ROW_BYTES + ((ch ^ (row & 7)) << 4));
}
template <int D>
__device__ __forceinline__ uint32_t tree_off8(int row, int ch) {
  if constexpr (D == 128) return (uint32_t)(row * 128 + ((ch ^ (((row >> 1) & 3) << 1) ^ ((row & 1) << 2)) << 4));
  else return (uint32_t)((row >> 1) * 128 + (((((row & 1) << 2) | ch) ^ (((row >> 1) & 3) << 1)) << 4));
}

constexpr int TREE_CLUSTER_MAX = 8;

template <int D, int FMT, int MT, int WR, bool CLUSTER>
__global__ void __launch_bounds__(CLUSTER ? 256 : 128, CLUSTER ? 1 : 2) tova_tree_mma_kernel(const __grid_constant__ TreeParams p) {
  using S = TreeMmaShape<D, FMT, MT, WR, CLUSTER ? 8 : 4>;
  constexpr int THREADS = S::THREADS, C = S::COLS, KS = S::KS, NB = S::NB, OB = D / 8;
  constexpr bool PLAIN = FMT == FORMAT_PLAIN;
  extern __shared__ __align__(128) unsigned char tree_smem[];
  unsigned char* ring = tree_smem;
  uint4* q_s = reinterpret_cast<uint4*>(tree_smem + S::STAGES * S::STAGE);    // operand order: [row tile][step][lane]

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int wr = warp / S::WK, wk = warp % S::WK;
  const int lr = lane >> 2, lc = lane & 3;
  const int b = blockIdx.z / p.Hkv, hk = blockIdx.z % p.Hkv;
  const int split = blockIdx.y;
  const int len = tree_len(p, b);
  const bool last = split == p.splits - 1;
  const int c0 = split * p.split_cols;
  const int c1 = last ? len : min(len, c0 + p.split_cols);
  const int n_tiles = c1 > c0 ? (c1 - c0 + C - 1) / C : 0;
  const uint32_t ring_a = smem_addr(ring);

  const unsigned char* Kg = static_cast<const unsigned char*>(p.K) + (long long)blockIdx.z * p.cap * S::ROW_BYTES;
  const unsigned char* Vg = static_cast<const unsigned char*>(p.V) + (long long)blockIdx.z * p.cap * S::ROW_BYTES;
  const float* ksg = PLAIN ? nullptr : p.k_scale + (long long)blockIdx.z * p.cap;
  const float* vsg = PLAIN ? nullptr : p.v_scale + (long long)blockIdx.z * p.cap;

  // Draft `row`'s chunk `ch` of k_new or v_new.
  auto draft_src = [&](const void* x, int row, int ch) {
    return static_cast<const unsigned char*>(x) + ((((long long)min(row, p.N - 1) * p.B + b) * p.Hkv + hk) * D + ch * 8) * 2;
  };
  const int n_loads = n_tiles + (last ? S::DRAFT_STAGES : 0);
  auto load_tile = [&](int i) {
    const int j0 = c0 + i * C;
    const uint32_t st = ring_a + (i % S::STAGES) * S::STAGE;
    constexpr int CH = S::ROW_BYTES / 16;
    if (i >= n_tiles) {
      constexpr int DC = D / 8;
#pragma unroll
      for (int x = 0; x < C * DC / THREADS; ++x) {
        const int e = x * THREADS + tid;
        const int row = e / DC, ch = e % DC;
        const uint32_t off = tree_off16<2 * D>(row, ch), size = row < p.N ? 16u : 0u;
        if (PLAIN) {
          cp_async16(st + off, draft_src(p.k_new, row, ch), size);
          cp_async16(st + S::TILE + off, draft_src(p.v_new, row, ch), size);
        } else {
          cp_async16(st + off, draft_src(i == n_tiles ? p.k_new : p.v_new, row, ch), size);
        }
      }
      return;
    }
#pragma unroll
    for (int x = 0; x < C * CH / THREADS; ++x) {
      const int e = x * THREADS + tid;
      const int row = e / CH, ch = e % CH;
      const bool in = j0 + row < c1;                       // columns behind the run are zeros, whatever lies there
      const long long at = (long long)(in ? j0 + row : c0) * S::ROW_BYTES + ch * 16;
      const uint32_t off = PLAIN ? tree_off16<S::ROW_BYTES>(row, ch) : tree_off8<D>(row, ch);
      cp_async16(st + off, Kg + at, in ? 16u : 0u);
      cp_async16(st + S::TILE + off, Vg + at, in ? 16u : 0u);
    }
    if constexpr (!PLAIN) {
      static_assert(THREADS == 2 * C, "one scale a thread");
      const int row = tid & (C - 1);
      const bool in = j0 + row < c1;
      cp_async4(st + 2 * S::TILE + tid * 4, (tid < C ? ksg : vsg) + (in ? j0 + row : c0), in ? 4u : 0u);
    }
  };
#pragma unroll
  for (int i = 0; i < S::STAGES - 1; ++i) {
    if (i < n_loads) load_tile(i);
    cp_async_commit();
  }

  __shared__ int par_s[TREE_MMA_NODES];
  __shared__ uint32_t anc_s[TREE_MMA_NODES][2];      // ancestor bits of every node
  __shared__ int odd_s;                              // some draft's value is not finite
  constexpr bool NAN_CODES = FMT == FORMAT_E4M3;
  __shared__ uint32_t nan_s[NAN_CODES ? D / 32 : 1]; // components with a NaN code in some row of V
  if (NAN_CODES && tid < D / 32) nan_s[tid] = 0;     // (the tiles' first barrier lies between this and its first use)
  if (last) {
    if (tid < p.N) par_s[tid] = p.parents ? p.parents[(long long)tid * p.B + b] : tid - 1;
    if (tid == 0) odd_s = 0;
    __syncthreads();
    if (tid < p.N) tree_ancestor_bits<2>(tid, p.parents == nullptr, par_s, anc_s[tid]);
  }
  // Q in operand order.  Step ks of the contraction: natural order (bf16 states) k = 16 ks + 2 lc + {0,1}, + 8; permuted
  // (8-bit states), with ks = 4 i + w: d = 64 i + 16 lc + 4 w + {0,1}, {2,3}.
  for (int e = tid; e < (S::ROWS / 16) * (D / 16) * 32; e += THREADS) {
    const int l = e & 31, ks = (e >> 5) % (D / 16), rt = (e >> 5) / (D / 16);
    const int r = l >> 2, c = l & 3;
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int m = rt * 16 + r + 8 * h;
      if (m < p.M) {
        const int n = m / p.G, g = m - n * p.G;
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.q) + (((long long)n * p.B + b) * p.H + hk * p.G + g) * D;
        const int d = PLAIN ? 16 * ks + 2 * c : 64 * (ks >> 2) + 16 * c + 4 * (ks & 3);
        w[h] = *reinterpret_cast<const uint32_t*>(src + d);
        w[2 + h] = *reinterpret_cast<const uint32_t*>(src + d + (PLAIN ? 8 : 2));
      }
    }
    q_s[e] = make_uint4(w[0], w[1], w[2], w[3]);
  }

  float o[MT][OB][4];
  float m_run[MT][2], l_run[MT][2];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
#pragma unroll
    for (int j = 0; j < OB; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[t][j][e] = 0.f;
    m_run[t][0] = m_run[t][1] = -INFINITY;
    l_run[t][0] = l_run[t][1] = 0.f;
  }

  // Soft-max of one tile's logits s (scaled, masked): weights in place, running maximum updated, sum and O rescaled if it
  // moved.
  auto softmax = [&](float (&s)[MT][NB][4]) {
    float corr[MT][2];
    bool moved = false;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float top = -INFINITY;
#pragma unroll
        for (int n = 0; n < NB; ++n) top = fmaxf(top, fmaxf(s[t][n][2 * h], s[t][n][2 * h + 1]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const float m_new = fmaxf(m_run[t][h], top);
        const float base = m_new == -INFINITY ? 0.f : m_new;
        corr[t][h] = ex2_approx(m_run[t][h] - base);
        moved |= m_new != m_run[t][h];
        m_run[t][h] = m_new;
        l_run[t][h] *= corr[t][h];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          s[t][n][2 * h] = ex2_approx(s[t][n][2 * h] - base);
          s[t][n][2 * h + 1] = ex2_approx(s[t][n][2 * h + 1] - base);
        }
      }
    if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int j = 0; j < OB; ++j) {
          o[t][j][0] *= corr[t][0];
          o[t][j][1] *= corr[t][0];
          o[t][j][2] *= corr[t][1];
          o[t][j][3] *= corr[t][1];
        }
    }
  };
  // Two neighbouring weights as operand elements, times the columns' value scales f (8-bit states); added to the running
  // sum as rounded, the scales' reciprocals r taken out again; where those would leave fp32's range (a row of zeros, or one
  // written with hardly more), as it was.  (The sum is this thread's; a row's four threads add up at the end.)
  auto weight2 = [&](float w0, float w1, float f0, float f1, float r0, float r1, float& sum) -> uint32_t {
    if constexpr (PLAIN) {
      const uint32_t u = pack_bf16(w0, w1);
      sum += __uint_as_float(u << 16) + __uint_as_float(u & 0xffff0000u);
      return u;
    } else {
      const uint32_t u = pack_bf16(w0 * f0, w1 * f1);
      sum += (fabsf(f0) >= 0x1p-100f ? __uint_as_float(u << 16) * r0 : w0) +
             (fabsf(f1) >= 0x1p-100f ? __uint_as_float(u & 0xffff0000u) * r1 : w1);
      return u;
    }
  };
  auto q_frag = [&](int t, int ks, uint32_t (&a)[4]) {
    const uint4 w = q_s[((wr * MT + t) * (D / 16) + ks) * 32 + lane];
    a[0] = w.x; a[1] = w.y; a[2] = w.z; a[3] = w.w;
  };
  const int kb = wk * KS;      // this warp's first column within a tile

  for (int i = 0; i < n_tiles; ++i) {
    cp_async_wait<S::STAGES - 2>();
    __syncthreads();
    if (i + S::STAGES - 1 < n_loads) load_tile(i + S::STAGES - 1);
    cp_async_commit();
    const unsigned char* stp = ring + (i % S::STAGES) * S::STAGE;
    const uint32_t st = smem_addr(stp);
    uint32_t nan_k = 0, nan_v = 0;                       // NaN codes among the tile's, as tree_nan_codes finds them
    float s[MT][NB][4];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[t][n][e] = 0.f;
    if constexpr (PLAIN) {
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        uint32_t a[MT][4];
#pragma unroll
        for (int t = 0; t < MT; ++t) q_frag(t, ks, a[t]);
#pragma unroll
        for (int n = 0; n < NB; n += 2) {
          uint32_t f[4];
          ldmatrix_x4(f, st + tree_off16<S::ROW_BYTES>(kb + n * 8 + ((lane >> 4) << 3) + (lane & 7), 2 * ks + ((lane >> 3) & 1)));
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            mma_bf16(s[t][n], a[t], f[0], f[1]);
            mma_bf16(s[t][n + 1], a[t], f[2], f[3]);
          }
        }
      }
    } else {
#pragma unroll
      for (int hf = 0; hf < D / 64; ++hf) {
        uint4 kw[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          kw[n] = *reinterpret_cast<const uint4*>(stp + tree_off8<D>(kb + n * 8 + lr, 4 * hf + lc));
          if (NAN_CODES) nan_k = tree_nan_codes(kw[n], nan_k);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t a[MT][4];
#pragma unroll
          for (int t = 0; t < MT; ++t) q_frag(t, 4 * hf + w, a[t]);
#pragma unroll
          for (int n = 0; n < NB; ++n) {
            const uint32_t x = w == 0 ? kw[n].x : w == 1 ? kw[n].y : w == 2 ? kw[n].z : kw[n].w;
            const uint32_t b0 = tree_codes2<FMT>(x, x, 0, 1), b1 = tree_codes2<FMT>(x, x, 2, 3);
#pragma unroll
            for (int t = 0; t < MT; ++t) mma_bf16(s[t][n], a[t], b0, b1);
          }
        }
      }
    }
    float* ks_s = reinterpret_cast<float*>(ring + (i % S::STAGES) * S::STAGE + 2 * S::TILE);
    if constexpr (NAN_CODES) {
      if (__any_sync(0xffffffffu, (nan_k & TREE_NAN_FOUND) != 0)) {      // (every warp that reads the column finds it itself)
#pragma unroll 1
        for (int n = 0; n < NB; ++n)
#pragma unroll 1
          for (int hf = 0; hf < D / 64; ++hf)
            if (tree_nan_codes(*reinterpret_cast<const uint4*>(stp + tree_off8<D>(kb + n * 8 + lr, 4 * hf + lc)), 0u) & TREE_NAN_FOUND)
              ks_s[kb + n * 8 + lr] = __uint_as_float(0x7fc00000u);
        __syncwarp();
      }
    }
    const int left = c1 - (c0 + i * C) - kb;             // columns of this warp's share that exist
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int col = n * 8 + 2 * lc + e;
        const float f = PLAIN ? p.scale2 : p.scale2 * ks_s[kb + col];
        const bool in = col < left;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          s[t][n][e] = in ? s[t][n][e] * f : -INFINITY;
          s[t][n][2 + e] = in ? s[t][n][2 + e] * f : -INFINITY;
        }
      }
    softmax(s);
#pragma unroll
    for (int kk = 0; kk < KS / 16; ++kk) {
      uint32_t a[MT][4];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int n = 2 * kk + x;
        float f[2] = {1.f, 1.f}, r[2] = {1.f, 1.f};
        if constexpr (!PLAIN) {
          const float2 w = *reinterpret_cast<const float2*>(ks_s + C + kb + n * 8 + 2 * lc);
          f[0] = w.x; f[1] = w.y;
          r[0] = __frcp_rn(w.x); r[1] = __frcp_rn(w.y);
        }
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          a[t][2 * x] = weight2(s[t][n][0], s[t][n][1], f[0], f[1], r[0], r[1], l_run[t][0]);
          a[t][2 * x + 1] = weight2(s[t][n][2], s[t][n][3], f[0], f[1], r[0], r[1], l_run[t][1]);
        }
      }
      if constexpr (PLAIN) {
#pragma unroll
        for (int j = 0; j < OB; j += 2) {
          uint32_t f[4];
          ldmatrix_x4_trans(f, st + S::TILE + tree_off16<S::ROW_BYTES>(kb + kk * 16 + (lane & 15), j + (lane >> 4)));
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            mma_bf16(o[t][j], a[t], f[0], f[1]);
            mma_bf16(o[t][j + 1], a[t], f[2], f[3]);
          }
        }
      } else {
        // rows (columns of the product) 2 lc, 2 lc + 1, + 8, + 9; bytes (D/8) lr ..: O's column block j is their byte j
        uint32_t vw[4][D / 32];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = kb + kk * 16 + 2 * lc + (r & 1) + 8 * (r >> 1);
          if constexpr (D == 128) {
            const uint4 x = *reinterpret_cast<const uint4*>(stp + S::TILE + tree_off8<D>(row, lr));
            vw[r][0] = x.x; vw[r][1] = x.y; vw[r][2] = x.z; vw[r][3] = x.w;
          } else {
            const uint2 x = *reinterpret_cast<const uint2*>(stp + S::TILE + tree_off8<D>(row, lr >> 1) + (lr & 1) * 8);
            vw[r][0] = x.x; vw[r][1] = x.y;
          }
          if (NAN_CODES) {
#pragma unroll
            for (int x = 0; x < D / 32; ++x) nan_v = tree_nan_codes(vw[r][x], nan_v);
          }
        }
#pragma unroll
        for (int j = 0; j < OB; ++j) {
          const uint32_t b0 = tree_codes2<FMT>(vw[0][j >> 2], vw[1][j >> 2], j & 3, 4 + (j & 3));
          const uint32_t b1 = tree_codes2<FMT>(vw[2][j >> 2], vw[3][j >> 2], j & 3, 4 + (j & 3));
#pragma unroll
          for (int t = 0; t < MT; ++t) mma_bf16(o[t][j], a[t], b0, b1);
        }
      }
    }
    if constexpr (NAN_CODES) {
      if ((nan_v & TREE_NAN_FOUND) != 0) {               // every real row sees the state's rows: only the components count
#pragma unroll 1
        for (int x = 0; x < KS / 4 * (D / 32); ++x) {
          const int r = x / (D / 32), row = kb + (r >> 2) * 16 + 2 * lc + (r & 1) + 8 * ((r >> 1) & 1), byte = OB * lr + 4 * (x % (D / 32));
          const uint32_t m = tree_which_nan(*reinterpret_cast<const uint32_t*>(stp + S::TILE + tree_off8<D>(row, byte >> 4) + (byte & 15)));
          if (m) atomicOr(&nan_s[byte >> 5], m << (byte & 31));
        }
      }
    }
  }
  cp_async_wait<0>();

  // The drafts: up to 64 more columns, in bf16, masked by ancestry.
  uint32_t real = 0;        // bit 2 t + h: this thread's row is a node's, not padding
  if (last) {
    unsigned char* dk = ring + (n_tiles % S::STAGES) * S::STAGE;
    unsigned char* dv = PLAIN ? dk + S::TILE : ring + ((n_tiles + 1) % S::STAGES) * S::STAGE;
    // A draft that a row does not see may hold anything, and 0 times an infinity is not 0: values that are not finite
    // are taken out (each thread looks at the chunks it copied) and added at the end to the rows that see them.
#pragma unroll
    for (int x = 0; x < C * (D / 8) / THREADS; ++x) {
      const int e = x * THREADS + tid;
      uint4* at = reinterpret_cast<uint4*>(dv + tree_off16<2 * D>(e / (D / 8), e % (D / 8)));
      uint4 w = *at;
      if (tree_drop_odd(w)) {
        *at = w;
        odd_s = 1;
      }
    }
    __syncthreads();
    if (kb < p.N) {           // this warp has drafts
      float s[MT][NB][4];
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[t][n][e] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        uint32_t a[MT][4];
#pragma unroll
        for (int t = 0; t < MT; ++t) q_frag(t, ks, a[t]);
#pragma unroll
        for (int n = 0; n < NB; n += 2) {
          uint32_t f[4];
          if constexpr (PLAIN) {
            ldmatrix_x4(f, smem_addr(dk) + tree_off16<2 * D>(kb + n * 8 + ((lane >> 4) << 3) + (lane & 7), 2 * ks + ((lane >> 3) & 1)));
          } else {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const uint2 w = *reinterpret_cast<const uint2*>(
                  dk + tree_off16<2 * D>(kb + (n + x) * 8 + lr, 8 * (ks >> 2) + 2 * lc + ((ks & 3) >> 1)) + (ks & 1) * 8);
              f[2 * x] = w.x;
              f[2 * x + 1] = w.y;
            }
          }
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            mma_bf16(s[t][n], a[t], f[0], f[1]);
            mma_bf16(s[t][n + 1], a[t], f[2], f[3]);
          }
        }
      }
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int m = (wr * MT + t) * 16 + lr + 8 * h;
          const uint32_t* anc = anc_s[min(m, p.M - 1) / p.G];
          const uint32_t a0 = m < p.M ? anc[0] : 0u, a1 = m < p.M ? anc[1] : 0u;
#pragma unroll
          for (int n = 0; n < NB; ++n) {
            const int col = kb + n * 8 + 2 * lc;          // even: both columns are in one word
            const uint32_t see = (col < 32 ? a0 : a1) >> (col & 31);
            s[t][n][2 * h] = (see & 1u) ? s[t][n][2 * h] * p.scale2 : -INFINITY;
            s[t][n][2 * h + 1] = (see & 2u) ? s[t][n][2 * h + 1] * p.scale2 : -INFINITY;
          }
        }
      softmax(s);
#pragma unroll
      for (int kk = 0; kk < KS / 16; ++kk) {
        uint32_t a[MT][4];
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            a[t][2 * x] = weight2(s[t][2 * kk + x][0], s[t][2 * kk + x][1], 1.f, 1.f, 1.f, 1.f, l_run[t][0]);
            a[t][2 * x + 1] = weight2(s[t][2 * kk + x][2], s[t][2 * kk + x][3], 1.f, 1.f, 1.f, 1.f, l_run[t][1]);
          }
        if constexpr (PLAIN) {
#pragma unroll
          for (int j = 0; j < OB; j += 2) {
            uint32_t f[4];
            ldmatrix_x4_trans(f, smem_addr(dv) + tree_off16<2 * D>(kb + kk * 16 + (lane & 15), j + (lane >> 4)));
#pragma unroll
            for (int t = 0; t < MT; ++t) {
              mma_bf16(o[t][j], a[t], f[0], f[1]);
              mma_bf16(o[t][j + 1], a[t], f[2], f[3]);
            }
          }
        } else {
#pragma unroll
          for (int j = 0; j < OB; j += 2) {               // O's columns (D/8) lr + j, + 1 of four drafts
            uint32_t w[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int row = kb + kk * 16 + 2 * lc + (r & 1) + 8 * (r >> 1);
              const int d = OB * lr + j;
              w[r] = *reinterpret_cast<const uint32_t*>(dv + tree_off16<2 * D>(row, d >> 3) + (d & 7) * 2);
            }
#pragma unroll
            for (int t = 0; t < MT; ++t) {
              mma_bf16(o[t][j], a[t], __byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410));
              mma_bf16(o[t][j + 1], a[t], __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632));
            }
          }
        }
      }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int m = (wr * MT + t) * 16 + lr + 8 * h;
        if (m < p.M) real |= (uint32_t)((anc_s[m / p.G][0] | anc_s[m / p.G][1]) != 0) << (2 * t + h);
      }
  }
  pdl_launch_dependents();

  // Join the warps that shared out the columns: maxima and sums first, then O scaled to the common maximum.
  __syncthreads();
  float* o_s = reinterpret_cast<float*>(ring);                       // [WK][ROWS][D]
  float2* ml_s = reinterpret_cast<float2*>(ring + S::WK * S::ROWS * D * 4);   // [WK][ROWS]
  // Float offset of 16-byte chunk q of row r: the chunks turn with the row, and where a thread holds whole chunks also with
  // their eighth, so that the lanes that store together meet different banks.
  auto place = [](int r, int q) { return PLAIN ? (q ^ ((r << 1) & 7)) * 4 : (q ^ ((r ^ ((q >> 3) << 1)) & 7)) * 4; };
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float l = l_run[t][h];
      l += __shfl_xor_sync(0xffffffffu, l, 1);
      l += __shfl_xor_sync(0xffffffffu, l, 2);
      const int r = (wr * MT + t) * 16 + lr + 8 * h;
      if (lc == 0) ml_s[wk * S::ROWS + r] = make_float2(m_run[t][h], last && !((real >> (2 * t + h)) & 1u) ? TREE_PADDING : l);
    }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = (wr * MT + t) * 16 + lr + 8 * h;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < S::WK; ++w) top = fmaxf(top, ml_s[w * S::ROWS + r].x);
      const float f = top == -INFINITY ? 0.f : ex2_approx(m_run[t][h] - top);
      if (r < p.M) {
        float* dst = o_s + (wk * S::ROWS + r) * D;
        if constexpr (PLAIN) {
#pragma unroll
          for (int j = 0; j < OB; ++j)
            *reinterpret_cast<float2*>(dst + place(r, 2 * j + (lc >> 1)) + 2 * (lc & 1)) = make_float2(o[t][j][2 * h] * f, o[t][j][2 * h + 1] * f);
        } else {
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int j = 0; j < OB; j += 4)
              *reinterpret_cast<float4*>(dst + place(r, OB / 4 * (2 * lc + e) + j / 4)) =
                  make_float4(o[t][j][2 * h + e] * f, o[t][j + 1][2 * h + e] * f, o[t][j + 2][2 * h + e] * f, o[t][j + 3][2 * h + e] * f);
        }
      }
    }
  __syncthreads();
  // A row's four components d .. d+3 over this block's warps; the row's maximum and sum.
  auto joined = [&](int r, int d, float& top, float& l) {
    top = -INFINITY;
    l = 0.f;
    bool pad = false;
#pragma unroll
    for (int w = 0; w < S::WK; ++w) top = fmaxf(top, ml_s[w * S::ROWS + r].x);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < S::WK; ++w) {
      const float2 ml = ml_s[w * S::ROWS + r];
      pad |= ml.y == TREE_PADDING;
      if (ml.x != -INFINITY) l += ml.y * ex2_approx(ml.x - top);
      const float4 x = *reinterpret_cast<const float4*>(o_s + (w * S::ROWS + r) * D + place(r, d >> 2));
      acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
    }
    if (last && odd_s && !pad) {
      float v[4] = {acc.x, acc.y, acc.z, acc.w};
      tree_add_odd<2, 4>(p, b, hk, anc_s[r / p.G], D, d, v);
      acc = make_float4(v[0], v[1], v[2], v[3]);
    }
    if constexpr (NAN_CODES) {
      const uint32_t m = nan_s[d >> 5] >> (d & 31);
      const float nan = __uint_as_float(0x7fc00000u);
      if (m & 1u) acc.x = nan;
      if (m & 2u) acc.y = nan;
      if (m & 4u) acc.z = nan;
      if (m & 8u) acc.w = nan;
    }
    if (pad) l = TREE_PADDING;
    return acc;
  };
  auto write = [&](int m, int d, const float4& acc, float l) {
    const float f = 1.f / l;      // (l = 0: every logit is minus infinity, and the result NaN)
    const int n = m / p.G, g = m - n * p.G;
    __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(p.out) + (((long long)n * p.B + b) * p.H + hk * p.G + g) * D + d;
    if (l == TREE_PADDING) tree_store4<__nv_bfloat16>(dst, 0.f, 0.f, 0.f, 0.f);
    else tree_store4<__nv_bfloat16>(dst, acc.x * f, acc.y * f, acc.z * f, acc.w * f);
  };
  if constexpr (CLUSTER) {
    // Every block leaves its row sums over its own first warp's partial result and its (maximum, sum) over Q; then the rows'
    // components are dealt out over the cluster's threads, and each is added up from all blocks.
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    float2* block_ml = reinterpret_cast<float2*>(q_s);
    for (int e = tid; e < p.M * (D / 4); e += THREADS) {
      const int r = e / (D / 4), d = (e % (D / 4)) * 4;
      float top, l;
      const float4 acc = joined(r, d, top, l);
      *reinterpret_cast<float4*>(o_s + r * D + place(r, d >> 2)) = acc;       // (read by this thread only, and just now)
      if (d == 0) block_ml[r] = make_float2(top, l);
    }
    cluster.sync();
    for (int e = split * THREADS + tid; e < p.M * (D / 4); e += p.splits * THREADS) {
      const int r = e / (D / 4), d = (e % (D / 4)) * 4;
      float2 ml[TREE_CLUSTER_MAX];
      float4 x[TREE_CLUSTER_MAX];
#pragma unroll
      for (int c = 0; c < TREE_CLUSTER_MAX; ++c) {
        ml[c] = make_float2(-INFINITY, 0.f);
        x[c] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c < p.splits) {
          ml[c] = cluster.map_shared_rank(block_ml, c)[r];
          x[c] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(o_s, c) + r * D + place(r, d >> 2));
        }
      }
      float top = -INFINITY, l = 0.f;
      bool pad = false;
#pragma unroll
      for (int c = 0; c < TREE_CLUSTER_MAX; ++c) {
        top = fmaxf(top, ml[c].x);
        pad |= ml[c].y == TREE_PADDING;
      }
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int c = 0; c < TREE_CLUSTER_MAX; ++c) {
        // A run without a finite logit has the factor 0, and adds its sums all the same: where its logits are NaN, so are
        // they, and the row's result.  (Its l may be NaN beside finite ones: it is left out, and the sums carry the NaN.)
        const float f = ml[c].x == -INFINITY ? 0.f : ex2_approx(ml[c].x - top);
        if (f != 0.f) l += f * ml[c].y;
        acc.x = fmaf(f, x[c].x, acc.x); acc.y = fmaf(f, x[c].y, acc.y);
        acc.z = fmaf(f, x[c].z, acc.z); acc.w = fmaf(f, x[c].w, acc.w);
      }
      write(r, d, acc, pad ? TREE_PADDING : l);
    }
    cluster.sync();      // no block leaves while another reads its shared memory
  } else {
    for (int e = tid; e < p.M * (D / 4); e += THREADS) {
      const int m = e / (D / 4), d = (e % (D / 4)) * 4;
      float top, l;
      const float4 acc = joined(m, d, top, l);
      if (p.splits == 1) {
        write(m, d, acc, l);
      } else {
        const long long at = ((long long)split * gridDim.z + blockIdx.z) * p.M + m;
        if (d == 0) p.part_ml[at] = make_float2(top, l);
        *reinterpret_cast<float4*>(p.part_acc + at * D + d) = acc;
      }
    }
  }
}

}  // namespace tova
