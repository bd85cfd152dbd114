// Attention of drafted tokens over a state on the 5th-generation tensor cores (see tova_tree.cuh for the operation):
// bf16 queries, more than 64 rows of the product (nodes x query heads of a KV head).
//
// Work.  A job is up to NT x 128 rows of one KV head of one sequence against all their columns, in tiles of 128; the
// drafts are its last tiles.  More rows than that are other jobs over the same columns: as many blocks as there are such
// jobs form a group and walk side by side, so that what one reads the others find in L2.  The tiles of all (sequence, KV
// head) pairs, one behind the other, are dealt out evenly to the groups (as many as fit the GPU at a time): each takes a
// run of `share` tiles and walks through the pairs in it.  A job that lies in one run is written out; one cut by the end of
// a run leaves (reference, sum, weighted sum) of its pieces in the workspace, at most two a block, and a second kernel joins
// them.  So lengths that differ cost nobody idle time, and hardly any job is cut.
//
// Roles in a block.  They meet through mbarriers only and run ahead of one another across jobs: while the rows of one job
// are written out, the next one's Q, K and V are on their way and its first logits computed.
//   producer warps      Q, then K and V tiles into a ring of shared-memory slots in the 128-byte-swizzled layout the tensor
//                       cores read: bf16 states by tiled TMA, as far ahead as there are slots (by cp.async the two warps
//                       could not keep up; values of rows behind a sequence's last are zeroed when they have landed,
//                       whatever lies there); 8-bit states from a raw ring, with an exact conversion (see
//                       tova_tree_mma.cuh); drafts by plain loads that take out infinities and NaN.
//   1 issuing thread    S = Q K^T (128 x 128, fp32 in TMEM) and O += P V.  Two row tiles (more than 128 rows of a bf16 state)
//                       fill the tensor memory, 256 columns each (S, O); their contractions take turns, PV_0(i) S_0(i+1)
//                       PV_1(i) S_1(i+1), so that one's run while the other's soft-max does.  One row tile has room for a
//                       second S: the next tile's logits are computed ahead of O += P V of this one.
//   1 copying thread    (8-bit states) bulk copies into the raw ring: a producer that had to wait for all of them to be done
//                       with a raw slot before it could ask for the next copy would hold up its own conversions
//   1 helper warp       ancestor bits of the next job's drafts, and whether one of their values is not finite
//   8 warps a row tile  two threads a row, 64 columns each: logits from TMEM, weights as bf16 back over them, where they are
//                       the A operand of O += P V.  The weights' reference is a whole number, set by a job's first tile
//                       (which takes a pass for the maximum) and hardly ever moved again: floating point loses nothing on
//                       weights above 1, so a later tile needs no maximum; only where a row's weights sum to more than 2^32
//                       is the tile done over, with a factor of a power of two on what was summed before.  The sum is taken
//                       over the rounded weights, so that the weights that multiply V add up to one.
// A tile of 128 columns, not 64, because S = Q K^T reads both operands from shared memory: 8 KiB per 64 cycles of math
// (128 x 128 x 16) are what shared memory delivers, 6 KiB per 32 cycles (128 x 64 x 16) are not.  TMEM: 256 columns per row
// tile (S 128, O 128).  Every wait is bounded; one that runs out leaves NaN in the rows that the block had yet to write.
// Measured (GPU time, in a captured graph; a call among others takes 162 and 96 us): trees of 63 drafts, 32 sequences x up to 4000
// bf16 rows, 32 query over 8 KV heads x 128 (89.5 GFLOP) 146 us, 610 TFLOP/s, bound by the round trips between contraction and
// soft-max; trees of 25, 4 x 16001 e4m3 rows, 8 query heads a KV head (26.2 GFLOP) 93 us, 280 TFLOP/s, bound by the
// instructions of the conversion and the soft-max.
#pragma once

#include "tova_tree_mma.cuh"

namespace tova {

constexpr int TREE_TC_ROWS = 128;      // rows of a tile
constexpr int TREE_TC_COLS = 128;      // columns of a tile
constexpr float TREE_TC_MOST = 4294967296.f;   // a larger sum of a thread's weights moves the row's reference

template <int D, int FMT, int NT>
struct TreeTcShape {
  static constexpr bool PLAIN = FMT == FORMAT_PLAIN;
  static constexpr int SOFT_WARPS = 8 * NT;
  static constexpr int PRODUCER_WARPS = PLAIN ? 2 : 8;
  static constexpr bool DOUBLE = NT == 1;                          // two S buffers
  static_assert(PLAIN || NT == 1, "an 8-bit state's conversion takes eight warps and their registers: one row tile");
  static constexpr int THREADS = 32 * (SOFT_WARPS + PRODUCER_WARPS + (PLAIN ? 2 : 3));
  static constexpr int Q_BYTES = TREE_TC_ROWS * D * 2;             // per row tile
  static constexpr int SLOT = TREE_TC_COLS * D * 2;
  static constexpr int SLOTS = (PLAIN && NT == 1 ? 5 : 4) * (128 / D);
  static constexpr int RAW = PLAIN ? 0 : TREE_TC_COLS * D;
  static constexpr int RAW_SLOTS = PLAIN ? 0 : 3 * (128 / D);
  // Tiles whose scales are kept.  K of tile i takes the slot of a copy SLOTS positions back, K of tile j = i - SLOTS/2.  When
  // that has been consumed, S of tile j is complete; with two S buffers it was issued behind the weights of tile j - 2, not
  // of tile j - 1, so the soft-max of tile i - SLOTS/2 - 2 has passed and that tile's scales may be written over, and no later
  // one's.
  static constexpr int SCALE_TILES = SLOTS / 2 + 2;
  static_assert(PLAIN || (DOUBLE && SLOTS % 2 == 0 && SCALE_TILES >= SLOTS / 2 + 2), "a tile's scales outlast its soft-max");
  static constexpr int SCALES = PLAIN ? 0 : SCALE_TILES * 3 * TREE_TC_COLS * 4;
  static constexpr int SMEM = NT * Q_BYTES + SLOTS * SLOT + RAW_SLOTS * RAW + SCALES + 1024;
  static constexpr int TMEM_COLS = DOUBLE ? 512 : 256 * NT;
  static constexpr int BUFFERS = DOUBLE ? 2 : NT;                  // S buffers (and barriers for them)
  // Trimmed tiles lie at least four ring positions apart (a job's last V, its drafts' K and V, the next job's K and V), and
  // no producer is more than SLOTS positions ahead of another: with this many barriers none can come round to one that
  // another still waits on.
  static constexpr int TRIMS = SLOTS / 4 + 2;
  static constexpr int NODES = TREE_MAX_NODES, WORDS = TREE_ANC_WORDS;
};

// --- how the work is dealt out -----------------------------------------------------------------------------------
// (On the host, too: a CPU test walks through every block's run.)
// Tiles of a job of sequence b.
__host__ __device__ __forceinline__ int tree_tc_tiles(const TreeParams& p, int b) {
  return (tree_len(p, b) + TREE_TC_COLS - 1) / TREE_TC_COLS + (p.N + TREE_TC_COLS - 1) / TREE_TC_COLS;
}
// Tiles a group takes: an even share of all, but no fewer than `least`.
__host__ __device__ __forceinline__ long long tree_tc_share(long long total, int groups, int least) {
  const long long even = (total + groups - 1) / groups;
  return even > least ? even : least;
}

// A job that starts in one block's run and goes on in the following ones'.
struct TreeTcCut {
  int pieces, b, hk, rb, part;     // pieces (0: there is none such), the job, the index of the first piece
};

// Where a block is in its run.  Every role holds its own copy and steps through the same pieces.
struct TreeTcRun {
  long long at, end, base;      // next tile, end of the run, first tile of sequence b's jobs
  int b, tiles;                 // sequence, tiles of each of its jobs
  bool first;
  // the current piece
  int hk, rb, i0, i1, len, n_state, part;
  bool last;                    // has the job's last tile

  __host__ __device__ __forceinline__ bool next(const TreeParams& p, int block) {
    if (at >= end) return false;
    const int jobs = p.Hkv * p.row_rounds;        // of a sequence, for this block
    while (at >= base + (long long)tiles * jobs) {
      base += (long long)tiles * jobs;
      ++b;
      tiles = tree_tc_tiles(p, b);
    }
    const long long r = at - base;
    const int job = (int)(r / tiles);
    i0 = (int)(r - (long long)job * tiles);
    i1 = (int)min((long long)tiles, i0 + (end - at));
    hk = job / p.row_rounds;
    rb = (job - hk * p.row_rounds) * p.group + block % p.group;
    len = tree_len(p, b);
    n_state = (len + TREE_TC_COLS - 1) / TREE_TC_COLS;
    last = i1 == tiles;
    part = i0 == 0 && last ? -1 : 2 * block + (first ? 0 : 1);
    first = false;
    at += i1 - i0;
    return true;
  }
};

// Walks through a block's run; drafts(piece) is called for every piece that has drafts, until it returns false (a wait ran
// out).  The job that starts in the run and goes on in another, if there is one, is found all the same: its pieces hold NaN
// then, and must reach the result.
template <typename F>
__host__ __device__ __forceinline__ TreeTcCut tree_tc_walk(TreeTcRun run, const TreeParams& p, int block, F drafts) {
  TreeTcCut cut{};
  const long long share = run.end - run.at;              // (only the last block's may be shorter, and it cuts nothing)
  bool ok = true;
  while (run.next(p, block)) {
    if (run.i0 == 0 && !run.last) {
      const long long first_tile = run.at - run.i1;
      cut.pieces = (int)((first_tile + run.tiles - 1) / share) - block / p.group + 1;
      cut.b = run.b;
      cut.hk = run.hk;
      cut.rb = run.rb;
      cut.part = run.part;
    }
    if (ok && run.i1 > run.n_state) ok = drafts(run);
  }
  return cut;
}

// Four floats of shared memory as two pairs.  (Volatile: read again where they are needed again, instead of being kept in
// registers that the rows need.)
__device__ __forceinline__ void lds_f2x2(const float* x, uint64_t (&r)[2]) {
  asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(r[0]), "=l"(r[1]) : "r"(smem_addr(x)));
}

__device__ __forceinline__ void tma_load_2d_tile(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_addr(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(smem_addr(bar))
      : "memory");
}

__device__ __forceinline__ void tma_load_3d_tile(void* dst, const CUtensorMap* map, int x, int y, int z, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_addr(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_addr(bar))
      : "memory");
}

// 16 columns of this thread's TMEM lane times f (a power of two or 0: exact).
__device__ __forceinline__ void tree_tc_scale16(uint32_t taddr, float f) {
  uint32_t v[16];
  tmem_ld16(taddr, v);
#pragma unroll
  for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * f);
  tmem_st16(taddr, v);
}

// One arrival for a whole warp: an arrival is an atomic operation on shared memory, and 32 of them on one word take as long
// as a tile's worth of copies.
__device__ __forceinline__ void warp_arrive(uint64_t* bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}

template <int D, int FMT, int NT>
__global__ void __launch_bounds__(TreeTcShape<D, FMT, NT>::THREADS, 1)
    tova_tree_tc_kernel(const __grid_constant__ TreeParams p, const __grid_constant__ CUtensorMap map_k,
                        const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_q) {
  using S = TreeTcShape<D, FMT, NT>;
  constexpr bool PLAIN = S::PLAIN;
  constexpr int C = TREE_TC_COLS, R = TREE_TC_ROWS;
  constexpr int PRODUCER = S::SOFT_WARPS, ISSUER = PRODUCER + S::PRODUCER_WARPS, HELPER = ISSUER + 1, COPIER = HELPER + 1;      // first warp of each role
  constexpr int PT = 32 * S::PRODUCER_WARPS;
  extern __shared__ unsigned char tree_tc_raw[];
  unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(tree_tc_raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* q_s = smem;                               // per row tile: boxes of [128 rows][128 bytes]
  unsigned char* slot_s = q_s + NT * S::Q_BYTES;           // per slot: boxes of [128 rows][128 bytes]
  unsigned char* raw_s = slot_s + S::SLOTS * S::SLOT;
  float* scale_s = reinterpret_cast<float*>(raw_s + S::RAW_SLOTS * S::RAW);   // [tile % SCALE_TILES][k times the logits' scale, v, 1/v][128]
  __shared__ __align__(8) uint64_t full[S::SLOTS], empty[S::SLOTS], bar_sc[S::SCALE_TILES];
  __shared__ __align__(8) uint64_t raw_full[PLAIN ? 1 : S::RAW_SLOTS], raw_empty[PLAIN ? 1 : S::RAW_SLOTS];
  // Q landed, Q free again, S computed, weights written, O complete, (two S buffers) a tile's O += P V
  // complete, ancestor bits there, ancestor bits free again, the
  // two warps of 32 rows meet, a tile that has to be trimmed landed
  __shared__ __align__(8) uint64_t bar_q, bar_qf, bar_s[S::BUFFERS], bar_p[S::BUFFERS], bar_o[NT], bar_v, bar_a, bar_af, bar_pair[NT * 4], bar_trim[S::TRIMS];
  __shared__ uint32_t tmem_base_s;
  __shared__ int odd_s;                                    // some draft's value is not finite
  __shared__ TreeTcRun run_s, soft_run_s[S::SOFT_WARPS];   // (the soft-max warps' registers are for the rows)
  __shared__ __align__(16) uint32_t anc_s[S::NODES][S::WORDS];     // ancestor bits of every node
  __shared__ int par_s[S::NODES];
  __shared__ float pair_s[NT * R][2];                      // what the two threads of a row tell each other
  __shared__ int flag_s[NT * 4];

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int i = 0; i < S::SLOTS; ++i) {
      mbar_init(&full[i], S::PRODUCER_WARPS);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < S::RAW_SLOTS; ++i) {
      mbar_init(&raw_full[i], 1);
      mbar_init(&raw_empty[i], S::PRODUCER_WARPS);
    }
    mbar_init(&bar_q, S::PRODUCER_WARPS);
    for (int i = 0; i < S::TRIMS; ++i) mbar_init(&bar_trim[i], 1);
    mbar_init(&bar_qf, 1);
    for (int t = 0; t < S::BUFFERS; ++t) {
      mbar_init(&bar_s[t], 1);
      mbar_init(&bar_p[t], 2 * R / 32);
    }
    for (int t = 0; t < NT; ++t) mbar_init(&bar_o[t], 1);
    mbar_init(&bar_v, 1);
    for (int i = 0; i < S::SCALE_TILES; ++i) mbar_init(&bar_sc[i], S::PRODUCER_WARPS);
    mbar_init(&bar_a, 1);
    mbar_init(&bar_af, S::SOFT_WARPS);
    for (int i = 0; i < NT * 4; ++i) mbar_init(&bar_pair[i], 2);
    mbar_fence_init();
  }
  if (tid < NT * 4) flag_s[tid] = -1;
  if (warp == ISSUER) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base_s)), "r"(S::TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (warp == HELPER) {
    // The block's run: all tiles, its share of them, and the sequence that the share starts in.
    const int jobs = p.Hkv * p.row_rounds;
    TreeTcRun r;
    long long total;
    if (p.lens) {
      long long x = 0;
      for (int b = lane; b < p.B; b += 32) x += tree_tc_tiles(p, b);
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
      total = x * jobs;
    } else {
      total = (long long)tree_tc_tiles(p, 0) * jobs * p.B;
    }
    const long long share = tree_tc_share(total, gridDim.x / p.group, p.least);
    r.at = min(total, blockIdx.x / p.group * share);
    r.end = min(total, r.at + share);
    r.base = 0;
    r.b = 0;
    if (r.at < r.end) {
      if (p.lens) {
        for (int b0 = 0;; b0 += 32) {           // (r.at < total, so some sequence holds it)
          const long long mine = b0 + lane < p.B ? (long long)tree_tc_tiles(p, b0 + lane) * jobs : 0;
          long long upto = mine;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += y;
          }
          const unsigned hit = __ballot_sync(0xffffffffu, r.base + upto > r.at);
          if (hit) {
            const int x = __ffs(hit) - 1;
            r.b = b0 + x;
            r.base += __shfl_sync(0xffffffffu, upto - mine, x);
            break;
          }
          r.base += __shfl_sync(0xffffffffu, upto, 31);
        }
      } else {
        const long long per = (long long)tree_tc_tiles(p, 0) * jobs;
        r.b = (int)(r.at / per);
        r.base = per * r.b;
      }
      r.tiles = tree_tc_tiles(p, r.b);
    }
    r.first = true;
    if (lane == 0) run_s = r;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  TreeTcRun run = run_s;
  bool ok = true;
  // S of row tile t, tile g: its buffer, the buffer's columns, and the phase of the buffer's barriers.
  auto s_buf = [](int t, int g) { return S::DOUBLE ? g & 1 : t; };
  auto s_col = [&](int t, int g) { return tmem + 256 * s_buf(t, g); };
  auto s_phase = [](int g) { return (uint32_t)((S::DOUBLE ? g >> 1 : g) & 1); };
  // Copies are made and consumed in the order Q K0 V0 K1 V1 ...; the counters go on from piece to piece.  Tile g (of the
  // block's run) has K at ring position 2 g and V at 2 g + 1.

  if (warp >= PRODUCER && warp < ISSUER) {
    // ============================== producers ==============================
    const int pt = tid - PRODUCER * 32;
    // Where 16-byte chunk ch of row `row` lies in a slot.
    auto place = [&](int row, int ch) { return (ch >> 3) * (C * 128) + row * 128 + (((ch & 7) ^ (row & 7)) << 4); };
    constexpr int QCH = D / 8, QSTEP = PT / QCH;           // a thread's chunks: one column, every STEP-th row
    constexpr int CH = PLAIN ? D / 8 : D / 16, STEP = PT / CH, PER = C / STEP;
    int g0 = 0, piece = 0, raw0 = 0;                       // tiles, pieces, raw copies before this piece
    uint32_t trims = 0;
    while (ok && run.next(p, blockIdx.x)) {
      const int n = run.i1 - run.i0, bh = run.b * p.Hkv + run.hk;
      auto slot_free = [&](int pos) {
        return pos < S::SLOTS || mbar_wait_bounded(&empty[pos % S::SLOTS], (uint32_t)((pos / S::SLOTS - 1) & 1));
      };
      // Q rows, K-major with the 128-byte swizzle; rows past the product are zeros.  After the piece's first K and V, which
      // need not wait for the piece before to be done with its Q.
      auto load_q = [&]() {
        ok = piece == 0 || mbar_wait_bounded(&bar_qf, (uint32_t)((piece - 1) & 1));
        if (!ok) return;
        const int m0 = run.rb * (R * NT);
        if (p.q_tiled) {
          // (a node's G heads are neighbours: rows (node, head) are boxes of 128 / G nodes, and nodes behind the last zeros)
          if (pt == 0) {
            mbar_expect_tx(&bar_q, NT * S::Q_BYTES);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int c = 0; c < D / 64; ++c)
                tma_load_3d_tile(q_s + t * S::Q_BYTES + c * (R * 128), &map_q, c * 64, run.b * p.H + run.hk * p.G, (m0 + t * R) / p.G, &bar_q);
          } else if (lane == 0) {
            mbar_arrive(&bar_q);
          }
          return;
        }
        const int row_q = pt / QCH, ch = pt % QCH;
        const uint32_t dst = smem_addr(q_s) + (ch >> 3) * (R * 128);
#pragma unroll 8
        for (int k = 0; k < NT * R / QSTEP; ++k) {
          const int r = k * QSTEP + row_q, m = m0 + r, mm = min(m, p.M - 1);
          const int nd = mm / p.G, g = mm - nd * p.G;
          cp_async16(dst + (r / R) * S::Q_BYTES + (r % R) * 128 + (((ch & 7) ^ (r & 7)) << 4),
                     static_cast<const __nv_bfloat16*>(p.q) + (((long long)nd * p.B + run.b) * p.H + run.hk * p.G + g) * D + ch * 8, m < p.M ? 16u : 0u);
        }
        cp_async_commit();
        cp_async_wait<0>();
        fence_proxy_async_smem();
        warp_arrive(&bar_q, lane);
      };
      const unsigned char* src[2] = {static_cast<const unsigned char*>(p.K) + (long long)bh * p.cap * (PLAIN ? 2 * D : D),
                                     static_cast<const unsigned char*>(p.V) + (long long)bh * p.cap * (PLAIN ? 2 * D : D)};
      const int row_t = pt / CH, ch_t = pt % CH;           // this thread's chunks of a tile: one column, every STEP-th row
      auto draft = [&](int x) {                            // x: position within the piece
        const bool is_k = !(x & 1);
        const int pos = 2 * g0 + x;
        unsigned char* dst = slot_s + (pos % S::SLOTS) * S::SLOT;
        const __nv_bfloat16* from = static_cast<const __nv_bfloat16*>(is_k ? p.k_new : p.v_new);
        const int j0 = (run.i0 + x / 2 - run.n_state) * C;
        const int row_q = pt / QCH, ch = pt % QCH;
        const __nv_bfloat16* at = from + (((long long)j0 * p.B + run.b) * p.Hkv + run.hk) * D + ch * 8;
        constexpr int BATCH = C / QSTEP < 8 ? C / QSTEP : 8;     // loads in flight per thread
        static_assert(C % (BATCH * QSTEP) == 0, "the batches end with the tile");
        for (int k = 0; k < C / QSTEP; k += BATCH) {
          uint4 w[BATCH];
#pragma unroll
          for (int u = 0; u < BATCH; ++u) {
            const int row = (k + u) * QSTEP + row_q;
            w[u] = j0 + row < p.N ? *reinterpret_cast<const uint4*>(at + (long long)row * p.B * p.Hkv * D) : make_uint4(0, 0, 0, 0);
          }
#pragma unroll
          for (int u = 0; u < BATCH; ++u) {
            if (!is_k) tree_drop_odd(w[u]);
            *reinterpret_cast<uint4*>(dst + place((k + u) * QSTEP + row_q, ch)) = w[u];
          }
        }
        fence_proxy_async_smem();
        warp_arrive(&full[pos % S::SLOTS], lane);
      };
      if constexpr (PLAIN) {
        for (int x = 0; x < 2 * n && ok; ++x) {
          const int pos = 2 * g0 + x, tile = run.i0 + x / 2;
          ok = slot_free(pos);
          if (!ok) break;
          unsigned char* dst = slot_s + (pos % S::SLOTS) * S::SLOT;
          if (tile >= run.n_state) {
            draft(x);
          } else if (p.tiled) {
            // Rows behind the sequence's last come along: of K they give logits that are masked, of V they must be zeros.
            const int valid = run.len - tile * C;
            const bool trim = (x & 1) && valid < C;
            uint64_t* bar = trim ? &bar_trim[trims % S::TRIMS] : &full[pos % S::SLOTS];
            if (pt == 0) {
              const int y = bh * p.cap + tile * C;
              mbar_expect_tx(bar, S::SLOT);
#pragma unroll
              for (int c = 0; c < D / 64; ++c) tma_load_2d_tile(dst + c * (C * 128), (x & 1) ? &map_v : &map_k, c * 64, y, bar);
            }
            if (trim) {
              ok = mbar_wait_bounded(bar, (trims / S::TRIMS) & 1u);
              ++trims;
              if (!ok) break;
              for (int e = valid * QCH + pt; e < C * QCH; e += PT)
                *reinterpret_cast<uint4*>(dst + place(e / QCH, e % QCH)) = make_uint4(0, 0, 0, 0);
              fence_proxy_async_smem();
              warp_arrive(&full[pos % S::SLOTS], lane);
            } else if (pt != 0 && lane == 0) {
              mbar_arrive(&full[pos % S::SLOTS]);
            }
          } else {
            const unsigned char* from = ((x & 1) ? src[1] : src[0]) + ch_t * 16;
#pragma unroll 8
            for (int k = 0; k < PER; ++k) {
              const int row = k * STEP + row_t, j = tile * C + row;
              cp_async16(smem_addr(dst) + place(row, ch_t), from + (long long)min(j, run.len - 1) * (2 * D), j < run.len ? 16u : 0u);
            }
            cp_async_commit();
            cp_async_wait<0>();
            fence_proxy_async_smem();
            warp_arrive(&full[pos % S::SLOTS], lane);
          }
          if (x == 1) load_q();
        }
      } else {
        const int n_raw = 2 * max(0, min(run.i1, run.n_state) - run.i0);     // raw copies of this piece
        const int turn = D == 128 ? (ch_t >> 2) & 1 : row_t & 1;
        // Two scales a thread and tile (columns behind the sequence's last get finite, positive ones: a masked logit is
        // minus infinity), fetched a tile early and stored with the tile's K.
        float next_k, next_v;                    // (as loaded: a product with one would wait for it here)
        auto fetch_scales = [&](int tile) {
          const int j = tile * C + (pt & (C - 1));           // (of 256 threads two fetch the same)
          const bool in = tile < run.n_state && j < run.len;
          next_k = in ? p.k_scale[(long long)bh * p.cap + j] : 1.f;
          next_v = in ? p.v_scale[(long long)bh * p.cap + j] : 1.f;
        };
        fetch_scales(run.i0);
        for (int x = 0; x < 2 * n && ok; ++x) {
          const int pos = 2 * g0 + x, tile = run.i0 + x / 2, g = g0 + x / 2;
          ok = slot_free(pos);
          if (!ok) break;
          if (!(x & 1)) {
            float* sc = scale_s + (g % S::SCALE_TILES) * 3 * C;
            if (pt < C) {
              sc[pt] = p.scale2 * next_k;
              // Below 2^-100 (a row of zeros among them) weight times scale would leave the range of a bf16 and its
              // reciprocal that of a float: such a row's values count as codes times 2^-100, less than 6e-28.
              const float v = fabsf(next_v) < 0x1p-100f ? copysignf(0x1p-100f, next_v) : next_v;
              sc[C + pt] = v;
              sc[2 * C + pt] = 1.f / v;
            }
            warp_arrive(&bar_sc[g % S::SCALE_TILES], lane);
            fetch_scales(tile + 1);
          }
          if (tile >= run.n_state) {
            draft(x);
          } else {
            const int rp = raw0 + x, valid = run.len - tile * C;      // rows that were copied
            ok = mbar_wait_bounded(&raw_full[rp % S::RAW_SLOTS], (uint32_t)((rp / S::RAW_SLOTS) & 1));
            if (!ok) break;
            unsigned char* dst = slot_s + (pos % S::SLOTS) * S::SLOT;
            const unsigned char* raw = raw_s + (rp % S::RAW_SLOTS) * S::RAW + pt * 16;
            uint32_t nan = 0;                    // e4m3: NaN codes among this thread's
#pragma unroll 4
            for (int k = 0; k < PER; ++k) {
              const int row = k * STEP + row_t;
              const uint4 w = row < valid ? *reinterpret_cast<const uint4*>(raw + k * (PT * 16)) : make_uint4(0, 0, 0, 0);
              if (FMT == FORMAT_E4M3) nan = tree_nan_codes(w, nan);
              const uint4 lo = make_uint4(tree_codes2<FMT>(w.x, w.x, 0, 1), tree_codes2<FMT>(w.x, w.x, 2, 3),
                                          tree_codes2<FMT>(w.y, w.y, 0, 1), tree_codes2<FMT>(w.y, w.y, 2, 3));
              const uint4 hi = make_uint4(tree_codes2<FMT>(w.z, w.z, 0, 1), tree_codes2<FMT>(w.z, w.z, 2, 3),
                                          tree_codes2<FMT>(w.w, w.w, 0, 1), tree_codes2<FMT>(w.w, w.w, 2, 3));
              // (one half of a row's threads starts with its second chunk: eight of them then meet eight bank groups)
              *reinterpret_cast<uint4*>(dst + place(row, 2 * ch_t + turn)) = turn ? hi : lo;
              *reinterpret_cast<uint4*>(dst + place(row, 2 * ch_t + (turn ^ 1))) = turn ? lo : hi;
            }
            if (FMT == FORMAT_E4M3 && (nan & TREE_NAN_FOUND) != 0) {
#pragma unroll 1
              for (int k = 0; k < 2 * PER; ++k) {          // once more over what this thread has written
                uint4* at = reinterpret_cast<uint4*>(dst + place((k >> 1) * STEP + row_t, 2 * ch_t + (k & 1)));
                const uint4 w = *at;
                *at = make_uint4(tree_mark_nan(w.x), tree_mark_nan(w.y), tree_mark_nan(w.z), tree_mark_nan(w.w));
              }
            }
            fence_proxy_async_smem();          // for the tensor cores' reads, and for the next copy into the raw slot
            warp_arrive(&full[pos % S::SLOTS], lane);
            if (lane == 0) mbar_arrive(&raw_empty[rp % S::RAW_SLOTS]);
          }
          if (x == 1) load_q();
        }
        raw0 += n_raw;
      }
      g0 += n;
      ++piece;
    }
    // (TMA: where a wait ran out it took two seconds, and whatever was on its way has landed since.)
  } else if (warp == ISSUER) {
    // ============================== issuing thread ==============================
    if (lane == 0) {
      const uint32_t idesc_s = umma_idesc_bf16(R, C, false);
      const uint32_t idesc_o = umma_idesc_bf16(R, D, true);
      // A descriptor's low word holds the address in units of 16 bytes, so stepping through an operand is an addition to
      // that word.  (The tensor cores take a contraction every 64 cycles; forming each descriptor anew took this thread
      // longer than that, beside the soft-max warps that share its scheduler.)
      const uint64_t q_d = umma_desc_sw128(smem_addr(q_s), 16, 1024);
      const uint64_t k_d = umma_desc_sw128(smem_addr(slot_s), 16, 1024), v_d = umma_desc_sw128(smem_addr(slot_s), C * 128, 1024);
      auto at = [](uint64_t d, uint32_t bytes) { return (d & 0xffffffff00000000ull) | (uint32_t)((uint32_t)d + (bytes >> 4)); };
      // (What the producers wrote through the generic proxy they have fenced themselves, before they reported it: the fence
      // takes hundreds of cycles, which this thread does not have.)
      auto landed = [&](int pos) { return mbar_wait_bounded(&full[pos % S::SLOTS], (uint32_t)((pos / S::SLOTS) & 1)); };
      int g0 = 0, piece = 0;
      while (ok && run.next(p, blockIdx.x)) {
        const int n = run.i1 - run.i0;
        auto issue_s = [&](int t, int x) {
          const int pos = 2 * (g0 + x);
          const uint64_t k_t = at(k_d, (pos % S::SLOTS) * S::SLOT);
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
            umma_bf16(s_col(t, g0 + x), at(q_d, t * S::Q_BYTES + (ks >> 2) * (R * 128) + (ks & 3) * 32),
                      at(k_t, (ks >> 2) * (C * 128) + (ks & 3) * 32), idesc_s, ks > 0 ? 1u : 0u);
          umma_commit(&bar_s[s_buf(t, g0 + x)]);
          if (t == NT - 1) {
            umma_commit(&empty[pos % S::SLOTS]);
            if (x == n - 1) umma_commit(&bar_qf);
          }
        };
        ok = mbar_wait_bounded(&bar_q, (uint32_t)(piece & 1)) && landed(2 * g0);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int t = 0; t < NT; ++t) issue_s(t, 0);
        for (int x = 0; x < n && ok; ++x) {
          const int g = g0 + x, pos = 2 * g + 1;
          const uint64_t v_t = at(v_d, (pos % S::SLOTS) * S::SLOT);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            if (S::DOUBLE && x + 1 < n) {
              ok = landed(pos + 1);
              if (!ok) break;
              tc_fence_after();
              issue_s(t, x + 1);
            }
            if (t == 0) ok = landed(pos);
            ok = ok && mbar_wait_bounded(&bar_p[s_buf(t, g)], s_phase(g));
            if (!ok) break;
            tc_fence_after();
            // (the weights of columns 64.. lie 64 TMEM columns up: each half of a row overwrites its own logits only)
#pragma unroll
            for (int kk = 0; kk < C / 16; ++kk)
              umma_bf16_a_tmem(tmem + 256 * t + 128, s_col(t, g) + (kk >> 2) * 64 + (kk & 3) * 8,
                               at(v_t, kk * 2048), idesc_o, (x > 0 || kk > 0) ? 1u : 0u);
            if (t == NT - 1) umma_commit(&empty[pos % S::SLOTS]);
            if (S::DOUBLE) umma_commit(&bar_v);
            if (x + 1 == n) {
              umma_commit(&bar_o[t]);
            } else if (!S::DOUBLE) {
              if (t == 0) ok = landed(pos + 1);
              if (!ok) break;
              tc_fence_after();
              issue_s(t, x + 1);
            }
          }
        }
        g0 += n;
        ++piece;
      }
    }
  } else if (!PLAIN && warp == COPIER) {
    // ============================== copying thread ==============================
    if (lane == 0) {
      int raw0 = 0;                              // raw copies before this piece
      while (ok && run.next(p, blockIdx.x)) {
        const long long row0 = (long long)(run.b * p.Hkv + run.hk) * p.cap;
        const int n_raw = 2 * max(0, min(run.i1, run.n_state) - run.i0);
        for (int x = 0; x < n_raw && ok; ++x) {
          const int rp = raw0 + x, j = (run.i0 + x / 2) * C, slot = rp % max(1, S::RAW_SLOTS);
          if (rp >= S::RAW_SLOTS) ok = mbar_wait_bounded(&raw_empty[slot], (uint32_t)((rp / max(1, S::RAW_SLOTS) - 1) & 1));
          if (!ok) break;
          const uint32_t bytes = (uint32_t)min(C, run.len - j) * D;
          mbar_expect_tx(&raw_full[slot], bytes);
          bulk_g2s(raw_s + slot * S::RAW, static_cast<const unsigned char*>((x & 1) ? p.V : p.K) + (row0 + j) * D, bytes, &raw_full[slot]);
        }
        raw0 += n_raw;
      }
      // (Where a wait ran out it took two seconds, and whatever was on its way has landed since.)
    }
  } else if (warp == HELPER) {
    // ============================== helper warp ==============================
    int done = 0;                                          // pieces with drafts so far
    // (The list is for the second kernel.)
    const TreeTcCut cut = tree_tc_walk(run, p, blockIdx.x, [&](const TreeTcRun& r) {
      if (done > 0 && !warp_wait(&bar_af, (uint32_t)((done - 1) & 1))) return false;
      for (int i = lane; i < p.N; i += 32) par_s[i] = p.parents ? p.parents[(long long)i * p.B + r.b] : i - 1;
      __syncwarp();
      for (int i = lane; i < p.N; i += 32) tree_ancestor_bits<S::WORDS>(i, p.parents == nullptr, par_s, anc_s[i]);
      bool odd = false;
#pragma unroll 4
      for (int e = lane; e < p.N * (D / 8); e += 32) {
        uint4 w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.v_new) +
                                                  (((long long)(e / (D / 8)) * p.B + r.b) * p.Hkv + r.hk) * D + (e % (D / 8)) * 8);
        odd |= tree_drop_odd(w);
      }
      odd = __any_sync(0xffffffffu, odd) != 0;
      if (lane == 0) odd_s = odd;
      warp_arrive(&bar_a, lane);
      ++done;
      return true;
    });
    if (lane == 0) static_cast<TreeTcCut*>(p.cuts)[blockIdx.x] = cut;
  } else {
    // ============================== soft-max: two threads per row ==============================
    // Warps 0-3 of a row tile take the first 64 columns of its rows, warps 4-7 the others; a warp reaches the 32 TMEM
    // lanes of its quarter (warp mod 4).
    const int t = warp >> 3, half = (warp >> 2) & 1, quarter = warp & 3;
    const int pair = t * 4 + quarter, row = t * R + quarter * 32 + lane;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
    const uint32_t base = tmem + 256 * t + lanes;
    const uint64_t scale_2 = pack_f2(p.scale2, p.scale2);
    volatile TreeTcRun& mr = soft_run_s[warp];
    int g0 = 0, piece = 0, done = 0;
    uint32_t met = 0;                    // phase of the pair's barrier
    // The two warps that share 32 rows meet: what either wrote to shared memory before is there for both.
    auto meet = [&]() {
      warp_arrive(&bar_pair[pair], lane);
      ok = __all_sync(0xffffffffu, mbar_wait_bounded(&bar_pair[pair], met)) != 0;
      met ^= 1u;
    };
    if (lane == 0) soft_run_s[warp] = run;
    __syncwarp();
    for (;;) {
      int more = 0;
      __syncwarp();
      if (lane == 0) more = soft_run_s[warp].next(p, blockIdx.x);
      __syncwarp();
      if (!__shfl_sync(0xffffffffu, more, 0)) break;
      const int n = mr.i1 - mr.i0;
      const bool drafts = mr.i1 > mr.n_state;
      const int m = mr.rb * (R * NT) + row;
      const int node = m < p.M ? m / p.G : -1;
      const uint32_t* anc = anc_s[max(node, 0)];
      bool real = false, looked = false;         // a node's row, not padding's or one behind the product
      auto look = [&]() {                        // the drafts' ancestor bits, from the first time they are needed
        ok = __all_sync(0xffffffffu, ok && mbar_wait_bounded(&bar_a, (uint32_t)(done & 1))) != 0;
        looked = true;
        if (ok && node >= 0) {
#pragma unroll
          for (int k = 0; k < S::WORDS; ++k) real |= anc[k] != 0;
        }
      };
      float m_ref = -INFINITY, l = 0.f;
      for (int x = 0; x < n && ok; ++x) {
        const int i = mr.i0 + x, g = g0 + x;
        const float* sc = scale_s + (g % S::SCALE_TILES) * 3 * C + 64 * half;
        const uint32_t mine = s_col(t, g) + lanes + 64 * half;                  // this thread's logits, and its weights
        ok = mbar_wait_bounded(&bar_s[s_buf(t, g)], s_phase(g));
        if constexpr (!PLAIN) ok = ok && mbar_wait_bounded(&bar_sc[g % S::SCALE_TILES], (uint32_t)((g / S::SCALE_TILES) & 1));
        ok = __all_sync(0xffffffffu, ok) != 0;
        if (ok && i >= mr.n_state && !looked) look();
        if (!ok) break;
        tc_fence_after();
        const int left = i < mr.n_state ? mr.len - i * C - 64 * half : 64;      // this half's columns that exist
        const bool masked = i >= mr.n_state || left < 64;                       // the same for the whole warp
        uint32_t see[2] = {0xffffffffu, 0xffffffffu};
        if (masked) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (i >= mr.n_state) {
              const int w = 4 * (i - mr.n_state) + 2 * half + h;
              see[h] = real && w < S::WORDS ? anc[w] : 0u;
            } else {
              see[h] = left >= 32 * h + 32 ? 0xffffffffu : left > 32 * h ? (1u << (left - 32 * h)) - 1u : 0u;
            }
          }
        }
        uint32_t w[32];            // packed weights, two bf16 each
        float sum;
        auto logits = [&](int h, uint32_t (&s)[32]) {
          tmem_ld32_start(mine + 32 * h, s);
          tmem_ld32_wait(s);
          if (masked) {
#pragma unroll
            for (int c = 0; c < 32; ++c) s[c] = ((see[h] >> c) & 1u) ? s[c] : 0xff800000u;
          }
        };
        auto weights = [&]() {
          const float ref = m_ref == -INFINITY ? 0.f : m_ref;
          const uint64_t mneg_2 = pack_f2(-ref, -ref);
          uint64_t sum2[2] = {pack_f2(0.f, 0.f), pack_f2(0.f, 0.f)};
          uint64_t kf[2] = {scale_2, scale_2}, vf[2], rf[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t s[32];
            logits(h, s);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              if constexpr (!PLAIN)
                if (e % 2 == 0) {
                  lds_f2x2(sc + 32 * h + 2 * e, kf);         // the logits' scale is in there
                  lds_f2x2(sc + C + 32 * h + 2 * e, vf);
                  lds_f2x2(sc + 2 * C + 32 * h + 2 * e, rf);
                }
              float x0, x1, e0, e1;
              unpack_f2(fma_f2(pack_f2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), kf[e & 1], mneg_2), x0, x1);
              e0 = ex2_approx(x0);
              e1 = ex2_approx(x1);
              if constexpr (PLAIN) {
                const uint32_t u = pack_bf16(e0, e1);
                sum2[e & 1] = add_f2(sum2[e & 1], pack_f2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)));
                w[16 * h + e] = u;
              } else {
                // The value scale goes into the weight before it is rounded, and out of the sum again: as above the sum
                // is over the weights as they are used (0.0019 from the exact result where 0.0024 without; 3 % of the time).
                unpack_f2(mul_f2(pack_f2(e0, e1), vf[e & 1]), e0, e1);
                const uint32_t u = pack_bf16(e0, e1);
                sum2[e & 1] = fma_f2(pack_f2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)), rf[e & 1], sum2[e & 1]);
                w[16 * h + e] = u;
              }
            }
          }
          float s0, s1;
          unpack_f2(add_f2(sum2[0], sum2[1]), s0, s1);
          sum = s0 + s1;
        };
        bool over = x == 0;              // the reference has to be found or moved
        if (x > 0) {
          weights();
          // Both threads of a row have to agree on its reference: the pair of warps meets, and a row of either whose sum
          // is too large (or not a number) sends both round again.
          if (__any_sync(0xffffffffu, !(sum <= TREE_TC_MOST) || m_ref == -INFINITY)) flag_s[pair] = g;
          meet();
          if (!ok) break;
          over = *reinterpret_cast<volatile int*>(&flag_s[pair]) == g;
        }
        if (over) {
          float top = -INFINITY;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t s[32];
            logits(h, s);
#pragma unroll
            for (int c = 0; c < 32; ++c) top = fmaxf(top, __uint_as_float(s[c]) * (PLAIN ? p.scale2 : sc[32 * h + c]));
          }
          pair_s[row][half] = top;
          meet();
          if (!ok) break;
          top = fmaxf(top, pair_s[row][half ^ 1]);
          // (a reference that is right already stays: another row of the warp asked)
          const bool beyond = top > m_ref + 16.f || (m_ref == -INFINITY && top > -INFINITY);
          const float m_new = beyond ? ceilf(top) : m_ref;
          const float corr = beyond ? ex2_approx(m_ref - m_new) : 1.f;       // a power of two, or 0
          m_ref = m_new;
          l *= corr;
          if (x > 0) {
            // O of the tiles so far, half the columns a thread.  (The last of them is complete where S of this tile was
            // issued behind it.)
            if (S::DOUBLE) {
              ok = __all_sync(0xffffffffu, mbar_wait_bounded(&bar_v, (uint32_t)((g - 1) & 1))) != 0;
              if (!ok) break;
              tc_fence_after();
            }
#pragma unroll
            for (int c = 0; c < D / 2; c += 16) tree_tc_scale16(base + 128 + half * (D / 2) + c, corr);
          }
          weights();
          meet();                                  // (pair_s may be written again)
          if (!ok) break;
        }
        l += sum;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t (&wh)[16] = *reinterpret_cast<uint32_t (*)[16]>(&w[16 * h]);
          tmem_st16(mine + 16 * h, wh);                                      // over logits that have been read
        }
        tmem_st_wait();
        tc_fence_before();
        warp_arrive(&bar_p[s_buf(t, g)], lane);
      }
      if (drafts && ok && !looked) look();
      if (ok) {
        ok = __all_sync(0xffffffffu, mbar_wait_bounded(&bar_o[t], (uint32_t)(piece & 1))) != 0;
        tc_fence_after();
      }
      // The row's sum: both halves'.
      if (ok) {
        pair_s[row][half] = l;
        meet();
        l += pair_s[row][half ^ 1];
        if (ok) meet();
      }
      if (mr.last && !real) l = TREE_PADDING;
      if (!ok) l = __uint_as_float(0x7fc00000u);
      const bool zero = l == TREE_PADDING;
      const float r = mr.part >= 0 ? 1.f : 1.f / l;
      const long long at = (long long)mr.part * (R * NT) + row;
      if (mr.part >= 0 && half == 0) p.part_ml[at] = make_float2(m_ref, l);
      const int gq = max(node, 0);
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) +
                           (((long long)gq * p.B + mr.b) * p.H + mr.hk * p.G + (max(m, 0) - gq * p.G)) * D + half * (D / 2);
      float* acc = p.part_acc + at * D + half * (D / 2);
#pragma unroll
      for (int c = 0; c < D / 2; c += 32) {
        float o[32];
        if (ok) {
          tmem_ld32(base + 128 + half * (D / 2) + c, o);
        } else {
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] = __uint_as_float(0x7fc00000u);
        }
        if (drafts && odd_s && real && ok) tree_add_odd<S::WORDS, 32>(p, mr.b, mr.hk, anc, D, half * (D / 2) + c, o);
        if (zero) {
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] = 0.f;
        }
        if (node >= 0 && mr.part < 0) {
#pragma unroll
          for (int k = 0; k < 32; k += 8)
            *reinterpret_cast<uint4*>(out + c + k) = make_uint4(pack_bf16(o[k] * r, o[k + 1] * r), pack_bf16(o[k + 2] * r, o[k + 3] * r),
                                                                pack_bf16(o[k + 4] * r, o[k + 5] * r), pack_bf16(o[k + 6] * r, o[k + 7] * r));
        } else if (mr.part >= 0) {
#pragma unroll
          for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(acc + c + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
        }
        __syncwarp();
      }
      tc_fence_before();                 // O has been read: the next piece's first weights are reported behind this
      if (drafts) {
        warp_arrive(&bar_af, lane);
        ++done;
      }
      g0 += n;
      ++piece;
    }
  }
  pdl_launch_dependents();
  tc_fence_before();
  __syncthreads();
  if (warp == ISSUER)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::TMEM_COLS) : "memory");
}

// Joins the pieces of the jobs that were cut, one warp per row.  grid = (blocks of the first kernel, rows of a job / 8).
constexpr int TREE_TC_JOIN_THREADS = 256;
template <int D, int NT>
__global__ void __launch_bounds__(TREE_TC_JOIN_THREADS) tova_tree_tc_join_kernel(const __grid_constant__ TreeParams p) {
  constexpr int ROWS = TREE_TC_ROWS * NT, E = D / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = blockIdx.y * (TREE_TC_JOIN_THREADS / 32) + warp;
  pdl_wait();
  const TreeTcCut cut = static_cast<const TreeTcCut*>(p.cuts)[blockIdx.x];
  const int m = cut.rb * ROWS + r;
  if (cut.pieces == 0 || m >= p.M) return;
  // The pieces behind the first are the first ones of the blocks that follow, group by group.
  auto part_row = [&](int c) { return (long long)(c == 0 ? cut.part : 2 * ((int)blockIdx.x + c * p.group)) * ROWS + r; };
  const int c0 = 0, c1 = cut.pieces - 1, b = cut.b, hk = cut.hk;
  float top = -INFINITY;
  bool pad = false;
  for (int c = c0 + lane; c <= c1; c += 32) {
    const float2 ml = p.part_ml[part_row(c)];
    top = fmaxf(top, ml.x);
    if (c == c1) pad = ml.y == TREE_PADDING;
  }
  top = warp_max(top);
  pad = __any_sync(0xffffffffu, pad) != 0;
  const float base = top == -INFINITY ? 0.f : top;
  float acc[E], l = 0.f;
#pragma unroll
  for (int j = 0; j < E; ++j) acc[j] = 0.f;
  for (int cc = c0; cc <= c1; cc += 32) {
    float f = 0.f;                 // this lane's piece: its factor, and its share of the sum
    if (cc + lane <= c1) {
      const float2 ml = p.part_ml[part_row(cc + lane)];
      f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - base);
      if (f != 0.f) l += f * ml.y;
    }
    const int n = min(32, c1 - cc + 1);
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const float fi = __shfl_sync(0xffffffffu, f, i);
      const float* a = p.part_acc + part_row(cc + i) * D + lane * E;
#pragma unroll
      for (int j = 0; j < E; ++j) acc[j] = fmaf(fi, a[j], acc[j]);
    }
  }
  l = warp_sum(l);
  const float inv = 1.f / l;
  const int n = m / p.G, g = m - n * p.G;
  __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(p.out) + (((long long)n * p.B + b) * p.H + hk * p.G + g) * D + lane * E;
#pragma unroll
  for (int j = 0; j < E; ++j) dst[j] = (__nv_bfloat16)(pad ? 0.f : acc[j] * inv);
}

}  // namespace tova
