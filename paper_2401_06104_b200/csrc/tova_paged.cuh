// A state kept in pages: rows written to it, and attention of one new token over it (sm_100a).
//
// Pages are small states [Hkv, rows, D] of a pool; a sequence's row j lies in page table[b][j / rows] at row j mod rows.  So
// sequences of any length share the pool, and nothing has a capacity but the table.  rows is a power of two.
#pragma once

#include "tova_mma.cuh"
#include "tova_tc.cuh"

namespace tova {

// ---------------------------------------------------------------------------------------------------------------------
// Rows into pages: token i of the packed rows belongs to the sequence b with offsets[b] <= i < offsets[b + 1] (one token a
// sequence where there are no offsets) and becomes its row first[b] + i - offsets[b].  DRAM bound; a block takes a few tokens,
// whose rows are on their way before their places have been looked up.  Measured (GPU time, in a captured graph): 20,342 tokens of
// 8 heads x 128 in bf16 (167 MB) 29.1 us, 5.7 TB/s, 0.87 of the copy rate, in fp32 56.8 us, 0.89 (bf16: 34 with divisions by run-time
// sizes, 33 with 16 tokens a block); 64 tokens 2.3 us.
constexpr int PAGED_WRITE_THREADS = 256;
constexpr int PAGED_WRITE_TOKENS = 4;

struct PagedWriteParams {
  const void* x[2];             // k, v rows [N, Hkv * D]
  void* y[2];                   // pages
  long long x_stride[2];        // in vectors of 16 bytes
  const int32_t *table, *first, *offsets;
  long long max_rows;           // max_pages * page_rows
  int S, N, Hkv, n_pages, max_pages, shift, tokens_per_block;
  int vec_shift;                // log2 of the vectors a head row
  unsigned magic;               // ceil(2^32 / (vectors of a token's row)), or 0: too many for it to divide exactly
};

// The sequence that packed token i, 0 <= i < N, belongs to (the last b with offsets[b] <= i, looked for by a whole warp, 32 places at
// a time) and its first token; -1 where there is none, or i lies behind the sequence's end.  Offsets outside 0..N are the nearest of
// them, as in packed attention.
__device__ __forceinline__ int packed_sequence(const int32_t* offsets, int S, int i, int lane, int& first) {
  int lo = 0, hi = S;                      // offsets[lo] <= i (if any), the answer lies in lo .. hi - 1
  for (;;) {
    const int step = (hi - lo + 31) / 32;
    const int at = lo + lane * step;
    const unsigned m = __ballot_sync(0xffffffffu, at < hi && offsets[at] <= i);
    if (m == 0) return -1;
    lo += (31 - __clz(m)) * step;
    hi = min(hi, lo + step);
    if (step == 1) break;
  }
  first = max(offsets[lo], 0);             // (no more than i; the end's bound is above i)
  return i < offsets[lo + 1] ? lo : -1;
}

__global__ void __launch_bounds__(PAGED_WRITE_THREADS) tova_paged_write_kernel(const __grid_constant__ PagedWriteParams p) {
  __shared__ long long place[PAGED_WRITE_TOKENS];          // first vector of the row in head 0 of its page, or -1
  constexpr int U = 4;
  const int i0 = blockIdx.x * p.tokens_per_block, n_tok = min(p.tokens_per_block, p.N - i0);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int per_row = p.Hkv << p.vec_shift, total = n_tok * 2 * per_row;
  for (int e0 = threadIdx.x; e0 < total + (int)threadIdx.x; e0 += U * PAGED_WRITE_THREADS) {
    uint4 w[U];
    int tok[U], kv[U], at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int e = e0 + u * PAGED_WRITE_THREADS;
      tok[u] = -1;
      if (e >= total) continue;
      const int r = p.magic ? (int)__umulhi((unsigned)e, p.magic) : e / per_row;      // (a division costs more than the rest)
      at[u] = e - r * per_row;
      tok[u] = r >> 1;
      kv[u] = r & 1;
      w[u] = __ldcs(static_cast<const uint4*>(p.x[kv[u]]) + (long long)(i0 + tok[u]) * p.x_stride[kv[u]] + at[u]);
    }
    if (e0 == (int)threadIdx.x) {
      for (int t = warp; t < n_tok; t += PAGED_WRITE_THREADS / 32) {
        const int i = i0 + t;
        int first = i;
        const int b = p.offsets ? packed_sequence(p.offsets, p.S, i, lane, first) : i;
        long long to = -1;
        if (b >= 0) {
          const long long j = (long long)(p.first ? p.first[b] : 0) + (i - first);
          if (j >= 0 && j < p.max_rows) {
            const int page = p.table[(long long)b * p.max_pages + (j >> p.shift)];
            if (page >= 0 && page < p.n_pages)
              to = ((((long long)page * p.Hkv) << p.shift) + (j & ((1 << p.shift) - 1))) << p.vec_shift;
          }
        }
        if (lane == 0) place[t] = to;
      }
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (tok[u] < 0 || place[tok[u]] < 0) continue;
      const int h = at[u] >> p.vec_shift;
      static_cast<uint4*>(p.y[kv[u]])[place[tok[u]] + ((((long long)h << p.shift) - h) << p.vec_shift) + at[u]] = w[u];
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Attention of one new token: o[h] = sum_j softmax_j(scale q[h] K[j]) V[j] over the len[b] rows of a sequence; nothing is
// written but the result.  Every row is used by the G query heads that share its KV head: 2 G flops a byte (bf16), DRAM bound.
//
// A block of four warps takes up to HEADS query heads of one KV head of one sequence and walks through rows in units of 64, 16
// a warp.  Nothing goes through shared memory on the way: a lane fetches 16-byte pieces of rows into registers, where they are
// operands of the warp's matrix instructions as they lie (bf16), or of its multiply-adds (fp32), and asks for the next tile's
// as soon as an operand is consumed.  What a warp has summed meets the other warps' in shared memory at the end.
//
// How the rows are dealt out.  RUNS: the units of all (sequence, KV head, head group) jobs, one behind the other, in even shares
// to as many blocks as are resident at a time, so that lengths that differ cost no idle time; a job cut by the end of a share
// leaves its parts in the workspace, and a second kernel joins them.  CLUSTER (few rows, where two launches would cost more than
// the rows): up to eight blocks share a job and join through distributed shared memory.
//
// A row behind the sequence's last, or in a page that is none of the pool's, is not read and has no weight.  A sequence without
// rows gives zeros.
//
// Measured (GPU time, in a captured graph), bf16, 32 query over 8 KV heads x 128, pages of 16 rows: 64 sequences of up to 8192 rows
// (1.4 GB) 224 us, 6.3 TB/s, 0.96 of the copy rate; 16 x 4000 47 us (0.85), 64 x 500 34 us (0.60), 1 x 32000 32 us (0.63), 1 x 1000
// 7 us: a call has about 7 us that do not shrink, and a warp's tile takes 1 us with 8 KB on their way.  fp32, MHA: 8 x up to 2001
// rows 57 us (0.83).  Pieces through shared memory instead of registers (16-byte asynchronous copies, two or three tiles ahead): the
// long ones 1.3 times as long, the short ones as they are; 128 registers and 16 warps an SM: 1.3 times, spills.
constexpr int PAGED_WARPS = 4, PAGED_THREADS = 32 * PAGED_WARPS, PAGED_UNIT = 16 * PAGED_WARPS;
constexpr float PAGED_NOTHING = -1.f;      // the sum that stands for "no row seen"

struct PagedCut {
  int pieces, block, part;                 // pieces of a job (0: it was not cut), the block that its first lies in, that one's place
};

struct PagedParams {
  const void* q;                           // [B,H,D]
  const void *K, *V;                       // [pages,Hkv,rows,D]
  const int32_t *table, *lens;
  void* out;                               // [B,H,D]
  float2* part_ml;                         // [2 * blocks][HEADS]
  float* part_acc;                         // [2 * blocks][HEADS][D]
  PagedCut* cuts;                          // [B * jobs]
  long long q_stride;
  int B, H, Hkv, G, hgroups, jobs;         // jobs of a sequence: Hkv * hgroups
  int n_pages, max_pages, shift, n_live, least;
  float scale2;                            // scale * log2(e)
};

__device__ __forceinline__ int paged_len(const PagedParams& p, int b) { return max(0, min(p.lens[b], p.n_live)); }
__device__ __forceinline__ int paged_units(const PagedParams& p, int b) { return max(1, (paged_len(p, b) + PAGED_UNIT - 1) / PAGED_UNIT); }
// The page that holds row j, or -1.
__device__ __forceinline__ int paged_page(const PagedParams& p, const int32_t* table, int j, int end) {
  int page = -1;
  if (j < end) page = __ldg(table + (j >> p.shift));
  return page < p.n_pages ? page : -1;
}

__device__ __forceinline__ uint4 ldg_stream(const void* x) {
  uint4 w;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "l"(x));
  return w;
}

// bf16.  S^T[rows, heads] = K q^T and O^T[D, heads] += V^T P^T as m16n8k16 products: 16 rows, 8 heads.  The contraction index of
// the first is permuted so that a lane's eight neighbouring components of a row are two products' operands; the rows of O^T so
// that its eight of a value row are eight products' (pairs of rows are interleaved by one byte permutation a pair).  The weights
// come from the accumulator's layout by 8 x 8 transposes, as two bf16 terms each (16 significant bits): their rounding is far
// below the result's.  A row's reference stays where it is while no logit is beyond it by more than 16 (2^16 times a weight of 1
// loses nothing in floating point).
template <int D_, int NT, bool SMALL>
struct PagedMma {
  using T = __nv_bfloat16;
  static constexpr int D = D_, HEADS = 8 * NT, MIN_BLOCKS = NT == 1 ? 3 : 2;
  static constexpr int KS = D / 32, VC = D / 64, OT = D / 16;

  // Sums over rows r0 .. r1 - 1 of this warp; acc [HEADS][D], ml [HEADS].
  __device__ static void run(const PagedParams& p, int b, int hk, int hg, int r0, int r1, float* acc, float2* ml) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    uint32_t qf[NT][KS][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int head = hg * HEADS + n * 8 + g;
        uint4 w = make_uint4(0, 0, 0, 0);
        if (head < p.G) w = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.q) + b * p.q_stride + (long long)(hk * p.G + head) * D + (4 * s + t) * 8);
        qf[n][s][0] = w.x; qf[n][s][1] = w.y; qf[n][s][2] = w.z; qf[n][s][3] = w.w;
      }
    float o[NT][OT][4], l[NT][2], ref[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int j = 0; j < OT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][j][e] = 0.f;
      l[n][0] = l[n][1] = 0.f;
      ref[n][0] = ref[n][1] = -INFINITY;
    }
    const int32_t* table = p.table + (long long)b * p.max_pages;
    const T* Kp = static_cast<const T*>(p.K);
    const T* Vp = static_cast<const T*>(p.V);
    const int in_page = (1 << p.shift) - 1;
    // Page (SMALL: of row lane mod 16) and the rows that count (one bit each) of the tile that starts at row j0.
    auto look = [&](int j0, int& page) {
      page = paged_page(p, table, SMALL ? j0 + (lane & 15) : j0, r1);
    };
    auto rows_of = [&](int j0, int page) -> uint32_t {
      if (SMALL) return __ballot_sync(0xffffffffu, page >= 0) & 0xffffu;
      const int left = r1 - j0;
      return page < 0 ? 0u : left >= 16 ? 0xffffu : (1u << left) - 1u;
    };
    auto row_at = [&](const T* base, int j0, int page, int r) -> const T* {
      const int pg = SMALL ? __shfl_sync(0xffffffffu, page, r) : page;
      return base + ((((long long)pg * p.Hkv + hk) << p.shift) + ((j0 + r) & in_page)) * D;
    };
    uint4 kr[2][KS], vr[4][VC];
    auto load_k = [&](int j0, int page, uint32_t rows) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = g + 8 * x;
        const T* at = row_at(Kp, j0, page, r);
#pragma unroll
        for (int s = 0; s < KS; ++s) kr[x][s] = (rows >> r) & 1u ? ldg_stream(at + (4 * s + t) * 8) : make_uint4(0, 0, 0, 0);
      }
    };
    auto load_v = [&](int j0, int page, uint32_t rows) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int r = 2 * t + (x & 1) + 8 * (x >> 1);
        const T* at = row_at(Vp, j0, page, r);
#pragma unroll
        for (int c = 0; c < VC; ++c) vr[x][c] = (rows >> r) & 1u ? ldg_stream(at + c * 64 + g * 8) : make_uint4(0, 0, 0, 0);
      }
    };
    bool seen = false;
    int j0 = r0 + 16 * warp, page, next_page;
    look(j0, page);
    uint32_t rows = rows_of(j0, page);
    load_k(j0, page, rows);
    load_v(j0, page, rows);
    look(j0 + PAGED_UNIT, next_page);
    for (; j0 < r1; j0 += PAGED_UNIT) {
      const uint32_t next_rows = rows_of(j0 + PAGED_UNIT, next_page);
      float s[NT][4], chain[4][NT][4];                   // (four chains of products)
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int n = 0; n < NT; ++n) chain[y][n][0] = chain[y][n][1] = chain[y][n][2] = chain[y][n][3] = 0.f;
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        const uint32_t a0[4] = {kr[0][x].x, kr[1][x].x, kr[0][x].y, kr[1][x].y};
        const uint32_t a1[4] = {kr[0][x].z, kr[1][x].z, kr[0][x].w, kr[1][x].w};
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_bf16(chain[(2 * x) & 3][n], a0, qf[n][x][0], qf[n][x][1]);
          mma_bf16(chain[(2 * x + 1) & 3][n], a1, qf[n][x][2], qf[n][x][3]);
        }
      }
      load_k(j0 + PAGED_UNIT, next_page, next_rows);
      seen |= rows != 0;
      const bool in0 = (rows >> g) & 1u, in1 = (rows >> (g + 8)) & 1u;
      bool beyond = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[n][e] = (chain[0][n][e] + chain[1][n][e]) + (chain[2][n][e] + chain[3][n][e]);
          s[n][e] = (e < 2 ? in0 : in1) ? s[n][e] * p.scale2 : -INFINITY;
          beyond |= s[n][e] > ref[n][e & 1] + 16.f;
        }
      if (__any_sync(0xffffffffu, beyond)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float top = fmaxf(s[n][e], s[n][e + 2]);
#pragma unroll
            for (int x = 4; x <= 16; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
            top = fmaxf(top, ref[n][e]);
            const float f = ref[n][e] == -INFINITY ? 0.f : ex2_approx(ref[n][e] - top);
            ref[n][e] = top;
            l[n][e] *= f;
#pragma unroll
            for (int j = 0; j < OT; ++j) {
              o[n][j][e] *= f;
              o[n][j][e + 2] *= f;
            }
          }
      }
      uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] = ex2_approx(s[n][e] - (ref[n][e & 1] == -INFINITY ? 0.f : ref[n][e & 1]));
          l[n][e & 1] += w[e];
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const __nv_bfloat162 h = __floats2bfloat162_rn(w[2 * x], w[2 * x + 1]);
          const uint32_t u = *reinterpret_cast<const uint32_t*>(&h);
          const __nv_bfloat162 r = __floats2bfloat162_rn(w[2 * x] - __uint_as_float(u << 16), w[2 * x + 1] - __uint_as_float(u & 0xffff0000u));
          hi[n][x] = movmatrix_trans(u);
          lo[n][x] = movmatrix_trans(*reinterpret_cast<const uint32_t*>(&r));
        }
      }
#pragma unroll
      for (int j = 0; j < OT; ++j) {
        // D = 128: rows g and g + 8 of the product are components 8 g + j and 64 + 8 g + j; D = 64: 8 g + 2 j and the next.
        uint32_t a[4];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int c = VC == 2 ? x : 0, el = VC == 2 ? j : 2 * j + x;
          auto word = [&](const uint4& v) { return (el >> 1) == 0 ? v.x : (el >> 1) == 1 ? v.y : (el >> 1) == 2 ? v.z : v.w; };
          const uint32_t pick = el & 1 ? 0x7632u : 0x5410u;
          a[x] = __byte_perm(word(vr[0][c]), word(vr[1][c]), pick);
          a[2 + x] = __byte_perm(word(vr[2][c]), word(vr[3][c]), pick);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_bf16(o[n][j], a, hi[n][0], hi[n][1]);
          mma_bf16(o[n][j], a, lo[n][0], lo[n][1]);
        }
      }
      load_v(j0 + PAGED_UNIT, next_page, next_rows);
      page = next_page;
      rows = next_rows;
      look(j0 + 2 * PAGED_UNIT, next_page);
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x <= 16; x <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], x);
        const int head = n * 8 + 2 * t + e;
        if (g == 0) ml[head] = make_float2(ref[n][e], seen ? l[n][e] : PAGED_NOTHING);
        float* to = acc + head * D + g * 8;
#pragma unroll
        for (int c = 0; c < VC; ++c)
#pragma unroll
          for (int x = 0; x < 8; x += 4) {
            float f[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) f[y] = VC == 2 ? o[n][x + y][2 * c + e] : o[n][(x + y) / 2][2 * (y & 1) + e];
            *reinterpret_cast<float4*>(to + c * 64 + x) = make_float4(f[0], f[1], f[2], f[3]);
          }
      }
  }
};

// fp32, every product in fp32: D / 16 lanes a row, 16 components each, so 64 / D * 8 rows at a time, each group of lanes with a
// maximum, a sum and a weighted sum of its own.
template <int D_, int GU>
struct PagedAlu {
  using T = float;
  static constexpr int D = D_, HEADS = GU, MIN_BLOCKS = GU == 4 ? 2 : 3;
  static constexpr int LANES = D / 16, AT = 32 / LANES, R = GU == 4 ? 1 : 2;       // rows at a time, of them R in flight

  __device__ static void run(const PagedParams& p, int b, int hk, int hg, int r0, int r1, float* acc, float2* ml) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gr = lane / LANES, lr = lane % LANES;
    float q[GU][16], o[GU][16], l[GU], m[GU];
#pragma unroll
    for (int h = 0; h < GU; ++h) {
      const int head = hg * GU + h;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
        if (head < p.G) w = *reinterpret_cast<const float4*>(static_cast<const float*>(p.q) + b * p.q_stride + (long long)(hk * p.G + head) * D + (i * LANES + lr) * 4);
        q[h][4 * i] = w.x; q[h][4 * i + 1] = w.y; q[h][4 * i + 2] = w.z; q[h][4 * i + 3] = w.w;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) o[h][i] = 0.f;
      l[h] = 0.f;
      m[h] = -INFINITY;
    }
    const int32_t* table = p.table + (long long)b * p.max_pages;
    const int in_page = (1 << p.shift) - 1;
    // A warp's rows: 16 of every unit, R * AT at a time.
    constexpr int STEP = R * AT, STEPS = 16 / STEP;
    static_assert(16 % STEP == 0, "a warp's share of a unit is whole steps");
    auto row_of = [&](int i, int k) { return r0 + (i / STEPS) * PAGED_UNIT + warp * 16 + (i % STEPS) * STEP + k * AT + gr; };
    bool seen = false;
    int page[R];
#pragma unroll
    for (int k = 0; k < R; ++k) page[k] = paged_page(p, table, row_of(0, k), r1);
    const int n = (r1 - r0 + PAGED_UNIT - 1) / PAGED_UNIT * STEPS;
    for (int i = 0; i < n; ++i) {
      uint4 kr[R][4], vr[R][4];
      bool in[R];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        in[k] = page[k] >= 0;
        const long long at = ((((long long)max(page[k], 0) * p.Hkv + hk) << p.shift) + (row_of(i, k) & in_page)) * D + lr * 4;
#pragma unroll
        for (int x = 0; x < 4; ++x) kr[k][x] = in[k] ? ldg_stream(static_cast<const float*>(p.K) + at + x * LANES * 4) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int x = 0; x < 4; ++x) vr[k][x] = in[k] ? ldg_stream(static_cast<const float*>(p.V) + at + x * LANES * 4) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int k = 0; k < R; ++k) page[k] = i + 1 < n ? paged_page(p, table, row_of(i + 1, k), r1) : -1;
#pragma unroll
      for (int h = 0; h < GU; ++h) {
        float s[R], top = m[h];
#pragma unroll
        for (int k = 0; k < R; ++k) {
          float x = 0.f;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            x = fmaf(q[h][4 * c], __uint_as_float(kr[k][c].x), x);
            x = fmaf(q[h][4 * c + 1], __uint_as_float(kr[k][c].y), x);
            x = fmaf(q[h][4 * c + 2], __uint_as_float(kr[k][c].z), x);
            x = fmaf(q[h][4 * c + 3], __uint_as_float(kr[k][c].w), x);
          }
#pragma unroll
          for (int y = LANES / 2; y >= 1; y >>= 1) x += __shfl_xor_sync(0xffffffffu, x, y);
          s[k] = in[k] ? x * p.scale2 : -INFINITY;
          top = fmaxf(top, s[k]);
        }
        const float base = top == -INFINITY ? 0.f : top;
        const float f = m[h] == -INFINITY ? 0.f : exp2f(m[h] - base);
        m[h] = top;
        float w[R];
        l[h] *= f;
#pragma unroll
        for (int k = 0; k < R; ++k) {
          w[k] = exp2f(s[k] - base);
          l[h] += w[k];
        }
#pragma unroll
        for (int c = 0; c < 16; ++c) {
          float x = o[h][c] * f;
#pragma unroll
          for (int k = 0; k < R; ++k) {
            const uint4& v = vr[k][c >> 2];
            x = fmaf(w[k], __uint_as_float((c & 3) == 0 ? v.x : (c & 3) == 1 ? v.y : (c & 3) == 2 ? v.z : v.w), x);
          }
          o[h][c] = x;
        }
      }
#pragma unroll
      for (int k = 0; k < R; ++k) seen |= in[k];
    }
    seen = __any_sync(0xffffffffu, seen) != 0;
    // The groups of the warp.
#pragma unroll
    for (int h = 0; h < GU; ++h) {
      float top = m[h];
#pragma unroll
      for (int x = LANES; x <= 16; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      const float f = m[h] == -INFINITY ? (m[h] == top ? 1.f : 0.f) : exp2f(m[h] - top);
      l[h] *= f;
#pragma unroll
      for (int x = LANES; x <= 16; x <<= 1) l[h] += __shfl_xor_sync(0xffffffffu, l[h], x);
#pragma unroll
      for (int c = 0; c < 16; ++c) {
        o[h][c] *= f;
#pragma unroll
        for (int x = LANES; x <= 16; x <<= 1) o[h][c] += __shfl_xor_sync(0xffffffffu, o[h][c], x);
      }
      if (gr == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<float4*>(acc + h * D + (i * LANES + lr) * 4) = make_float4(o[h][4 * i], o[h][4 * i + 1], o[h][4 * i + 2], o[h][4 * i + 3]);
        if (lr == 0) ml[h] = make_float2(top, seen ? l[h] : PAGED_NOTHING);
      }
    }
  }
};

// Joins n partial results of one head (the same for all lanes that call it): their common reference, sum, and the factor of each.
struct PagedJoin {
  float base, l;
  bool seen;
  __device__ __forceinline__ void start() { base = -INFINITY; l = 0.f; seen = false; }
  __device__ __forceinline__ void look(float2 ml) {
    base = fmaxf(base, ml.x);
    seen |= ml.y != PAGED_NOTHING;
  }
  __device__ __forceinline__ float factor(float2 ml) {       // (after all have been looked at)
    // Without a row, or without a logit above minus infinity where another part has one: nothing for the sum, and 0 times the
    // part's weighted sum, which is 0 unless it is not finite.
    if (ml.y == PAGED_NOTHING || (ml.x == -INFINITY && base != -INFINITY && ml.y == 0.f)) return 0.f;
    const float f = ml.x == -INFINITY ? 1.f : exp2f(ml.x - base);
    l = fmaf(f, ml.y, l);
    return f;
  }
  // y += this part's four components; where the factor is 0 too: an infinity or a NaN among a part's values stays one, wherever
  // the largest logit lies.
  __device__ __forceinline__ void add(float2 ml, const float4& a, float4& y) {
    const float f = factor(ml);
    y = make_float4(fmaf(f, a.x, y.x), fmaf(f, a.y, y.y), fmaf(f, a.z, y.z), fmaf(f, a.w, y.w));
  }
};

// Four components of a result: y / l, zeros where no row was seen.
template <typename T>
__device__ __forceinline__ void paged_store(const PagedParams& p, int b, int head, int D, int d, const float4& y, float l) {
  const float r = 1.f / l;
  const bool none = l == PAGED_NOTHING;
  const float v[4] = {none ? 0.f : y.x * r, none ? 0.f : y.y * r, none ? 0.f : y.z * r, none ? 0.f : y.w * r};
  T* out = static_cast<T*>(p.out) + ((long long)b * p.H + head) * D + d;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(out) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(out) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  }
}

// A block's run of units.
struct PagedRun {
  long long at, end, base;
  int b, units;
  bool first;
};

template <typename Core, bool CLUSTER>
__global__ void __launch_bounds__(PAGED_THREADS, Core::MIN_BLOCKS) tova_paged_kernel(const __grid_constant__ PagedParams p) {
  constexpr int D = Core::D, HEADS = Core::HEADS;
  using T = typename Core::T;
  __shared__ __align__(16) float acc_s[PAGED_WARPS][HEADS][D];
  __shared__ float2 ml_s[PAGED_WARPS][HEADS];
  __shared__ float2 cta_ml[HEADS];
  __shared__ PagedRun run_s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // The warps' sums of head h, components d .. d + 3; l: the sum, ref: their reference.
  auto joined = [&](int h, int d, float& ref, float& l) {
    PagedJoin j;
    j.start();
    float2 ml[PAGED_WARPS];
#pragma unroll
    for (int w = 0; w < PAGED_WARPS; ++w) {
      ml[w] = ml_s[w][h];
      j.look(ml[w]);
    }
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < PAGED_WARPS; ++w) j.add(ml[w], *reinterpret_cast<const float4*>(&acc_s[w][h][d]), x);
    ref = j.base;
    l = j.seen ? j.l : PAGED_NOTHING;
    return x;
  };
  if constexpr (CLUSTER) {
    const int splits = gridDim.x, rank = blockIdx.x;
    const int b = blockIdx.y / p.jobs, job = blockIdx.y - b * p.jobs, hk = job / p.hgroups, hg = job - hk * p.hgroups;
    const int len = paged_len(p, b), units = (len + PAGED_UNIT - 1) / PAGED_UNIT, share = (units + splits - 1) / splits;
    const int r0 = min(len, rank * share * PAGED_UNIT), r1 = min(len, r0 + share * PAGED_UNIT);
    Core::run(p, b, hk, hg, r0, r1, &acc_s[warp][0][0], ml_s[warp]);
    __syncthreads();
    const int heads = min(HEADS, p.G - hg * HEADS);
    if (splits == 1) {
      for (int e = tid; e < heads * (D / 4); e += PAGED_THREADS) {
        const int h = e / (D / 4), d = (e - h * (D / 4)) * 4;
        float ref, l;
        const float4 x = joined(h, d, ref, l);
        paged_store<T>(p, b, hk * p.G + hg * HEADS + h, D, d, x, l);
      }
      return;
    }
    // (each thread writes over what only it reads)
    for (int e = tid; e < heads * (D / 4); e += PAGED_THREADS) {
      const int h = e / (D / 4), d = (e - h * (D / 4)) * 4;
      float ref, l;
      const float4 x = joined(h, d, ref, l);
      *reinterpret_cast<float4*>(&acc_s[0][h][d]) = x;
      if (d == 0) cta_ml[h] = make_float2(ref, l);
    }
    cluster_arrive_release();
    cluster_wait_acquire();
    auto peer = [](const void* x, int r) {
      uint32_t a;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(x)), "r"(r));
      return a;
    };
    for (int e = rank * PAGED_THREADS + tid; e < heads * (D / 4); e += splits * PAGED_THREADS) {
      const int h = e / (D / 4), d = (e - h * (D / 4)) * 4;
      float2 ml[8];
      float4 x[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        if (r >= splits) break;
        asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(ml[r].x), "=f"(ml[r].y) : "r"(peer(&cta_ml[h], r)) : "memory");
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(x[r].x), "=f"(x[r].y), "=f"(x[r].z), "=f"(x[r].w)
                     : "r"(peer(&acc_s[0][h][d], r))
                     : "memory");
      }
      PagedJoin j;
      j.start();
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (r < splits) j.look(ml[r]);
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (r < splits) j.add(ml[r], x[r], y);
      paged_store<T>(p, b, hk * p.G + hg * HEADS + h, D, d, y, j.seen ? j.l : PAGED_NOTHING);
    }
    cluster_arrive_release();             // nobody leaves while another reads its sums
    cluster_wait_acquire();
  } else {
    if (warp == 0) {
      long long x = 0;
      for (int b = lane; b < p.B; b += 32) x += paged_units(p, b);
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
      const long long total = x * p.jobs, even = (total + gridDim.x - 1) / gridDim.x, share = max(even, (long long)p.least);
      PagedRun r;
      r.at = min(total, blockIdx.x * share);
      r.end = min(total, r.at + share);
      r.base = 0;
      r.b = 0;
      r.units = 1;
      r.first = true;
      if (r.at < r.end) {
        for (int b0 = 0;; b0 += 32) {           // (r.at < total, so some sequence holds it)
          const long long mine = b0 + lane < p.B ? (long long)paged_units(p, b0 + lane) * p.jobs : 0;
          long long upto = mine;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += y;
          }
          const unsigned hit = __ballot_sync(0xffffffffu, r.base + upto > r.at);
          if (hit) {
            const int k = __ffs(hit) - 1;
            r.b = b0 + k;
            r.base += __shfl_sync(0xffffffffu, upto - mine, k);
            break;
          }
          r.base += __shfl_sync(0xffffffffu, upto, 31);
        }
        r.units = paged_units(p, r.b);
      }
      if (lane == 0) run_s = r;
    }
    __syncthreads();
    PagedRun r = run_s;
    const long long share = r.end - r.at;       // (only the last block's may be shorter, and it cuts nothing)
    while (r.at < r.end) {
      while (r.at >= r.base + (long long)r.units * p.jobs) {
        r.base += (long long)r.units * p.jobs;
        r.units = paged_units(p, ++r.b);
      }
      const long long x = r.at - r.base;
      const int job = (int)(x / r.units), u0 = (int)(x - (long long)job * r.units);
      const int u1 = (int)min((long long)r.units, u0 + (r.end - r.at));
      const int hk = job / p.hgroups, hg = job - hk * p.hgroups, len = paged_len(p, r.b);
      const bool whole = u0 == 0 && u1 == r.units;
      const int part = 2 * blockIdx.x + (r.first ? 0 : 1);
      if (u0 == 0 && tid == 0) {
        PagedCut cut;
        cut.pieces = whole ? 0 : (int)((r.at + r.units - 1) / share) - blockIdx.x + 1;
        cut.block = blockIdx.x;
        cut.part = part;
        p.cuts[(long long)r.b * p.jobs + job] = cut;
      }
      Core::run(p, r.b, hk, hg, u0 * PAGED_UNIT, min(len, u1 * PAGED_UNIT), &acc_s[warp][0][0], ml_s[warp]);
      __syncthreads();
      const int heads = min(HEADS, p.G - hg * HEADS);
      for (int e = tid; e < heads * (D / 4); e += PAGED_THREADS) {
        const int h = e / (D / 4), d = (e - h * (D / 4)) * 4;
        float ref, l;
        const float4 y = joined(h, d, ref, l);
        if (whole) {
          paged_store<T>(p, r.b, hk * p.G + hg * HEADS + h, D, d, y, l);
        } else {
          *reinterpret_cast<float4*>(p.part_acc + ((long long)part * HEADS + h) * D + d) = y;
          if (d == 0) p.part_ml[part * HEADS + h] = make_float2(ref, l);
        }
      }
      __syncthreads();
      r.first = false;
      r.at += u1 - u0;
    }
    pdl_launch_dependents();
  }
}

// Joins the parts of the jobs that were cut.  WIDE (few jobs, many parts each): a block per job and head, grid = (jobs, HEADS),
// whose warps share out the parts; else a warp per head, grid = (jobs, HEADS / 8).
constexpr int PAGED_JOIN_WARPS = 8, PAGED_JOIN_THREADS = 32 * PAGED_JOIN_WARPS;
template <typename Core, bool WIDE>
__global__ void __launch_bounds__(PAGED_JOIN_THREADS) tova_paged_join_kernel(const __grid_constant__ PagedParams p) {
  constexpr int D = Core::D, HEADS = Core::HEADS, LANES = D / 4, AT = 32 / LANES;      // lanes a part's row, parts a warp takes at a time
  __shared__ float4 acc_s[WIDE ? PAGED_JOIN_WARPS : 1][LANES];
  __shared__ float sum_s[WIDE ? PAGED_JOIN_WARPS : 1];
  pdl_wait();
  const PagedCut cut = p.cuts[blockIdx.x];
  if (cut.pieces == 0) return;
  const int b = blockIdx.x / p.jobs, job = blockIdx.x - b * p.jobs, hk = job / p.hgroups, hg = job - hk * p.hgroups;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int h = WIDE ? blockIdx.y : blockIdx.y * PAGED_JOIN_WARPS + warp;
  if (h >= min(HEADS, p.G - hg * HEADS)) return;
  // The parts behind the first are the first ones of the blocks that follow.
  auto part = [&](int c) { return c == 0 ? cut.part : 2 * (cut.block + c); };
  PagedJoin j;
  j.start();
  for (int c = lane; c < cut.pieces; c += 32) j.look(p.part_ml[part(c) * HEADS + h]);
  j.base = warp_max(j.base);
  j.seen = __any_sync(0xffffffffu, j.seen) != 0;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
  const int first = (WIDE ? warp : 0) * AT + lane / LANES, step = (WIDE ? PAGED_JOIN_WARPS : 1) * AT, d = lane % LANES;
#pragma unroll 4
  for (int c = first; c < cut.pieces; c += step) {
    const float4 a = *reinterpret_cast<const float4*>(p.part_acc + ((long long)part(c) * HEADS + h) * D + d * 4);
    j.add(p.part_ml[part(c) * HEADS + h], a, y);
  }
  float l = j.l;
  if constexpr (AT == 2) {
    l += __shfl_xor_sync(0xffffffffu, l, LANES);
    y.x += __shfl_xor_sync(0xffffffffu, y.x, LANES);
    y.y += __shfl_xor_sync(0xffffffffu, y.y, LANES);
    y.z += __shfl_xor_sync(0xffffffffu, y.z, LANES);
    y.w += __shfl_xor_sync(0xffffffffu, y.w, LANES);
  }
  if constexpr (WIDE) {
    if (lane < LANES) acc_s[warp][d] = y;
    if (lane == 0) sum_s[warp] = l;
    __syncthreads();
    if (warp != 0) return;
    l = 0.f;
    y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < PAGED_JOIN_WARPS; ++w) {
      const float4 a = acc_s[w][d];
      l += sum_s[w];
      y = make_float4(y.x + a.x, y.y + a.y, y.z + a.z, y.w + a.w);
    }
  }
  if (lane < LANES) paged_store<typename Core::T>(p, b, hk * p.G + hg * HEADS + h, D, d * 4, y, j.seen ? l : PAGED_NOTHING);
}

}  // namespace tova
