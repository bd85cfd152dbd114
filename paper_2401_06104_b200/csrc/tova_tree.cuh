// Attention of drafted tokens over a state (sm_100a).
//
// N drafted tokens of a sequence (nodes) hang below its last settled token as a tree, parents[i] < i, -1 for the root.
// A node sees the state's live rows, its ancestors and itself:
//   o_i = sum_j p_ij v_j,  p_ij = softmax_j(scale q_i k_j)  over j in state rows + {i, parent(i), parent(parent(i)), ...}
// A node whose parent is neither -1 nor an earlier node, and every node below it, is padding: it sees nothing, o = 0.
// Any other node sees itself; where all its logits are minus infinity it has no soft-max, and 0 / 0 makes the row NaN.
// The state is only read.  N = 1 is a plain step without eviction.
//
// The rows of the product are the M = N G pairs (node, query head) that share a KV head; its columns the state's rows,
// then the drafted tokens.  The state's bytes are what cannot be avoided, and M of these rows use each of them: few
// rows leave the kernel waiting for memory, many for the contractions.  The columns are cut into `splits` runs so that
// even one sequence gives every SM something to do; a run's (max, sum, weighted sum) go through the caller's
// workspace and a second kernel joins them.  One run writes the result itself.
#pragma once

#include "tova_quant.cuh"

namespace tova {

constexpr int TREE_MAX_NODES = 256;
constexpr int TREE_ANC_WORDS = TREE_MAX_NODES / 32;
constexpr float TREE_PADDING = -1.f;     // the sum that stands for "a padding node" in a partial result

struct TreeParams {
  const void* q;               // [N,B,H,D]
  const void* k_new;           // [N,B,Hkv,D]
  const void* v_new;
  const void* K;               // [B,Hkv,cap,D]
  const void* V;
  const float* k_scale;        // [B,Hkv,cap], 8-bit states
  const float* v_scale;
  const int32_t* lens;         // [B] or NULL: n_live rows in every sequence
  const int32_t* parents;      // [N,B] or NULL: a chain
  void* out;                   // [N,B,H,D]
  float2* part_ml;             // [splits][B,Hkv,M] running max (base 2), sum
  float* part_acc;             // [splits][B,Hkv,M][D]
  int N, B, H, Hkv, G, M, cap, n_live;
  int splits, split_cols;      // columns of a run (a multiple of the kernel's tile); the last run also has the drafts
  int group, row_rounds, least;    // tcgen05 kernel: blocks side by side, rounds of their rows per KV head, fewest tiles of a run
  void* cuts;                  // tcgen05 kernel: one TreeTcCut per block
  int tiled, q_tiled;          // tcgen05 kernel: there are tensor maps of a bf16 state, of q
  float scale2;                // scale * log2(e)
};

__host__ __device__ __forceinline__ int tree_len(const TreeParams& p, int b) {
  return p.lens ? max(0, min(p.lens[b], p.n_live)) : p.n_live;
}

// Ancestor bits of node i: bit j of word w says that node 32 w + j is i or above it; all zero for padding.  par holds the
// sequence's parents (or it is a chain); the walk goes strictly down in index, so it ends.
template <int WORDS>
__device__ __forceinline__ void tree_ancestor_bits(int i, bool chain, const int* par, uint32_t* anc) {
  uint32_t w[WORDS];
#pragma unroll
  for (int k = 0; k < WORDS; ++k) w[k] = chain ? (i >= 32 * k + 31 ? 0xffffffffu : i >= 32 * k ? (2u << (i & 31)) - 1u : 0u) : 0u;
  int j = chain ? -1 : i;
  while (j >= 0) {
#pragma unroll
    for (int k = 0; k < WORDS; ++k) w[k] |= (j >> 5) == k ? 1u << (j & 31) : 0u;
    const int up = par[j];
    if (up < -1 || up >= j) {
#pragma unroll
      for (int k = 0; k < WORDS; ++k) w[k] = 0;
      break;
    }
    j = up;
  }
#pragma unroll
  for (int k = 0; k < WORDS; ++k) anc[k] = w[k];
}

// Zeroes the infinities and NaN among eight bf16 values; true if there were any.
__device__ __forceinline__ bool tree_drop_odd(uint4& w) {
  uint32_t* x = reinterpret_cast<uint32_t*>(&w);
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (x[i] & 0x00007f80u) == 0x00007f80u, hi = (x[i] & 0x7f800000u) == 0x7f800000u;
    odd |= lo | hi;
    x[i] &= (lo ? 0xffff0000u : 0xffffffffu) & (hi ? 0x0000ffffu : 0xffffffffu);
  }
  return odd;
}

// Adds the values that tree_drop_odd took out, of the drafts whose bits are set, to a row's components d0..d0+E-1 before
// normalisation: a positive weight times an infinity or NaN is that again.
template <int WORDS, int E>
__device__ __forceinline__ void tree_add_odd(const TreeParams& p, int b, int hk, const uint32_t* anc, int D, int d0, float* acc) {
  for (int j = 0; j < p.N; ++j) {
    uint32_t word = 0;
#pragma unroll
    for (int k = 0; k < WORDS; ++k)
      if (k == (j >> 5)) word = anc[k];
    if (!((word >> (j & 31)) & 1u)) continue;
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.v_new) + (((long long)j * p.B + b) * p.Hkv + hk) * D + d0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float v = __bfloat162float(src[e]);
      if (!isfinite(v)) acc[e] += v;
    }
  }
}

template <typename T>
__device__ __forceinline__ void tree_store4(T* dst, float a, float b, float c, float d);
template <>
__device__ __forceinline__ void tree_store4<float>(float* dst, float a, float b, float c, float d) {
  *reinterpret_cast<float4*>(dst) = make_float4(a, b, c, d);
}
template <>
__device__ __forceinline__ void tree_store4<__nv_bfloat16>(__nv_bfloat16* dst, float a, float b, float c, float d) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(a, b), hi = __floats2bfloat162_rn(c, d);   // the result's one rounding
  *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}

// ---------------------------------------------------------------------------------------------------------------
// Copies to shared memory that run on; bytes past src_bytes become zeros.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t src_bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, uint32_t src_bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Plain-ALU kernel: every product in fp32.  Serves fp32 queries, whose results the tensor cores' bf16 operands could not
// give one contraction at a time (three bf16 terms a factor, six contractions, could; not built).  A block takes R rows of the product (64,
// or 16 or 4 where there are no more) and a run of columns in tiles of 32, all in shared memory as fp32.  Bound by shared
// memory and the FMA pipes together, so a thread does as much as it can with what it reads: 4 x 4 logits from eight 16-byte
// reads (64 FMA), the weighted sum in 8 rows x 8 components from four (64 FMA; the weights lie transposed).  Keys of the next
// tile are on their way while the weighted sum runs, values while the logits are formed: each has one buffer, free at just
// that time.  8-bit codes wait in registers.  Measured (D 128, 8 sequences x 4096 rows, 32 query heads): a single step over 32 KV
// heads 265 us (4.1 TB/s of state), 64 chained drafts over 8 KV heads 1140 us (30.6 TFLOP/s).  Without the early copies 793 and
// 1463 us.  grid = (ceil(M / R), splits, B * Hkv).
constexpr int TREE_ALU_THREADS = 128;
constexpr int TREE_ALU_COLS = 32;

template <int D, int R>
inline size_t tree_alu_smem_bytes() {
  return sizeof(float) * (R * (D + 4) + TREE_ALU_COLS * (2 * D + 4) + TREE_ALU_COLS * (R + 4));
}

template <int D, int FMT, int R>
__global__ void __launch_bounds__(TREE_ALU_THREADS) tova_tree_alu_kernel(const __grid_constant__ TreeParams p) {
  constexpr int C = TREE_ALU_COLS, TH = TREE_ALU_THREADS;
  constexpr int LD = D + 4;                      // row stride of Q and K in shared memory: rows 4 banks apart
  constexpr int LP = R + 4;                      // ... of the weights, a column's R rows
  constexpr int QR = R == 64 ? 4 : R == 16 ? 2 : 1, QC = QR;    // logits of a thread
  constexpr int CG = C / QC;                                    // threads of a row: neighbouring lanes
  constexpr int PR = R == 64 ? 8 : R == 16 ? 4 : D / 32;        // weighted sum of a thread: PR rows x PC components
  constexpr int XG = TH / (R / PR), PC = D / XG;
  constexpr int PV = PC < 4 ? PC : 4;                           // ... in pieces of PV neighbours, XG * PV apart
  static_assert(CG * (R / QR) == TH && XG * (R / PR) == TH, "every thread has a share");
  extern __shared__ __align__(16) float tree_alu_smem[];
  float* q_s = tree_alu_smem;                    // [R][LD]
  float* k_s = q_s + R * LD;                     // [C][LD]
  float* v_s = k_s + C * LD;                     // [C][D]
  float* p_s = v_s + C * D;                      // [C][LP]
  __shared__ int par_s[TREE_MAX_NODES];
  __shared__ uint32_t anc_s[TREE_MAX_NODES][TREE_ANC_WORDS];
  __shared__ float m_s[R], corr_s[R];

  const int tid = threadIdx.x;
  const int b = blockIdx.z / p.Hkv, hk = blockIdx.z % p.Hkv;
  const int split = blockIdx.y, row0 = blockIdx.x * R;
  const int len = tree_len(p, b);
  const bool last = split == p.splits - 1;
  const int c0 = split * p.split_cols;
  const int c1 = last ? len : min(len, c0 + p.split_cols);
  const int n_state = c1 > c0 ? (c1 - c0 + C - 1) / C : 0;
  const int n_draft = last ? (p.N + C - 1) / C : 0;

  // One tile's rows of keys (x = 0) or values (1) on their way: 16 bytes of floats go straight to shared memory, codes and
  // their scales to registers, from where landed() converts them.  Rows past the end: zeros.
  constexpr int CHUNKS = C * D / 4 / TH;
  constexpr bool CODES = FMT != FORMAT_PLAIN;
  uint32_t code[CODES ? CHUNKS : 1];
  float code_scale[CODES ? CHUNKS : 1];
  auto fetch = [&](int tile, int x) {
    const bool draft = tile >= n_state;
    const int j0 = draft ? (tile - n_state) * C : c0 + tile * C, jn = draft ? p.N : c1;
    float* dst = x ? v_s : k_s;
    const int ld = x ? D : LD;
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) {
      const int i = u * TH + tid, r = i / (D / 4), d = (i % (D / 4)) * 4;
      const bool in = j0 + r < jn;
      const int j = in ? j0 + r : j0;          // (a tile has at least one row)
      if (!CODES || draft) {
        const float* src = draft ? static_cast<const float*>(x ? p.v_new : p.k_new) + (((long long)j * p.B + b) * p.Hkv + hk) * D + d
                                 : static_cast<const float*>(x ? p.V : p.K) + ((long long)blockIdx.z * p.cap + j) * D + d;
        cp_async16(smem_addr(dst + r * ld + d), src, in ? 16 : 0);
      } else if constexpr (CODES) {
        const long long row = (long long)blockIdx.z * p.cap + j;
        code[u] = in ? *reinterpret_cast<const uint32_t*>(static_cast<const unsigned char*>(x ? p.V : p.K) + row * D + d) : 0u;
        code_scale[u] = in ? (x ? p.v_scale : p.k_scale)[row] : 0.f;
      }
    }
    cp_async_commit();
  };
  auto landed = [&](int tile, int x) {
    if (CODES && tile < n_state) {
      float* dst = x ? v_s : k_s;
      const int ld = x ? D : LD;
#pragma unroll
      for (int u = 0; u < CHUNKS; ++u) {
        const int i = u * TH + tid, r = i / (D / 4), d = (i % (D / 4)) * 4;
        float a[4];
        if constexpr (CODES) {
          quant_unpack4<FMT>(code[u], a);
          const float f = code_scale[u];
          *reinterpret_cast<float4*>(dst + r * ld + d) = make_float4(a[0] * f, a[1] * f, a[2] * f, a[3] * f);
        }
      }
    }
    cp_async_wait<0>();
    __syncthreads();
  };
  if (n_state + n_draft > 0) fetch(0, 0);

  if (last) {
    for (int i = tid; i < p.N; i += TH) par_s[i] = p.parents ? p.parents[(long long)i * p.B + b] : i - 1;
    __syncthreads();
    for (int i = tid; i < p.N; i += TH) tree_ancestor_bits<TREE_ANC_WORDS>(i, p.parents == nullptr, par_s, anc_s[i]);
  }
  // Q rows, scaled into the base-2 domain
  for (int i = tid; i < R * (D / 4); i += TH) {
    const int r = i / (D / 4), d = (i % (D / 4)) * 4;
    const int m = row0 + r;
    float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
    if (m < p.M) {
      const int n = m / p.G, g = m - n * p.G;
      w = *reinterpret_cast<const float4*>(static_cast<const float*>(p.q) + (((long long)n * p.B + b) * p.H + hk * p.G + g) * D + d);
    }
    *reinterpret_cast<float4*>(q_s + r * LD + d) = make_float4(w.x * p.scale2, w.y * p.scale2, w.z * p.scale2, w.w * p.scale2);
  }
  const int lr = (tid / CG) * QR, lc = tid % CG;         // logits: rows lr.., columns lc + CG k
  const int orow = (tid / XG) * PR, ox = (tid % XG) * PV; // weighted sum: rows orow.., components ox + XG PV j + 0..PV-1
  // Warps whose rows all lie behind the last have nothing to do (129 rows are two blocks and a warp); what they hold is not used.
  const bool has_logits = row0 + (tid & ~31) / CG * QR < p.M, has_sums = row0 + (tid & ~31) / XG * PR < p.M;
  float acc[PR][PC];
#pragma unroll
  for (int i = 0; i < PR; ++i)
#pragma unroll
    for (int j = 0; j < PC; ++j) acc[i][j] = 0.f;
  float m_run[QR], l_run[QR];
#pragma unroll
  for (int i = 0; i < QR; ++i) { m_run[i] = -INFINITY; l_run[i] = 0.f; }

  for (int tile = 0; tile < n_state + n_draft; ++tile) {
    const bool draft = tile >= n_state;
    const int j0 = draft ? (tile - n_state) * C : c0 + tile * C;      // first column of the tile, in its own numbering
    const int jn = draft ? p.N : c1;
    landed(tile, 0);            // (and every thread has done with the values and weights of the last tile)
    fetch(tile, 1);
    if (has_logits) {
      float s[QR][QC];
#pragma unroll
      for (int i = 0; i < QR; ++i)
#pragma unroll
        for (int k = 0; k < QC; ++k) s[i][k] = 0.f;
#pragma unroll 4
      for (int d = 0; d < D; d += 4) {
        float4 q[QR];
#pragma unroll
        for (int i = 0; i < QR; ++i) q[i] = *reinterpret_cast<const float4*>(q_s + (lr + i) * LD + d);
#pragma unroll
        for (int k = 0; k < QC; ++k) {
          const float4 kk = *reinterpret_cast<const float4*>(k_s + (lc + CG * k) * LD + d);
#pragma unroll
          for (int i = 0; i < QR; ++i)
            s[i][k] = fmaf(q[i].x, kk.x, fmaf(q[i].y, kk.y, fmaf(q[i].z, kk.z, fmaf(q[i].w, kk.w, s[i][k]))));
        }
      }
      float e[QC][QR];
#pragma unroll
      for (int i = 0; i < QR; ++i) {
        const int m = row0 + lr + i;
        const uint32_t see = draft ? (m < p.M ? anc_s[m / p.G][j0 >> 5] : 0u) : 0u;
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < QC; ++k) {
          const int c = lc + CG * k;
          const bool vis = draft ? ((see >> c) & 1u) != 0 : j0 + c < jn;
          if (!vis) s[i][k] = -INFINITY;
          top = fmaxf(top, s[i][k]);
        }
#pragma unroll
        for (int o = CG / 2; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float m_new = fmaxf(m_run[i], top);
        const float base = m_new == -INFINITY ? 0.f : m_new;
        const float corr = exp2f(m_run[i] - base);       // 0 while nothing has been seen
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < QC; ++k) {
          e[k][i] = exp2f(s[i][k] - base);
          sum += e[k][i];
        }
#pragma unroll
        for (int o = CG / 2; o >= 1; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        l_run[i] = l_run[i] * corr + sum;
        m_run[i] = m_new;
        if (lc == 0) corr_s[lr + i] = corr;
      }
#pragma unroll
      for (int k = 0; k < QC; ++k) {
        float* dst = p_s + (lc + CG * k) * LP + lr;
        if constexpr (QR == 4) *reinterpret_cast<float4*>(dst) = make_float4(e[k][0], e[k][1], e[k][2], e[k][3]);
        else if constexpr (QR == 2) *reinterpret_cast<float2*>(dst) = make_float2(e[k][0], e[k][1]);
        else *dst = e[k][0];
      }
    }
    landed(tile, 1);            // (and every thread has done with the keys)
    if (tile + 1 < n_state + n_draft) fetch(tile + 1, 0);
    if (!has_sums) continue;
#pragma unroll
    for (int i = 0; i < PR; ++i) {
      const float corr = corr_s[orow + i];
#pragma unroll
      for (int j = 0; j < PC; ++j) acc[i][j] *= corr;
    }
    auto column = [&](int c, float (&w)[PR], float (&v)[PC]) {
      if constexpr (PR % 4 == 0) {
#pragma unroll
        for (int i = 0; i < PR; i += 4) {
          const float4 x = *reinterpret_cast<const float4*>(p_s + c * LP + orow + i);
          w[i] = x.x; w[i + 1] = x.y; w[i + 2] = x.z; w[i + 3] = x.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < PR; ++i) w[i] = p_s[c * LP + orow + i];
      }
#pragma unroll
      for (int j = 0; j < PC; j += PV) {
        const float* src = v_s + c * D + ox + XG * j;
        if constexpr (PV == 4) {
          const float4 x = *reinterpret_cast<const float4*>(src);
          v[j] = x.x; v[j + 1] = x.y; v[j + 2] = x.z; v[j + 3] = x.w;
        } else if constexpr (PV == 2) {
          const float2 x = *reinterpret_cast<const float2*>(src);
          v[j] = x.x; v[j + 1] = x.y;
        } else {
          v[j] = *src;
        }
      }
    };
    if (!draft) {
#pragma unroll 2
      for (int c = 0; c < C; ++c) {
        float w[PR], v[PC];
        column(c, w, v);
#pragma unroll
        for (int i = 0; i < PR; ++i)
#pragma unroll
          for (int j = 0; j < PC; ++j) acc[i][j] = fmaf(w[i], v[j], acc[i][j]);
      }
    } else {
      // Drafts that a row does not see may hold anything: 0 times an infinity must not reach the sum.
      for (int c = 0; c < C; ++c) {
        float w[PR], v[PC];
        column(c, w, v);
#pragma unroll
        for (int i = 0; i < PR; ++i)
          if (w[i] != 0.f) {
#pragma unroll
            for (int j = 0; j < PC; ++j) acc[i][j] = fmaf(w[i], v[j], acc[i][j]);
          }
      }
    }
  }
  __syncthreads();
  if (lc == 0) {
#pragma unroll
    for (int i = 0; i < QR; ++i) {
      const int m = row0 + lr + i;
      float l = l_run[i];
      if (last && m < p.M) {
        const int n = m / p.G;
        if (((anc_s[n][n >> 5] >> (n & 31)) & 1u) == 0) l = TREE_PADDING;
      }
      m_s[lr + i] = m_run[i];
      corr_s[lr + i] = l;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PR; ++i) {
    const int m = row0 + orow + i;
    if (m >= p.M) continue;
    const float l = corr_s[orow + i];
    const float r = 1.f / l;
    const int n = m / p.G, g = m - n * p.G;
    const long long at = ((long long)split * gridDim.z + blockIdx.z) * p.M + m;
    float* out = static_cast<float*>(p.out) + (((long long)n * p.B + b) * p.H + hk * p.G + g) * D;
    if (p.splits > 1 && ox == 0) p.part_ml[at] = make_float2(m_s[orow + i], l);
#pragma unroll
    for (int j = 0; j < PC; ++j) {
      const int d = ox + XG * (j / PV * PV) + j % PV;
      if (p.splits == 1) out[d] = l == TREE_PADDING ? 0.f : acc[i][j] * r;
      else p.part_acc[at * D + d] = acc[i][j];
    }
  }
}

// Joins the runs' partial results: o = sum_s 2^(m_s - m) acc_s / sum_s 2^(m_s - m) l_s.  One warp per row of the
// product, its lanes first over the runs, then over D; grid = ceil(B Hkv M / 4), 128 threads.
constexpr int TREE_MERGE_THREADS = 128;
template <typename T, int D>
__global__ void __launch_bounds__(TREE_MERGE_THREADS) tova_tree_merge_kernel(const __grid_constant__ TreeParams p) {
  const int lane = threadIdx.x & 31;
  const long long rows = (long long)p.B * p.Hkv * p.M;
  const long long row = (long long)blockIdx.x * (TREE_MERGE_THREADS / 32) + (threadIdx.x >> 5);
  if (row >= rows) return;
  pdl_wait();
  float m = -INFINITY;
  bool pad = false;
  for (int s = lane; s < p.splits; s += 32) {
    const float2 ml = p.part_ml[s * rows + row];
    m = fmaxf(m, ml.x);
    if (s == p.splits - 1) pad = ml.y == TREE_PADDING;
  }
  m = warp_max(m);
  pad = __any_sync(0xffffffffu, pad) != 0;
  const float base = m == -INFINITY ? 0.f : m;
  constexpr int E = D / 32;
  float acc[E], l = 0.f;
#pragma unroll
  for (int j = 0; j < E; ++j) acc[j] = 0.f;
  const float* src = p.part_acc + row * D + lane * E;
  for (int s0 = 0; s0 < p.splits; s0 += 32) {
    // lane's run: its factor, and its share of the sum.  (A run without a visible column has the factor 0 and zeros.)
    float w = 0.f;
    if (s0 + lane < p.splits) {
      const float2 ml = p.part_ml[(s0 + lane) * rows + row];
      w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - base);
      if (w != 0.f) l += w * ml.y;
    }
    const int n = min(32, p.splits - s0);
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const float f = __shfl_sync(0xffffffffu, w, i);
      const float* a = src + (s0 + i) * rows * D;
#pragma unroll
      for (int j = 0; j < E; ++j) acc[j] = fmaf(f, a[j], acc[j]);
    }
  }
  l = warp_sum(l);
  const int bh = (int)(row / p.M), mm = (int)(row - (long long)bh * p.M);
  const int b = bh / p.Hkv, hk = bh - b * p.Hkv, n = mm / p.G, g = mm - n * p.G;
  T* dst = static_cast<T*>(p.out) + (((long long)n * p.B + b) * p.H + hk * p.G + g) * D + lane * E;
  const float r = 1.f / l;
#pragma unroll
  for (int j = 0; j < E; ++j) dst[j] = (T)(pad ? 0.f : acc[j] * r);
}

}  // namespace tova
