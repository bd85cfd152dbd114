// Norms of queries and keys, each head by itself, with the rotation in the same pass, and the gradient (sm_100a).
//
// Forward, a head's row x of D components at position p:
//   r = (mean x^2 + eps)^(-1/2),  y = R_p(x r w)
// with w the weights of q or of k and R_p the rotation of tova_rope.cuh (its factor m included).  Backward, with g = R_p^T dy
// (the rotation by -p, same factor) and xh = x r:
//   dw = sum over all rows of g xh,   dx = r (g w - xh mean(g w xh)).
// The statistics are formed again from x, which the gradient has to read anyway: nothing is kept from the forward pass.
//
// Every component is read once and written once (gradient: two reads, one write) with about ten operations on it: DRAM
// bound.  A row lies in a group of D / 2N neighbouring lanes, two vectors of 16 bytes each, so chosen that both components of a
// pair meet in one lane; N pairs a lane, the same ones in every row.  The sum of squares takes log2(D / 2N) shuffles.  Cosines
// and sines are formed once per token and serve all heads; they, and the weights, lie in shared memory in the lanes' order, so
// that a lane reads them 16 bytes at a time without bank conflicts.
//
// Measured (GPU time, in a captured graph): 4 x 4096 tokens of 32 + 8 heads x 128 in bf16 (335 MB) 57 us, 5.9 TB/s, 0.89 of the
// copy rate; their gradient over 4 x 2047 tokens (252 MB) 56 us, 4.5 TB/s: 124 registers leave 16 warps an SM, whose two reductions
// a row are not covered (three blocks an SM, one row in flight a thread: spills, 62; 128 threads a block: 57); 64 tokens 3.1 us.
// fp32: the first 107 us (6.3 TB/s), the gradient 89 (5.7).  64 or 96 of 128 components turning: 61 and 58-59 us; 20 (pairs that split
// vectors, single components) 117 and 96; interleaved 60 and 57.
// With one vector a lane, so that a pair's other half came by shuffles, the first took 120 us, the second 88.
#pragma once

#include "tova_rope.cuh"
#include "tova_tc.cuh"

namespace tova {

constexpr int NORM_THREADS = 256;
constexpr int NORM_MAX_TOKENS = 4;                 // tokens of a block, forward
constexpr int NORM_BACK_THREADS = 256, NORM_BACK_BLOCKS = 2;      // gradient: blocks resident on an SM
constexpr int NORM_BACK_TOKENS = 8;                // tokens a block has angles for at a time
// Half layout: whole heads; parts of heads; pairs that split vectors.
enum : int { NORM_HALF = 0, NORM_INTERLEAVED = 1, NORM_HALF_ODD = 2, NORM_HALF_PART = 3 };

struct NormRopeParams {
  const void* x[2];             // q, k: element strides between the rows of consecutive (token, sequence) pairs
  const void* dy[2];            // gradient only
  void* y[2];                   // results, or gradients of the inputs
  const void* w[2];             // weights [D], or NULL: ones
  float* dw_part;               // gradient: [blocks][2][D]
  long long x_stride[2], dy_stride[2], y_stride[2];
  int heads[2];                 // heads of q, of k (0: no k)
  const int32_t* positions;     // [T,B] or NULL: first_pos + token
  long long rows;               // T * B
  int first_pos, B, rot;
  int tokens_per_block;         // (gradient: in all)
  unsigned magic[3];            // ceil(2^32 / heads) for q, k and both: head row i belongs to token i * magic / 2^32
  float factor, eps;
  double turns[ROPE_MAX_PAIRS];
};

// A row's D / 2 pairs: N in each of LANES lanes.  Behind the rot / 2 pairs that turn, neighbouring components that pass through
// are pairs that turn by nothing.
template <typename T, int D, int MODE>
struct NormShape {
  static constexpr int N = Vec16<T>::N, LANES = D / (2 * N);
  // Pair k of lane c, and its two components.
  __device__ __forceinline__ static int pair(int c, int k) { return MODE == NORM_HALF_ODD ? k * LANES + c : c * N + k; }
  __device__ __forceinline__ static void components(int i, int half, int& a, int& b) {
    if (MODE == NORM_INTERLEAVED || i >= half) {
      a = 2 * i;                // (of the half layout's passing ones: 2 half + 2 (i - half))
      b = a + 1;
    } else {
      a = i;
      b = i + half;
    }
  }
  // Where pair k of lane c lies in a table in the lanes' order.
  __device__ __forceinline__ static int place(int c, int k) { return ((k >> 2) * LANES + c) * 4 + (k & 3); }

  struct Raw {
    uint4 v[2];
  };
  // A lane's components of a row, as they lie; split: the pairs' first and second components in order.
  __device__ __forceinline__ static void load(const T* row, int c, int half, Raw& r) {
    if constexpr (MODE == NORM_HALF_ODD) {
      T* x = reinterpret_cast<T*>(r.v);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        int a, b;
        components(pair(c, k), half, a, b);
        x[k] = row[a];
        x[N + k] = row[b];
      }
    } else {
      int a, b;
      vectors(c, half, a, b);
      r.v[0] = __ldcs(reinterpret_cast<const uint4*>(row + a));
      r.v[1] = __ldcs(reinterpret_cast<const uint4*>(row + b));
    }
  }
  __device__ __forceinline__ static void store(T* row, int c, int half, const uint64_t (&g)[2][N / 2]) {
    float f[2][N];
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      unpack_f2(g[0][k / 2], f[0][k], f[0][k + 1]);
      unpack_f2(g[1][k / 2], f[1][k], f[1][k + 1]);
    }
    if constexpr (MODE == NORM_HALF_ODD) {
#pragma unroll
      for (int k = 0; k < N; ++k) {
        int a, b;
        components(pair(c, k), half, a, b);
        row[a] = (T)f[0][k];
        row[b] = (T)f[1][k];
      }
    } else {
      int a, b;
      vectors(c, half, a, b);
      float u[2][N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (apart(c, half)) {
          u[0][k] = f[0][k];
          u[1][k] = f[1][k];
        } else {
          u[(2 * k) / N][(2 * k) % N] = f[0][k];
          u[(2 * k) / N][(2 * k) % N + 1] = f[1][k];
        }
      }
      __stcs(reinterpret_cast<uint4*>(row + a), rope_pack<T>(u[0]));
      __stcs(reinterpret_cast<uint4*>(row + b), rope_pack<T>(u[1]));
    }
  }
  // The lane's pairs are (a + k, b + k) for its two vectors; else they are neighbours in both.
  __device__ __forceinline__ static bool apart(int c, int half) { return MODE == NORM_HALF || (MODE == NORM_HALF_PART && c * N < half); }
  __device__ __forceinline__ static void vectors(int c, int half, int& a, int& b) {
    a = apart(c, half) ? c * N : 2 * c * N;
    b = apart(c, half) ? c * N + half : 2 * c * N + N;
  }
  // The pairs' first and second components, two pairs packed.
  __device__ __forceinline__ static void split(const Raw& r, int c, int half, uint64_t (&f)[2][N / 2]) {
    float u[2][N];
    Vec16<T>::unpack(r.v[0], u[0]);
    Vec16<T>::unpack(r.v[1], u[1]);
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      if (MODE == NORM_HALF_ODD || apart(c, half)) {
        f[0][k / 2] = pack_f2(u[0][k], u[0][k + 1]);
        f[1][k / 2] = pack_f2(u[1][k], u[1][k + 1]);
      } else {
        f[0][k / 2] = pack_f2(u[(2 * k) / N][(2 * k) % N], u[(2 * k) / N][(2 * k) % N + 2]);
        f[1][k / 2] = pack_f2(u[(2 * k) / N][(2 * k) % N + 1], u[(2 * k) / N][(2 * k) % N + 3]);
      }
    }
  }
  __device__ __forceinline__ static void table(const float* t, int c, uint64_t (&f)[N / 2]) {
#pragma unroll
    for (int k = 0; k < N; k += 4) {
      const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(t + place(c, k));
      f[k / 2] = x.x;
      f[k / 2 + 1] = x.y;
    }
  }
  // Token and head of head row i (of `heads` a token).
  __device__ __forceinline__ static void locate(int i, int heads, unsigned magic, int& tok, int& head) {
    tok = heads == 1 ? i : (int)__umulhi((unsigned)i, magic);
    head = i - tok * heads;
  }
  __device__ __forceinline__ static float squares(const uint64_t (&x)[2][N / 2]) {
    uint64_t q = mul_f2(x[0][0], x[0][0]);
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
      if (k > 0) q = fma_f2(x[0][k], x[0][k], q);
      q = fma_f2(x[1][k], x[1][k], q);
    }
    float a, b;
    unpack_f2(q, a, b);
    return sum(a + b);
  }
  __device__ __forceinline__ static float sum(float x) {
#pragma unroll
    for (int o = LANES / 2; o >= 1; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
  }
  // Angles of the block's tokens.
  __device__ __forceinline__ static void angles(const NormRopeParams& p, long long row0, int n_tok, float (*cs)[D / 2], float (*sn)[D / 2]) {
    const int half = p.rot >> 1;
    for (int i = threadIdx.x; i < n_tok * (D / 2); i += blockDim.x) {
      const int t = i / (D / 2), at = i - t * (D / 2), k = at / LANES, c = at - k * LANES, j = pair(c, k);
      float s = 0.f, co = 1.f;
      if (j < half) {
        const long long row = row0 + t;
        const double pos = p.positions ? (double)p.positions[row] : (double)p.first_pos + (double)(row / p.B);
        double a = pos * p.turns[j];
        a -= rint(a);
        sincospif((float)(2.0 * a), &s, &co);
        co *= p.factor;
        s *= p.factor;
      }
      cs[t][place(c, k)] = co;
      sn[t][place(c, k)] = s;
    }
  }
};

// Forward.  grid = ceil(rows / tokens_per_block).
template <typename T, int D, int MODE>
__global__ void __launch_bounds__(NORM_THREADS, 4) tova_norm_rope_kernel(const __grid_constant__ NormRopeParams p) {
  using S = NormShape<T, D, MODE>;
  constexpr int N = S::N, U = 2, GROUPS = NORM_THREADS / S::LANES;      // rows at a time
  __shared__ __align__(16) float cs[NORM_MAX_TOKENS][D / 2], sn[NORM_MAX_TOKENS][D / 2], w_s[2][2][D / 2];
  const int group = threadIdx.x / S::LANES, c = threadIdx.x % S::LANES, half = p.rot >> 1;
  const long long row0 = (long long)blockIdx.x * p.tokens_per_block;
  const int n_tok = (int)min((long long)p.tokens_per_block, p.rows - row0);
  const int per_tok = p.heads[0] + p.heads[1], total = n_tok * per_tok;
  for (int i0 = 0; i0 < total; i0 += U * GROUPS) {
    typename S::Raw raw[U];
    int tok[U], which[U], head[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + u * GROUPS + group, total - 1);       // (rows behind the last are formed once more, and not stored)
      S::locate(i, per_tok, p.magic[2], tok[u], head[u]);
      which[u] = head[u] >= p.heads[0];
      if (which[u]) head[u] -= p.heads[0];
      S::load(static_cast<const T*>(p.x[which[u]]) + (row0 + tok[u]) * p.x_stride[which[u]] + (long long)head[u] * D, c, half, raw[u]);
    }
    if (i0 == 0) {
      for (int i = threadIdx.x; i < 2 * (D / 2); i += NORM_THREADS) {
        const int k = i / (D / 2), j = i - k * (D / 2), kk = j / S::LANES, cc = j - kk * S::LANES;
        int a, b;
        S::components(S::pair(cc, kk), half, a, b);
        w_s[k][0][S::place(cc, kk)] = p.w[k] ? (float)static_cast<const T*>(p.w[k])[a] : 1.f;
        w_s[k][1][S::place(cc, kk)] = p.w[k] ? (float)static_cast<const T*>(p.w[k])[b] : 1.f;
      }
      S::angles(p, row0, n_tok, cs, sn);
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * GROUPS >= total) break;
      uint64_t x[2][N / 2], co[N / 2], si[N / 2], w[2][N / 2];
      S::split(raw[u], c, half, x);
      const float r = rsqrtf(S::squares(x) * (1.f / D) + p.eps);
      const uint64_t r2 = pack_f2(r, r), minus = pack_f2(-1.f, -1.f);
      S::table(cs[tok[u]], c, co);
      S::table(sn[tok[u]], c, si);
      S::table(w_s[which[u]][0], c, w[0]);
      S::table(w_s[which[u]][1], c, w[1]);
#pragma unroll
      for (int k = 0; k < N / 2; ++k) {
        const uint64_t a = mul_f2(mul_f2(x[0][k], r2), w[0][k]), b = mul_f2(mul_f2(x[1][k], r2), w[1][k]);
        x[0][k] = fma_f2(a, co[k], mul_f2(mul_f2(b, minus), si[k]));
        x[1][k] = fma_f2(b, co[k], mul_f2(a, si[k]));
      }
      if (i0 + u * GROUPS + group < total)
        S::store(static_cast<T*>(p.y[which[u]]) + (row0 + tok[u]) * p.y_stride[which[u]] + (long long)head[u] * D, c, half, x);
    }
  }
}

// Backward.  A block walks over its share of the tokens, once for q and once for k, whose weights and weights' gradients a lane
// then holds in registers; dw_part[block] is what the block's rows add to the weights' gradients.
template <typename T, int D, int MODE>
__global__ void __launch_bounds__(NORM_BACK_THREADS, NORM_BACK_BLOCKS) tova_norm_rope_back_kernel(const __grid_constant__ NormRopeParams p) {
  using S = NormShape<T, D, MODE>;
  constexpr int N = S::N, U = 2, GROUPS = NORM_BACK_THREADS / S::LANES;
  __shared__ __align__(16) float cs[NORM_BACK_TOKENS][D / 2], sn[NORM_BACK_TOKENS][D / 2];
  __shared__ float sum_s[NORM_BACK_THREADS / 32][D];
  const int group = threadIdx.x / S::LANES, c = threadIdx.x % S::LANES, half = p.rot >> 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int which = 0; which < 2; ++which) {
    const int heads = p.heads[which];
    uint64_t w[2][N / 2], dw[2][N / 2];
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      float v[2][2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        int a, b;
        S::components(S::pair(c, k + x), half, a, b);
        v[0][x] = p.w[which] ? (float)static_cast<const T*>(p.w[which])[a] : 1.f;
        v[1][x] = p.w[which] ? (float)static_cast<const T*>(p.w[which])[b] : 1.f;
      }
      w[0][k / 2] = pack_f2(v[0][0], v[0][1]);
      w[1][k / 2] = pack_f2(v[1][0], v[1][1]);
      dw[0][k / 2] = dw[1][k / 2] = pack_f2(0.f, 0.f);
    }
    const long long first = (long long)blockIdx.x * p.tokens_per_block, behind = min(p.rows, first + p.tokens_per_block);
    for (long long row0 = first; row0 < behind && heads > 0; row0 += NORM_BACK_TOKENS) {
      const int n_tok = (int)min((long long)NORM_BACK_TOKENS, behind - row0);
      const int total = n_tok * heads;
      for (int i0 = 0; i0 < total; i0 += U * GROUPS) {
        typename S::Raw raw[U], graw[U];
        int tok[U], head[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = min(i0 + u * GROUPS + group, total - 1);
          S::locate(i, heads, p.magic[which], tok[u], head[u]);
          S::load(static_cast<const T*>(p.x[which]) + (row0 + tok[u]) * p.x_stride[which] + (long long)head[u] * D, c, half, raw[u]);
          S::load(static_cast<const T*>(p.dy[which]) + (row0 + tok[u]) * p.dy_stride[which] + (long long)head[u] * D, c, half, graw[u]);
        }
        if (i0 == 0) {
          __syncthreads();               // (the tokens before have been turned)
          S::angles(p, row0, n_tok, cs, sn);
          __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (i0 + u * GROUPS >= total) break;
          const bool in = i0 + u * GROUPS + group < total;
          uint64_t x[2][N / 2], g[2][N / 2], co[N / 2], si[N / 2];
          S::split(raw[u], c, half, x);
          const float r = rsqrtf(S::squares(x) * (1.f / D) + p.eps);
          const uint64_t r2 = pack_f2(r, r), minus = pack_f2(-1.f, -1.f);
          S::split(graw[u], c, half, g);
          S::table(cs[tok[u]], c, co);
          S::table(sn[tok[u]], c, si);
          uint64_t sum2 = pack_f2(0.f, 0.f);
#pragma unroll
          for (int k = 0; k < N / 2; ++k) {
            const uint64_t a = fma_f2(g[0][k], co[k], mul_f2(g[1][k], si[k])), b = fma_f2(g[1][k], co[k], mul_f2(mul_f2(g[0][k], minus), si[k]));
            x[0][k] = mul_f2(x[0][k], r2);
            x[1][k] = mul_f2(x[1][k], r2);
            if (in) {
              dw[0][k] = fma_f2(a, x[0][k], dw[0][k]);
              dw[1][k] = fma_f2(b, x[1][k], dw[1][k]);
            }
            g[0][k] = mul_f2(a, w[0][k]);
            g[1][k] = mul_f2(b, w[1][k]);
            sum2 = fma_f2(g[0][k], x[0][k], fma_f2(g[1][k], x[1][k], sum2));
          }
          float s0, s1;
          unpack_f2(sum2, s0, s1);
          const float along = S::sum(s0 + s1) * (-1.f / D);
          const uint64_t along2 = pack_f2(along, along);
#pragma unroll
          for (int k = 0; k < N / 2; ++k) {
            g[0][k] = mul_f2(r2, fma_f2(x[0][k], along2, g[0][k]));
            g[1][k] = mul_f2(r2, fma_f2(x[1][k], along2, g[1][k]));
          }
          if (in) S::store(static_cast<T*>(p.y[which]) + (row0 + tok[u]) * p.y_stride[which] + (long long)head[u] * D, c, half, g);
        }
      }
    }
    // The groups of a warp, the warps, and out.
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int k = 0; k < N; ++k) {
        float both[2];
        unpack_f2(dw[x][k / 2], both[0], both[1]);
        float t = both[k & 1];
#pragma unroll
        for (int o = S::LANES; o <= 16; o <<= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
        int a, b;
        S::components(S::pair(c, k), half, a, b);
        if (lane < S::LANES) sum_s[warp][x ? b : a] = t;
      }
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += NORM_BACK_THREADS) {
      float t = 0.f;
#pragma unroll
      for (int x = 0; x < NORM_BACK_THREADS / 32; ++x) t += sum_s[x][d];
      p.dw_part[((long long)blockIdx.x * 2 + which) * D + d] = t;
    }
  }
  pdl_launch_dependents();
}

// dw[k][d] = the blocks' parts, in their order (64 bits: the sum over all rows is long).  grid = (D / 32, 2), 1024 threads:
// 32 columns, 32 runs of blocks.
__global__ void __launch_bounds__(1024) tova_norm_rope_weights_kernel(const float* part, int blocks, int D, float* dqw, float* dkw) {
  __shared__ double sum_s[32][33];
  const int col = threadIdx.x & 31, run = threadIdx.x >> 5, d = blockIdx.x * 32 + col, k = blockIdx.y;
  pdl_wait();
  float* out = k ? dkw : dqw;
  if (!out) return;
  double s = 0.0;
#pragma unroll 4
  for (int b = run; b < blocks; b += 32) s += (double)part[((long long)b * 2 + k) * D + d];
  sum_s[run][col] = s;
  __syncthreads();
  if (run == 0) {
    s = 0.0;
#pragma unroll
    for (int r = 0; r < 32; ++r) s += sum_s[r][col];
    out[d] = (float)s;
  }
}

}  // namespace tova
