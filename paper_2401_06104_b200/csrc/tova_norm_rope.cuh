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
// bound.  A row lies in a group of D / N neighbouring lanes, 16 bytes each, so that a lane meets the same components in every
// row: its weights stay in registers, and so do its shares of dw.  The sum of squares takes log2(D / N) shuffles, the other
// half of a pair one shuffle a component (the half layout with whole vectors), none (interleaved), or a trip through the
// warp's own shared memory (other sizes of the rotated part).  Cosines and sines are formed once per token and serve all heads.
#pragma once

#include "tova_rope.cuh"

namespace tova {

constexpr int NORM_THREADS = 256;
constexpr int NORM_MAX_TOKENS = 4;                 // tokens a block has angles for at a time
enum : int { NORM_HALF = 0, NORM_INTERLEAVED = 1, NORM_HALF_ODD = 2 };     // the last: pairs that split vectors

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
  int first_pos, B, rot, tokens_per_block;
  float factor, eps;
  double turns[ROPE_MAX_PAIRS];
};

template <typename T, int D>
struct NormShape {
  static constexpr int N = Vec16<T>::N, LANES = D / N, GROUPS = NORM_THREADS / LANES;     // lanes a row, rows at a time
};

// The row's part of a pair that other lanes hold, for each of this lane's components; f: this lane's.  half: rot / 2.
template <typename T, int D, int MODE>
__device__ __forceinline__ void norm_partner(const float (&f)[Vec16<T>::N], float (&o)[Vec16<T>::N], int c, int half, float* stage) {
  constexpr int N = Vec16<T>::N, LANES = D / N;
  if constexpr (MODE == NORM_HALF) {
    const int mate = c * N < half ? c + half / N : c * N < 2 * half ? c - half / N : c;
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] = __shfl_sync(0xffffffffu, f[e], mate, LANES);
  } else if constexpr (MODE == NORM_INTERLEAVED) {
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      o[e] = f[e + 1];
      o[e + 1] = f[e];
    }
  } else {
    __syncwarp();
#pragma unroll
    for (int e = 0; e < N; ++e) stage[c * N + e] = f[e];
    __syncwarp();
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int d = c * N + e;
      o[e] = stage[d < half ? d + half : d < 2 * half ? d - half : d];
    }
  }
}

// f turned by the token's angles (by their negatives where dir is -1).
template <typename T, int D, int MODE>
__device__ __forceinline__ void norm_turn(float (&f)[Vec16<T>::N], int c, int half, const float* cs, const float* sn, float dir, float* stage) {
  constexpr int N = Vec16<T>::N;
  float o[N];
  norm_partner<T, D, MODE>(f, o, c, half, stage);
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const int d = c * N + e;
    if (d < 2 * half) {
      const int pair = MODE == NORM_INTERLEAVED ? d >> 1 : d < half ? d : d - half;
      const bool first = MODE == NORM_INTERLEAVED ? !(e & 1) : d < half;
      const float s = sn[pair] * dir;
      f[e] = f[e] * cs[pair] + o[e] * (first ? -s : s);
    }
  }
}

template <int LANES>
__device__ __forceinline__ float norm_group_sum(float x) {
#pragma unroll
  for (int o = LANES / 2; o >= 1; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// Angles of the block's tokens.
__device__ __forceinline__ void norm_angles(const NormRopeParams& p, long long row0, int n_tok, float (*cs)[ROPE_MAX_PAIRS],
                                            float (*sn)[ROPE_MAX_PAIRS]) {
  const int half = p.rot >> 1;
  for (int i = threadIdx.x; i < n_tok * half; i += NORM_THREADS) {
    const int t = i / half, j = i - t * half;
    const long long row = row0 + t;
    const double pos = p.positions ? (double)p.positions[row] : (double)p.first_pos + (double)(row / p.B);
    double a = pos * p.turns[j];
    a -= rint(a);
    float s, c;
    sincospif((float)(2.0 * a), &s, &c);
    cs[t][j] = c * p.factor;
    sn[t][j] = s * p.factor;
  }
}

// Forward.  grid = ceil(rows / tokens_per_block).
template <typename T, int D, int MODE>
__global__ void __launch_bounds__(NORM_THREADS) tova_norm_rope_kernel(const __grid_constant__ NormRopeParams p) {
  using S = NormShape<T, D>;
  constexpr int N = S::N, U = 4;
  __shared__ __align__(16) float cs[NORM_MAX_TOKENS][ROPE_MAX_PAIRS], sn[NORM_MAX_TOKENS][ROPE_MAX_PAIRS];
  __shared__ float stage_s[MODE == NORM_HALF_ODD ? S::GROUPS : 1][D + 1];
  const int group = threadIdx.x / S::LANES, c = threadIdx.x % S::LANES, half = p.rot >> 1;
  float* stage = stage_s[MODE == NORM_HALF_ODD ? group : 0];
  const long long row0 = (long long)blockIdx.x * p.tokens_per_block;
  const int n_tok = (int)min((long long)p.tokens_per_block, p.rows - row0);
  const int per_tok = p.heads[0] + p.heads[1], total = n_tok * per_tok;
  float w[2][N];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (p.w[k]) {
      Vec16<T>::unpack(*reinterpret_cast<const uint4*>(static_cast<const T*>(p.w[k]) + c * N), w[k]);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) w[k][e] = 1.f;
    }
  }
  for (int i0 = 0; i0 < total; i0 += U * S::GROUPS) {
    uint4 raw[U];
    int tok[U], which[U], head[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = min(i0 + u * S::GROUPS + group, total - 1);       // (rows behind the last are formed once more, and not stored)
      tok[u] = i / per_tok;
      head[u] = i - tok[u] * per_tok;
      which[u] = head[u] >= p.heads[0];
      if (which[u]) head[u] -= p.heads[0];
      raw[u] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(p.x[which[u]]) + (row0 + tok[u]) * p.x_stride[which[u]] +
                                                     (long long)head[u] * D + c * N));
    }
    if (i0 == 0) {
      norm_angles(p, row0, n_tok, cs, sn);
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * S::GROUPS >= total) break;
      float f[N], sum = 0.f;
      Vec16<T>::unpack(raw[u], f);
#pragma unroll
      for (int e = 0; e < N; ++e) sum = fmaf(f[e], f[e], sum);
      const float r = rsqrtf(norm_group_sum<S::LANES>(sum) * (1.f / D) + p.eps);
#pragma unroll
      for (int e = 0; e < N; ++e) f[e] = f[e] * r * (which[u] ? w[1][e] : w[0][e]);
      norm_turn<T, D, MODE>(f, c, half, cs[tok[u]], sn[tok[u]], 1.f, stage);
      if (i0 + u * S::GROUPS + group < total)
        __stcs(reinterpret_cast<uint4*>(static_cast<T*>(p.y[which[u]]) + (row0 + tok[u]) * p.y_stride[which[u]] + (long long)head[u] * D + c * N),
               rope_pack<T>(f));
    }
  }
}

// Backward.  Blocks walk over the tokens; dw_part[block] is what the block's rows add to the weights' gradients.
template <typename T, int D, int MODE>
__global__ void __launch_bounds__(NORM_THREADS) tova_norm_rope_back_kernel(const __grid_constant__ NormRopeParams p) {
  using S = NormShape<T, D>;
  constexpr int N = S::N, U = 2;
  __shared__ __align__(16) float cs[NORM_MAX_TOKENS][ROPE_MAX_PAIRS], sn[NORM_MAX_TOKENS][ROPE_MAX_PAIRS];
  __shared__ float stage_s[MODE == NORM_HALF_ODD ? S::GROUPS : 1][D + 1];
  __shared__ float sum_s[S::GROUPS][D];
  const int group = threadIdx.x / S::LANES, c = threadIdx.x % S::LANES, half = p.rot >> 1;
  float* stage = stage_s[MODE == NORM_HALF_ODD ? group : 0];
  const int per_tok = p.heads[0] + p.heads[1];
  float w[2][N], dw[2][N];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      w[k][e] = 1.f;
      dw[k][e] = 0.f;
    }
    if (p.w[k]) Vec16<T>::unpack(*reinterpret_cast<const uint4*>(static_cast<const T*>(p.w[k]) + c * N), w[k]);
  }
  for (long long row0 = (long long)blockIdx.x * p.tokens_per_block; row0 < p.rows; row0 += (long long)gridDim.x * p.tokens_per_block) {
    const int n_tok = (int)min((long long)p.tokens_per_block, p.rows - row0);
    const int total = n_tok * per_tok;
    for (int i0 = 0; i0 < total; i0 += U * S::GROUPS) {
      uint4 raw[U], graw[U];
      int tok[U], which[U], head[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = min(i0 + u * S::GROUPS + group, total - 1);
        tok[u] = i / per_tok;
        head[u] = i - tok[u] * per_tok;
        which[u] = head[u] >= p.heads[0];
        if (which[u]) head[u] -= p.heads[0];
        const long long at = (long long)head[u] * D + c * N;
        raw[u] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(p.x[which[u]]) + (row0 + tok[u]) * p.x_stride[which[u]] + at));
        graw[u] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(p.dy[which[u]]) + (row0 + tok[u]) * p.dy_stride[which[u]] + at));
      }
      if (i0 == 0) {
        __syncthreads();               // (the tokens before have been turned)
        norm_angles(p, row0, n_tok, cs, sn);
        __syncthreads();
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i0 + u * S::GROUPS >= total) break;
        const bool in = i0 + u * S::GROUPS + group < total;
        float x[N], g[N], sum = 0.f;
        Vec16<T>::unpack(raw[u], x);
        Vec16<T>::unpack(graw[u], g);
        norm_turn<T, D, MODE>(g, c, half, cs[tok[u]], sn[tok[u]], -1.f, stage);
#pragma unroll
        for (int e = 0; e < N; ++e) sum = fmaf(x[e], x[e], sum);
        const float r = rsqrtf(norm_group_sum<S::LANES>(sum) * (1.f / D) + p.eps);
        float along = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) {
          x[e] *= r;
          const float add = in ? g[e] * x[e] : 0.f;
          if (which[u]) dw[1][e] += add;
          else dw[0][e] += add;
          g[e] *= which[u] ? w[1][e] : w[0][e];
          along = fmaf(g[e], x[e], along);
        }
        along = norm_group_sum<S::LANES>(along) * (1.f / D);
#pragma unroll
        for (int e = 0; e < N; ++e) g[e] = r * (g[e] - x[e] * along);
        if (in)
          __stcs(reinterpret_cast<uint4*>(static_cast<T*>(p.y[which[u]]) + (row0 + tok[u]) * p.y_stride[which[u]] + (long long)head[u] * D + c * N),
                 rope_pack<T>(g));
      }
    }
  }
  for (int k = 0; k < 2; ++k) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < N; ++e) sum_s[group][c * N + e] = dw[k][e];
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += NORM_THREADS) {
      float t = 0.f;
#pragma unroll
      for (int x = 0; x < S::GROUPS; ++x) t += sum_s[x][d];
      p.dw_part[((long long)blockIdx.x * 2 + k) * D + d] = t;
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
