// Rotary position embedding of queries and keys (sm_100a): what turns a projection's q and k into the ones the decode
// step takes ("callers pass post-RoPE q and k").
//
// Pair i of a head, i < rotary_dim / 2, at position p:  (a, b) -> m (a c - b s, b c + a s),  c = cos(p w_i),
// s = sin(p w_i), with w_i the pair's frequency and m the factor on both (1 unless the scaling asks for another).  A
// pair is (i, i + rotary_dim/2) in the half layout, (2i, 2i + 1) in the interleaved one; the components from
// rotary_dim on pass through.  The inverse turns by -p w_i and keeps m: it is the transposed map, so it is also what
// a gradient of the result goes through.
//
// The map reads and writes every component once and does three operations on it: DRAM bound.  A block takes a few
// tokens; their cosines and sines are formed once - the angle as a fraction of a turn in 64 bits, since p w_i in 32
// bits is off by whole degrees at far positions, then sincospi in 32 - and serve all H + Hkv heads from shared memory.
// Measured (GPU time, in a captured graph): 4 x 4096 tokens of 32 + 8 heads x 128 in bf16 (335 MB) 54 us, 6.2 TB/s; one step's
// 64 tokens 2.8 us.  Four tokens a block are few bytes where heads are few or small, and half the bytes in flight where half a
// head passes through: 4 x 16384 tokens of 8 + 2 heads x 64 (168 MB) 47 us, 3.6 TB/s; the first case with 64 of 128
// components turning 67 us.
#pragma once

#include "tova_device.cuh"

namespace tova {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_MAX_PAIRS = 64;    // head_dim <= 128
constexpr int ROPE_MAX_TOKENS = 4;    // tokens per block

struct RopeParams {
  const void* x[2];             // q, k: element strides between the rows of consecutive (token, sequence) pairs
  void* y[2];
  long long x_stride[2], y_stride[2];
  int heads[2];                 // heads of q, of k (0: no k)
  const int32_t* positions;     // [T,B] or NULL: first_pos + token
  long long rows;               // T * B
  int first_pos, B, D, rot, tokens_per_block;
  float factor, sign;           // m; +1, or -1 for the inverse
  double turns[ROPE_MAX_PAIRS]; // w_i / 2 pi
};

template <typename T>
__device__ __forceinline__ uint4 rope_pack(const float (&f)[Vec16<T>::N]);
template <>
__device__ __forceinline__ uint4 rope_pack<float>(const float (&f)[4]) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <>
__device__ __forceinline__ uint4 rope_pack<__nv_bfloat16>(const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);   // the result's one rounding
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// VEC: units of 16 bytes (rotary_dim a multiple of 2 vectors in the half layout, of one in the interleaved one);
// otherwise a unit is one pair, or one component of the rest.  grid = ceil(rows / tokens_per_block).
template <typename T, bool HALF, bool VEC>
__global__ void __launch_bounds__(ROPE_THREADS) tova_rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int N = Vec16<T>::N;
  __shared__ __align__(16) float cs[ROPE_MAX_TOKENS][ROPE_MAX_PAIRS], sn[ROPE_MAX_TOKENS][ROPE_MAX_PAIRS];
  const long long row0 = (long long)blockIdx.x * p.tokens_per_block;
  const int n_tok = (int)min((long long)p.tokens_per_block, p.rows - row0);
  const int half = p.rot >> 1;
  const int turning = VEC ? (HALF ? half / N : p.rot / N) : half;       // units that turn, per head
  const int passing = VEC ? (p.D - p.rot) / N : p.D - p.rot;            // units that pass through
  const int per_head = turning + passing;
  const int per_tok = (p.heads[0] + p.heads[1]) * per_head;
  const int total = n_tok * per_tok;
  // Where unit i is: its token in the block, its position in the head, its head's place in the input and the output.
  auto locate = [&](int i, int& t, int& u, const T*& x, T*& y) {
    t = i / per_tok;
    const int rem = i - t * per_tok;
    int h = rem / per_head;
    u = rem - h * per_head;
    const int which = h >= p.heads[0];
    if (which) h -= p.heads[0];
    x = static_cast<const T*>(p.x[which]) + (row0 + t) * p.x_stride[which] + (long long)h * p.D;
    y = static_cast<T*>(p.y[which]) + (row0 + t) * p.y_stride[which] + (long long)h * p.D;
  };
  auto angles = [&]() {
    for (int i = threadIdx.x; i < n_tok * half; i += ROPE_THREADS) {
      const int t = i / half, j = i - t * half;
      const long long row = row0 + t;
      const double pos = p.positions ? (double)p.positions[row] : (double)p.first_pos + (double)(row / p.B);
      double a = pos * p.turns[j];
      a -= rint(a);
      float s, c;
      sincospif((float)(2.0 * a), &s, &c);
      cs[t][j] = c * p.factor;
      sn[t][j] = s * p.factor * p.sign;
    }
    __syncthreads();
  };
  if constexpr (VEC) {
    // U units a thread are loaded before any is used, the first ones before the angles are formed.
    constexpr int U = HALF ? 2 : 4;
    for (int i0 = threadIdx.x; i0 < total + (int)threadIdx.x; i0 += U * ROPE_THREADS) {
      uint4 wa[U], wb[U];
      int t[U], u[U];
      T* y[U];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int i = i0 + k * ROPE_THREADS;
        u[k] = -1;
        if (i >= total) continue;
        const T* x;
        locate(i, t[k], u[k], x, y[k]);
        const int d = u[k] < turning ? u[k] * N : p.rot + (u[k] - turning) * N;
        wa[k] = __ldcs(reinterpret_cast<const uint4*>(x + d));
        if (HALF && u[k] < turning) wb[k] = __ldcs(reinterpret_cast<const uint4*>(x + half + d));
      }
      if (i0 == (int)threadIdx.x) angles();
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (u[k] < 0) continue;
        if (u[k] >= turning) {
          __stcs(reinterpret_cast<uint4*>(y[k] + p.rot + (u[k] - turning) * N), wa[k]);
          continue;
        }
        const int d = u[k] * N;
        float a[N];
        Vec16<T>::unpack(wa[k], a);
        if constexpr (HALF) {
          float b[N], ya[N], yb[N];
          Vec16<T>::unpack(wb[k], b);
#pragma unroll
          for (int e = 0; e < N; e += 4) {
            const float4 c4 = *reinterpret_cast<const float4*>(&cs[t[k]][d + e]);
            const float4 s4 = *reinterpret_cast<const float4*>(&sn[t[k]][d + e]);
            const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              ya[e + x] = a[e + x] * c[x] - b[e + x] * s[x];
              yb[e + x] = b[e + x] * c[x] + a[e + x] * s[x];
            }
          }
          __stcs(reinterpret_cast<uint4*>(y[k] + d), rope_pack<T>(ya));
          __stcs(reinterpret_cast<uint4*>(y[k] + half + d), rope_pack<T>(yb));
        } else {
#pragma unroll
          for (int e = 0; e < N; e += 2) {
            const float c = cs[t[k]][(d + e) >> 1], s = sn[t[k]][(d + e) >> 1];
            const float lo = a[e] * c - a[e + 1] * s;
            a[e + 1] = a[e + 1] * c + a[e] * s;
            a[e] = lo;
          }
          __stcs(reinterpret_cast<uint4*>(y[k] + d), rope_pack<T>(a));
        }
      }
    }
  } else {
    angles();
    for (int i = threadIdx.x; i < total; i += ROPE_THREADS) {
      int t, u;
      const T* x;
      T* y;
      locate(i, t, u, x, y);
      if (u >= turning) {
        const int d = p.rot + u - turning;
        y[d] = x[d];
      } else {
        const int da = HALF ? u : 2 * u, db = HALF ? u + half : 2 * u + 1;
        const float a = (float)x[da], b = (float)x[db], c = cs[t][u], s = sn[t][u];
        y[da] = (T)(a * c - b * s);
        y[db] = (T)(b * c + a * s);
      }
    }
  }
}

}  // namespace tova
