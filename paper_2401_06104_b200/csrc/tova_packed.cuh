// Causal attention of packed prompts (sm_100a): sequences of different lengths, one behind the other, every token of which
// attends to itself and the earlier tokens of its sequence,
//   o_i[h] = sum_{j <= i} softmax_j(scale q_i[h] k_j[hk]) v_j[hk],   hk = h / (H / Hkv).
//
// Here: how the work is dealt out, and the kernel on the plain ALUs (fp32, every product in fp32: four prompts of 1500 tokens, 32
// heads x 128, 2.1 ms, 34.7 TFLOP/s, 0.47 of the multiply-adds' peak: shared-memory reads and the unhidden copies between).
#pragma once

#include "tova_mma.cuh"
#include "tova_tc.cuh"

namespace tova {

struct PackedParams {
  const void *q, *k, *v;       // [N, heads * D], rows q_stride, k_stride, v_stride elements apart
  void* out;                   // [N,H,D]
  const int32_t* offsets;      // [S + 1]
  const int4* list;            // (first token of the sequence, the first behind it, tile, 0), those with the most columns first;
                               // NULL: found by every block itself
  const int* n_list;
  long long q_stride, k_stride, v_stride;
  int S, N, H, Hkv, G;
  int pairs;                   // tcgen05 kernel: two heads an item
  float scale2;                // scale * log2(e)
};

// First and last token of sequence b; offsets that fall, or lie outside the tokens, give sequences without tokens.
__device__ __forceinline__ void packed_bounds(const PackedParams& p, int b, int& t0, int& t1) {
  t0 = min(max(p.offsets[b], 0), p.N);
  t1 = min(max(p.offsets[b + 1], t0), p.N);
}

// Sequence and tile number x of `rows` tokens, counted through the sequences, by a whole warp; false behind the last.
__device__ __forceinline__ bool packed_find(const PackedParams& p, int rows, int x, int lane, int& b, int& tile) {
  int base = 0;
  for (int b0 = 0; b0 < p.S; b0 += 32) {
    int mine = 0;
    if (b0 + lane < p.S) {
      int t0, t1;
      packed_bounds(p, b0 + lane, t0, t1);
      mine = (t1 - t0 + rows - 1) / rows;
    }
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, base + upto > x);
    if (hit) {
      const int k = __ffs(hit) - 1;
      b = b0 + k;
      tile = x - base - __shfl_sync(0xffffffffu, upto - mine, k);
      return true;
    }
    base += __shfl_sync(0xffffffffu, upto, 31);
  }
  return false;
}

// The list of all tiles, in order of falling work (to a 1024th of the longest; which of equal ones comes first changes no
// result).  One block.  `room`: entries there are (offsets that overlap could make more tiles than tokens allow).
constexpr int PACKED_PLAN_THREADS = 1024, PACKED_BUCKETS = 1024;
__global__ void __launch_bounds__(PACKED_PLAN_THREADS) tova_packed_plan_kernel(const __grid_constant__ PackedParams p, int rows, int4* list,
                                                                              int* n_list, int room) {
  __shared__ int count[PACKED_BUCKETS], most_s, warp_s[32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  count[tid] = 0;
  if (tid == 0) most_s = 1;
  __syncthreads();
  auto tiles_of = [&](int b) {
    int t0, t1;
    packed_bounds(p, b, t0, t1);
    return (t1 - t0 + rows - 1) / rows;
  };
  for (int b = tid; b < p.S; b += PACKED_PLAN_THREADS) atomicMax(&most_s, tiles_of(b));
  __syncthreads();
  const int most = most_s;
  auto bucket = [&](int tile) { return PACKED_BUCKETS - 1 - (int)((long long)tile * PACKED_BUCKETS / most); };
  for (int b = warp; b < p.S; b += 32) {
    const int n = tiles_of(b);
    for (int i = lane; i < n; i += 32) atomicAdd(&count[bucket(i)], 1);
  }
  __syncthreads();
  const int mine = count[tid];
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  if (lane == 31) warp_s[warp] = upto;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < warp; ++w) before += warp_s[w];
  count[tid] = before + upto - mine;
  if (tid == PACKED_PLAN_THREADS - 1) *n_list = min(room, before + upto);
  __syncthreads();
  for (int b = warp; b < p.S; b += 32) {
    int t0, t1;
    packed_bounds(p, b, t0, t1);
    const int n = (t1 - t0 + rows - 1) / rows;
    for (int i = lane; i < n; i += 32) {
      const int at = atomicAdd(&count[bucket(i)], 1);
      if (at < room) list[at] = make_int4(t0, t1, i, 0);
    }
  }
  pdl_launch_dependents();
}

// Plain ALUs: 64 tokens of one head a block, 64 columns at a time through shared memory; a thread has 4 x 4 logits and 4 x D/16
// components of the result, a row's 16 threads are neighbouring lanes.  grid = (tiles, H).
constexpr int PACKED_ALU_ROWS = 64, PACKED_ALU_THREADS = 256;
template <int D>
constexpr int packed_alu_smem() { return (2 * 64 * (D + 4) + 64 * 68) * 4; }      // (two blocks an SM)

template <typename T, int D>
__global__ void __launch_bounds__(PACKED_ALU_THREADS, 2) tova_packed_alu_kernel(const __grid_constant__ PackedParams p) {
  constexpr int R = PACKED_ALU_ROWS, LD = D + 4, LP = 68, N = Vec16<T>::N;
  extern __shared__ __align__(16) float packed_alu_raw[];
  float *q_s = packed_alu_raw, *k_s = q_s + R * LD, *v_s = k_s, *p_s = k_s + R * LD;      // (V takes the place of K)
  __shared__ int4 found_s;
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  pdl_wait();
  if (tid < 32) {
    int b = 0, tile = 0;
    int4 e = make_int4(0, 0, 0, 0);
    if (p.list) {
      if ((int)blockIdx.x < *p.n_list) e = p.list[blockIdx.x];
    } else if (packed_find(p, R, blockIdx.x, tid, b, tile)) {
      packed_bounds(p, b, e.x, e.y);
      e.z = tile;
    }
    if (tid == 0) found_s = e;
  }
  __syncthreads();
  const int t0 = found_s.x, t1 = found_s.y, tile = found_s.z, h = blockIdx.y, hk = h / p.G;
  if (t0 == t1) return;                  // (no tile lies in a sequence without tokens)
  const int row0 = t0 + tile * R, rows = min(R, t1 - row0);          // first token of the tile
  // 64 rows of one head, those behind `n` zeros.
  auto load = [&](float* to, const void* from, long long stride, int first, int head, int n) {
#pragma unroll 4
    for (int e = tid; e < R * (D / N); e += PACKED_ALU_THREADS) {
      const int r = e / (D / N), c = (e - r * (D / N)) * N;
      float f[N];
      uint4 w = make_uint4(0, 0, 0, 0);
      if (r < n) w = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(from) + (first + r) * stride + (long long)head * D + c));
      Vec16<T>::unpack(w, f);
#pragma unroll
      for (int x = 0; x < N; x += 4) *reinterpret_cast<float4*>(to + r * LD + c + x) = make_float4(f[x], f[x + 1], f[x + 2], f[x + 3]);
    }
  };
  load(q_s, p.q, p.q_stride, row0, h, rows);
  uint64_t o[4][D / 32];                   // pairs of components
  float m[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int c = 0; c < D / 32; ++c) o[i][c] = 0ull;
    m[i] = -INFINITY;
    l[i] = 0.f;
  }
  for (int j = 0; j <= tile; ++j) {
    __syncthreads();
    const int n = min(R, t1 - (t0 + j * R));
    load(k_s, p.k, p.k_stride, t0 + j * R, hk, n);
    __syncthreads();
    float s[4][4];
    {
      uint64_t s2[4][4];                     // even and odd components, packed
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) s2[i][c] = 0ull;
#pragma unroll 4
      for (int d = 0; d < D; d += 4) {
        ulonglong2 a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const ulonglong2*>(q_s + (ty * 4 + i) * LD + d);
#pragma unroll
        for (int c = 0; c < 4; ++c) b[c] = *reinterpret_cast<const ulonglong2*>(k_s + (tx + 16 * c) * LD + d);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c) s2[i][c] = fma_f2(a[i].y, b[c].y, fma_f2(a[i].x, b[c].x, s2[i][c]));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float lo, hi;
          unpack_f2(s2[i][c], lo, hi);
          s[i][c] = lo + hi;
        }
    }
    __syncthreads();
    load(v_s, p.v, p.v_stride, t0 + j * R, hk, n);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = ty * 4 + i;
      float top = m[i];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s[i][c] = j < tile || tx + 16 * c <= r ? s[i][c] * p.scale2 : -INFINITY;
        top = fmaxf(top, s[i][c]);
      }
#pragma unroll
      for (int x = 8; x >= 1; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      const float base = top == -INFINITY ? 0.f : top, f = m[i] == -INFINITY ? 0.f : exp2f(m[i] - base);
      m[i] = top;
      l[i] *= f;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) o[i][c] = mul_f2(o[i][c], pack_f2(f, f));
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float w = exp2f(s[i][c] - base);
        l[i] += w;
        p_s[r * LP + tx + 16 * c] = w;
      }
    }
    __syncthreads();            // (V has landed; a row's weights are written and read by the same half warp)
    // A masked weight is 0, and 0 times a value that is not finite would be NaN: on the diagonal the columns end with the row.
    if (j < tile) {
#pragma unroll 4
      for (int k = 0; k < R; k += 4) {
        float4 a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4*>(p_s + (ty * 4 + i) * LP + k);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          uint64_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float y = x == 0 ? a[i].x : x == 1 ? a[i].y : x == 2 ? a[i].z : a[i].w;
            w[i] = pack_f2(y, y);
          }
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            const ulonglong2 b = *reinterpret_cast<const ulonglong2*>(v_s + (k + x) * LD + c * 64 + tx * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              o[i][2 * c] = fma_f2(w[i], b.x, o[i][2 * c]);
              o[i][2 * c + 1] = fma_f2(w[i], b.y, o[i][2 * c + 1]);
            }
          }
        }
      }
    } else {
      for (int k = 0; k < min(rows, ty * 4 + 4); ++k) {
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
          const ulonglong2 b = *reinterpret_cast<const ulonglong2*>(v_s + k * LD + c * 64 + tx * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (k > ty * 4 + i) continue;
            const float y = p_s[(ty * 4 + i) * LP + k];
            const uint64_t w = pack_f2(y, y);
            o[i][2 * c] = fma_f2(w, b.x, o[i][2 * c]);
            o[i][2 * c + 1] = fma_f2(w, b.y, o[i][2 * c + 1]);
          }
        }
      }
    }
    __syncwarp();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int x = 8; x >= 1; x >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
    const int r = ty * 4 + i;
    if (r >= rows) continue;
    T* out = static_cast<T*>(p.out) + ((long long)(row0 + r) * p.H + h) * D + tx * 4;
    const float inv = 1.f / l[i];
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      float lo, hi;
      unpack_f2(o[i][c], lo, hi);
      out[(c >> 1) * 64 + 2 * (c & 1)] = (T)(lo * inv);
      out[(c >> 1) * 64 + 2 * (c & 1) + 1] = (T)(hi * inv);
    }
  }
}

}  // namespace tova
