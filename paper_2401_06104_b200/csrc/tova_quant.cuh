// The 8-bit state (sm_100a): keys and values of new tokens quantised as they are written into the state's slots, and
// rows of the state read back.
//
// A row is one token's key or value of one KV head, x[D].  With a = max |x_d| and Q = 127 (int8) or 448 (e4m3):
//   scale = fp32(a / Q),   code_d = nearest(fp32(x_d fp32(Q / a)))   (ties to even),   value = code_d scale.
// The two quotients are the correctly rounded fp32 ones and the product is rounded once, so the codes are a function
// of the inputs alone, not of how they are computed.  a < 2^-100: scale 0, codes 0 (Q / a would leave fp32's range).
// A row with an infinity or NaN gets scale NaN and codes 0: it reads back as NaN and cannot pass for a finite one.
//
// Reading D values and writing D codes does a few operations a value: DRAM bound, if enough loads are in flight and the two
// correctly rounded quotients of a row, some 20 instructions each, are not formed by all of its lanes.  A group of lanes
// holds eight rows in registers (16 bytes a lane and row, all loaded before the first is used), reduces their eight maxima
// in one transposing tree that leaves row j's in lane j, forms each row's quotients once, in that lane, and passes them round.
// Measured (GPU time, in a captured graph): 8 x 4096 tokens of 8 heads x 128 from bf16 to int8 (203 MB) 41 us, 4.9 TB/s; a state
// of 4 x 4001 rows of 32 heads back from e4m3 to bf16 (397 MB) 68 us, 5.8 TB/s; one step's rows of 32 sequences 2.7 us.
// Listed slots are another matter: every block looks through those of all later tokens, T^2 / 16 reads a sequence.  The first
// case with its slots listed takes 59 us, 32768 tokens of one sequence 181 (contiguous 41), 65536 of 4 heads 631 (61).
#pragma once

#include "tova_device.cuh"

namespace tova {

constexpr int QUANT_THREADS = 256;
constexpr int QUANT_MAX_TOKENS = 8;   // tokens per block

enum : int { FORMAT_PLAIN = 0, FORMAT_INT8 = 1, FORMAT_E4M3 = 2 };

struct QuantParams {
  const void* x[2];            // k, v rows [T,B,Hkv,D], element stride between consecutive (token, sequence) pairs
  void* y[2];                  // reading: where rows go, [T,B,Hkv,D]
  long long x_stride[2];
  void* codes[2];              // [B,Hkv,cap,D]
  float* scale[2];             // [B,Hkv,cap]
  const int32_t* slots;        // [T,B] or NULL: first_slot + token
  int T, B, Hkv, cap, first_slot, tokens_per_block;
};

__device__ __forceinline__ uint32_t quant_pack4_int8(float a, float b, float c, float d) {
  const uint32_t w0 = (uint32_t)__float2int_rn(a), w1 = (uint32_t)__float2int_rn(b);
  const uint32_t w2 = (uint32_t)__float2int_rn(c), w3 = (uint32_t)__float2int_rn(d);
  return __byte_perm(__byte_perm(w0, w1, 0x0040), __byte_perm(w2, w3, 0x0040), 0x5410);
}
__device__ __forceinline__ uint32_t quant_pack4_e4m3(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | ((uint32_t)hi << 16);
}

// Four codes as floats (exact).
template <int FMT>
__device__ __forceinline__ void quant_unpack4(uint32_t w, float (&f)[4]) {
  if constexpr (FMT == FORMAT_INT8) {
    f[0] = (float)(int8_t)(w & 0xff);
    f[1] = (float)(int8_t)((w >> 8) & 0xff);
    f[2] = (float)(int8_t)((w >> 16) & 0xff);
    f[3] = (float)(int8_t)(w >> 24);
  } else {
    uint32_t h01, h23;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h01) : "h"((uint16_t)(w & 0xffff)));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h23) : "h"((uint16_t)(w >> 16)));
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}"
        : "=f"(f[0]), "=f"(f[1]) : "r"(h01));
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}"
        : "=f"(f[2]), "=f"(f[3]) : "r"(h23));
  }
}

// Writing.  grid = (ceil(T / tokens_per_block), B): a block takes all KV heads of some tokens of one sequence.  Slots
// outside 0..cap-1 are skipped.  Where a slot is named twice in a call the later token's row stands: a block looks
// through the tokens behind its own for their slots and leaves out the rows that will be overwritten.
template <typename T, int D, int FMT>
__global__ void __launch_bounds__(QUANT_THREADS) tova_quant_write_kernel(const __grid_constant__ QuantParams p) {
  constexpr int N = Vec16<T>::N;                 // values a lane holds
  constexpr int L = D / N;                       // lanes a row
  constexpr int ROWS = QUANT_THREADS / L;        // rows of a pass
  __shared__ int slot_s[QUANT_MAX_TOKENS];
  const int b = blockIdx.y;
  const int t0 = blockIdx.x * p.tokens_per_block;
  const int n_tok = min(p.tokens_per_block, p.T - t0);
  if (p.slots) {
    if ((int)threadIdx.x < n_tok) slot_s[threadIdx.x] = p.slots[(long long)(t0 + threadIdx.x) * p.B + b];
    __syncthreads();
    int mine[QUANT_MAX_TOKENS];
#pragma unroll
    for (int i = 0; i < QUANT_MAX_TOKENS; ++i) mine[i] = i < n_tok ? slot_s[i] : -1;
    __syncthreads();
    for (int t = t0 + 1 + (int)threadIdx.x; t < p.T; t += QUANT_THREADS) {
      const int s = p.slots[(long long)t * p.B + b];
#pragma unroll
      for (int i = 0; i < QUANT_MAX_TOKENS; ++i)
        if (s == mine[i] && t > t0 + i) slot_s[i] = -1;
    }
  } else if ((int)threadIdx.x < n_tok) {
    slot_s[threadIdx.x] = p.first_slot + t0 + (int)threadIdx.x;
  }
  __syncthreads();
  const int lane = threadIdx.x % L, r0 = threadIdx.x / L;
  const int total = n_tok * p.Hkv;
  const float qmax = FMT == FORMAT_INT8 ? 127.f : 448.f;
  constexpr int U = 4;                           // (token, head) pairs a group holds at a time: U rows of K and U of V
  for (int base = 0; base < total; base += U * ROWS) {
    uint4 w[U][2];
    long long dst[U];                            // row of the state, -1: nothing to write
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = base + u * ROWS + r0;
      const bool in = i < total;
      const int ti = in ? i / p.Hkv : 0, h = in ? i - ti * p.Hkv : 0;
      const int slot = slot_s[ti];
      const bool ok = in && (unsigned)slot < (unsigned)p.cap;
      dst[u] = ok ? ((long long)b * p.Hkv + h) * p.cap + slot : -1;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv)
        w[u][kv] = ok ? __ldcs(reinterpret_cast<const uint4*>(static_cast<const T*>(p.x[kv]) + ((long long)(t0 + ti) * p.B + b) * p.x_stride[kv] +
                                                              (long long)h * D + lane * N))
                      : make_uint4(0, 0, 0, 0);
    }
    uint32_t top[2 * U];     // bits of |x|: ordered like the values, infinities and NaN on top
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        float f[N];
        Vec16<T>::unpack(w[u][kv], f);
        uint32_t t = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) t = max(t, __float_as_uint(f[e]) & 0x7fffffffu);
        top[2 * u + kv] = t;
      }
    // eight maxima over eight lanes: lane j keeps row j's; then over the group's other lanes
#pragma unroll
    for (int half = U; half >= 1; half >>= 1) {
      const bool upper = (lane & half) != 0;
#pragma unroll
      for (int i = 0; i < half; ++i) {
        const uint32_t send = upper ? top[i] : top[i + half], keep = upper ? top[i + half] : top[i];
        top[i] = max(keep, __shfl_xor_sync(0xffffffffu, send, half));
      }
    }
#pragma unroll
    for (int o = 8; o < L; o <<= 1) top[0] = max(top[0], __shfl_xor_sync(0xffffffffu, top[0], o));
    const float a = __uint_as_float(top[0]);
    const bool finite = top[0] < 0x7f800000u, some = finite && a >= 0x1p-100f;
    const float scale_j = some ? __fdiv_rn(a, qmax) : (finite ? 0.f : __uint_as_float(0x7fc00000u));
    const float r_j = some ? __fdiv_rn(qmax, a) : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const int j = (threadIdx.x & 31 & ~7) | (2 * u + kv);
        const float r = __shfl_sync(0xffffffffu, r_j, j), scale = __shfl_sync(0xffffffffu, scale_j, j);
        float f[N];
        Vec16<T>::unpack(w[u][kv], f);
        uint32_t c[N / 4];
#pragma unroll
        for (int e = 0; e < N / 4; ++e) {
          float y[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) y[k] = __fmul_rn(f[4 * e + k], r);
          c[e] = FMT == FORMAT_INT8 ? quant_pack4_int8(y[0], y[1], y[2], y[3]) : quant_pack4_e4m3(y[0], y[1], y[2], y[3]);
          if (r == 0.f) c[e] = 0;                // (0 times an infinity)
        }
        if (dst[u] >= 0) {
          unsigned char* at = static_cast<unsigned char*>(p.codes[kv]) + dst[u] * D + lane * N;
          if constexpr (N == 8) *reinterpret_cast<uint2*>(at) = make_uint2(c[0], c[N / 4 - 1]);
          else *reinterpret_cast<uint32_t*>(at) = c[0];
          if (lane == 0) p.scale[kv][dst[u]] = scale;
        }
      }
  }
}

// Reading back: value = fp32(code scale), rounded once more where the caller's type is bf16.  Same grid; a slot outside
// 0..cap-1 gives a row of zeros.  A lane writes 16 bytes, so that a warp's stores are whole lines; U rows of K and of V are
// on their way at a time.
template <typename T, int D, int FMT>
__global__ void __launch_bounds__(QUANT_THREADS) tova_quant_read_kernel(const __grid_constant__ QuantParams p) {
  constexpr int N = Vec16<T>::N;
  constexpr int L = D / N;
  constexpr int ROWS = QUANT_THREADS / L;
  constexpr int U = 4;
  const int b = blockIdx.y;
  const int t0 = blockIdx.x * p.tokens_per_block;
  const int n_tok = min(p.tokens_per_block, p.T - t0);
  const int lane = threadIdx.x % L;
  const int total = n_tok * p.Hkv;
  for (int base = threadIdx.x / L; base < total; base += U * ROWS) {
    uint2 c[U][2];               // (fp32: the first word)
    float s[U][2];
    long long dst[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = base + u * ROWS;
      const bool in = i < total;
      const int ti = in ? i / p.Hkv : 0, h = in ? i - ti * p.Hkv : 0;
      const long long tb = (long long)(t0 + ti) * p.B + b;
      const int slot = p.slots ? p.slots[tb] : p.first_slot + t0 + ti;
      const bool ok = in && (unsigned)slot < (unsigned)p.cap;
      const long long row = ((long long)b * p.Hkv + h) * p.cap + slot;
      dst[u] = in ? (tb * p.Hkv + h) * D + lane * N : -1;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        c[u][kv] = make_uint2(0, 0);
        s[u][kv] = 0.f;
        if (ok && p.y[kv]) {
          const unsigned char* src = static_cast<const unsigned char*>(p.codes[kv]) + row * D + lane * N;
          if constexpr (N == 8) c[u][kv] = *reinterpret_cast<const uint2*>(src);
          else c[u][kv].x = *reinterpret_cast<const uint32_t*>(src);
          s[u][kv] = p.scale[kv][row];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        if (dst[u] < 0 || p.y[kv] == nullptr) continue;
        const uint32_t w[2] = {c[u][kv].x, c[u][kv].y};
        uint32_t x[4];
#pragma unroll
        for (int e = 0; e < N / 4; ++e) {
          float g[4];
          quant_unpack4<FMT>(w[e], g);
#pragma unroll
          for (int k = 0; k < 4; ++k) g[k] *= s[u][kv];
          if constexpr (N == 8) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const __nv_bfloat162 hh = __floats2bfloat162_rn(g[2 * k], g[2 * k + 1]);
              x[2 * e + k] = *reinterpret_cast<const uint32_t*>(&hh);
            }
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = __float_as_uint(g[k]);
          }
        }
        *reinterpret_cast<uint4*>(static_cast<T*>(p.y[kv]) + dst[u]) = make_uint4(x[0], x[1], x[2], x[3]);
      }
  }
}

}  // namespace tova
