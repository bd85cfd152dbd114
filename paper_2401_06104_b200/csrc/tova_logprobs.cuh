// Log probabilities of given tokens, entropy, the most probable alternatives (sm_100a).
//
// A row x of V logits:  m = max x,  S = sum exp(x - m),  E = sum exp(x - m) (x - m);
//   log p(t) = (x_t - m) - log S,   entropy = log S - E / S,   and the n largest logits, equal ones in the tokens' order.
//
// One pass over the row, in which every thread keeps a maximum, S and E against it, rescaled when the maximum moves; joined at
// the end.  Exponentials are the hardware's approximation (2^-22 relative; the sums' own roundings are of the same size: log p is
// off from 64 bits by 3e-8 to 1e-7 of its size).  A thread that meets an infinity or a NaN forms its share's sums once more, one
// by one.  DRAM bound for many rows.  The n largest need no second pass over the row: they lie in the shares of the n threads
// whose maxima are the largest (of equal ones all, or those whose first such element comes first where they are many), since
// every other thread's elements have n ahead of them.  Those shares, V / threads elements each, are read again by the warps; what
// is no less than the n-th of the maxima is collected and ordered by counting.  Where more is collected than there is room for (rows of equal logits), n
// passes over the shares find one after the other.
//
// Measured (GPU time, in a captured graph): 4095 rows of 64,000 in bf16 (524 MB) 88 us without alternatives, 105 us with five, 128 us
// with 20 (5.9, 5.0 and 4.1 TB/s; 0.90 to 0.62 of the copy rate: behind the pass a block's selection, some 3 us, hardly overlaps the
// others'); 4095 rows of 32,000 in fp32 84 us, 92 with five; one row of 32,000 in fp32 with 20 alternatives 8.5 us.  With logits of
// minus infinity in every thread's share the first takes 233 us, with five alternatives 254 (the last 64 of a row alone: 167, 188),
// 2048 rows of 64,000 in fp32 310 for 84, the one row 9 to 31; with the type's lowest value in their place no longer than without.
//
// A block per row; a cluster of eight blocks where rows are few, each with an eighth of the row, which join in the first
// block's shared memory.
#pragma once

#include "tova_rope.cuh"
#include "tova_tc.cuh"

namespace tova {

constexpr int LOGPROBS_THREADS = 256, LOGPROBS_BLOCKS = 4, LOGPROBS_WARPS = LOGPROBS_THREADS / 32;
constexpr int LOGPROBS_MAX_TOP = 32;
constexpr int LOGPROBS_ROOM = 1024;          // elements collected at most
constexpr int LOGPROBS_SHARES = 64;          // threads' shares read again at most
constexpr int LOGPROBS_CLUSTER = 8;

struct LogprobsParams {
  const void* x;               // [T, V]
  const int32_t* tokens;       // [T]
  float *lp, *entropy;         // [T]; entropy may be NULL
  int32_t* ids;                // [T, top]
  float* top_lp;               // [T, top]
  long long row_stride;
  int T, V, top;
};

// A key that orders logits: larger is earlier.  -0 counts as 0; a NaN comes before everything, and leaves room for a start before
// the first of all (the order of a NaN at token 0 is below ~0).
constexpr uint32_t LOGIT_KEY_NAN = 0xfffffffeu;
__device__ __forceinline__ uint32_t logit_key(float x) {
  if (x != x) return LOGIT_KEY_NAN;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
// The logit of a key (of a NaN: a NaN).
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
// ... with the token: distinct for all elements of a row, never 0 and never ~0.
__device__ __forceinline__ unsigned long long logit_order(uint32_t key, int token) {
  return ((unsigned long long)key << 32) | (0xffffffffu - (uint32_t)token);
}

template <typename T>
__device__ __forceinline__ float logit_at(const T* row, int i) { return (float)row[i]; }

// N neighbouring elements that start at element i (a multiple of N behind the first 16-byte boundary, so i may be negative);
// those outside lo .. hi - 1 are `other`.
template <typename T>
__device__ __forceinline__ void logits_load(const T* row, int i, int lo, int hi, float other, float (&f)[Vec16<T>::N]) {
  constexpr int N = Vec16<T>::N;
  if (i >= lo && i + N <= hi) {
    Vec16<T>::unpack(__ldg(reinterpret_cast<const uint4*>(row + i)), f);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) f[e] = i + e >= lo && i + e < hi ? logit_at(row, i + e) : other;
  }
}

// A 16-byte vector as it lies: two logits as a packed pair of fp32, the largest logit.
__device__ __forceinline__ uint64_t logits_pair(const float*, const uint4& w, int k) {
  return k == 0 ? (uint64_t)w.y << 32 | w.x : (uint64_t)w.w << 32 | w.z;
}
__device__ __forceinline__ uint64_t logits_pair(const __nv_bfloat16*, const uint4& w, int k) {
  const uint32_t x = k == 0 ? w.x : k == 1 ? w.y : k == 2 ? w.z : w.w;
  return (uint64_t)(x & 0xffff0000u) << 32 | x << 16;
}
template <int U>
__device__ __forceinline__ float logits_most(const float*, const uint4 (&w)[U]) {
  float m = __uint_as_float(w[0].x);
#pragma unroll
  for (int u = 0; u < U; ++u)
    m = fmaxf(fmaxf(fmaxf(m, __uint_as_float(w[u].x)), fmaxf(__uint_as_float(w[u].y), __uint_as_float(w[u].z))), __uint_as_float(w[u].w));
  return m;
}
template <int U>
__device__ __forceinline__ float logits_most(const __nv_bfloat16*, const uint4 (&w)[U]) {
  auto h = [](uint32_t x) { return *reinterpret_cast<const __nv_bfloat162*>(&x); };
  __nv_bfloat162 m = h(w[0].x);
#pragma unroll
  for (int u = 0; u < U; ++u) m = __hmax2(m, __hmax2(__hmax2(h(w[u].x), h(w[u].y)), __hmax2(h(w[u].z), h(w[u].w))));
  return fmaxf(__low2float(m), __high2float(m));
}
template <typename T>
struct LogitLowest;            // the lowest finite logit, as it lies in a vector
template <>
struct LogitLowest<float> {
  static constexpr uint32_t word = 0xff7fffffu, value = 0xff7fffffu;
};
template <>
struct LogitLowest<__nv_bfloat16> {
  static constexpr uint32_t word = 0xff7fff7fu, value = 0xff7f0000u;
};

template <typename T, bool CLUSTER>
__global__ void __launch_bounds__(LOGPROBS_THREADS, LOGPROBS_BLOCKS) tova_logprobs_kernel(const __grid_constant__ LogprobsParams p) {
  constexpr int N = Vec16<T>::N, U = 4, TH = LOGPROBS_THREADS;
  __shared__ float red_s[LOGPROBS_WARPS][3];
  __shared__ uint32_t key_s[TH];
  __shared__ int first_s[TH], win_s[LOGPROBS_SHARES];
  __shared__ unsigned long long pool_s[LOGPROBS_ROOM];
  __shared__ unsigned long long best_s[LOGPROBS_MAX_TOP], warp_best_s[LOGPROBS_WARPS];
  __shared__ uint32_t bar_s;
  __shared__ int n_pool, n_above_s, n_win_s;
  __shared__ float all_s[3];
  // what the blocks of a cluster leave in the first one's memory
  __shared__ float peer_red[CLUSTER ? LOGPROBS_CLUSTER : 1][3];
  __shared__ unsigned long long peer_best[CLUSTER ? LOGPROBS_CLUSTER : 1][LOGPROBS_MAX_TOP];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = CLUSTER ? blockIdx.x % LOGPROBS_CLUSTER : 0;
  const int t = CLUSTER ? blockIdx.x / LOGPROBS_CLUSTER : blockIdx.x;
  const T* row = static_cast<const T*>(p.x) + t * p.row_stride;
  const int shift = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));      // elements behind a 16-byte boundary
  // This block's elements lo .. hi - 1; vector k starts at element base + k N.
  int lo = 0, hi = p.V;
  if constexpr (CLUSTER) {
    cluster_arrive_release();                 // (waited for before the first store into another block's memory)
    const int share = ((p.V + shift + N - 1) / N + LOGPROBS_CLUSTER - 1) / LOGPROBS_CLUSTER * N;
    lo = min(p.V, max(0, rank * share - shift));
    hi = min(p.V, max(lo, (rank + 1) * share - shift));
  }
  const int base = lo == 0 ? -shift : lo, n_vec = hi > lo ? (hi - base + N - 1) / N : 0;
  const int top = min(p.top, hi - lo);        // of this block
  constexpr float L2E = 1.4426950408889634f;
  const int tok = p.tokens[t];
  const bool known = tok >= 0 && tok < p.V;
  float chosen = -INFINITY;
  if (tid == 0 && rank == 0 && known) chosen = logit_at(row, tok);

  // --- the pass.  Places that hold no element count as the lowest finite logit, whose weight is 0 unless nothing else is there.
  float m = -INFINITY, s = 0.f, e = 0.f;
  bool nan = false;
  {
    const float lowest = __uint_as_float(LogitLowest<T>::value);
    const T* kind = nullptr;
    const uint64_t l2e_2 = pack_f2(L2E, L2E);
    uint64_t s2 = pack_f2(0.f, 0.f), e2 = s2;
    // A larger maximum: what was summed against the one before is scaled.
    auto raise = [&](float most) {
      if (most > m) {
        if (m != -INFINITY) {
          const float d = m - most, r = ex2_approx(d * L2E);
          e2 = mul_f2(fma_f2(pack_f2(d, d), s2, e2), pack_f2(r, r));
          s2 = mul_f2(s2, pack_f2(r, r));
        }
        m = most;
      }
    };
    const int whole0 = base < lo ? 1 : 0, whole1 = (hi - base) / N;        // vectors that lie in the row
    auto fetch = [&](int k, uint4 (&w)[U]) {
#pragma unroll
      for (int u = 0; u < U; ++u, k += TH) {
        constexpr uint32_t low = LogitLowest<T>::word;
        w[u] = make_uint4(low, low, low, low);
        if (k >= whole0 && k < whole1) w[u] = __ldg(reinterpret_cast<const uint4*>(row + base + k * N));
      }
    };
    auto take = [&](const uint4 (&w)[U]) {
      raise(logits_most(kind, w));
      const uint64_t neg_2 = pack_f2(-m, -m);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int x = 0; x < N / 2; ++x) {
          const uint64_t d = add_f2(logits_pair(kind, w[u], x), neg_2);
          float x0, x1;
          unpack_f2(mul_f2(d, l2e_2), x0, x1);
          const uint64_t wt = pack_f2(ex2_approx(x0), ex2_approx(x1));
          s2 = add_f2(s2, wt);
          e2 = fma_f2(wt, d, e2);
        }
    };
    uint4 wa[U], wb[U];                        // one is on its way while the other is taken
    fetch(tid, wa);
    for (int k = tid; k < n_vec; k += 2 * U * TH) {
      fetch(k + U * TH, wb);
      take(wa);
      fetch(k + 2 * U * TH, wa);
      take(wb);
    }
    // The vectors at the row's ends.
    for (int end = 0; end < 2; ++end) {
      const int k = end ? n_vec - 1 : 0;
      if (k < 0 || k >= n_vec || k % TH != tid || (k >= whole0 && k < whole1) || (end && k == 0)) continue;
      float f[N], most = -INFINITY;
      logits_load<T>(row, base + k * N, lo, hi, lowest, f);
#pragma unroll
      for (int x = 0; x < N; ++x) most = fmaxf(most, f[x]);
      raise(most);
#pragma unroll
      for (int x = 0; x < N; ++x) {
        const float d = f[x] - m, w = ex2_approx(d * L2E);
        s2 = add_f2(s2, pack_f2(w, 0.f));
        e2 = add_f2(e2, pack_f2(w * d, 0.f));
      }
    }
    float a, b;
    unpack_f2(s2, a, b);
    s = a + b;
    unpack_f2(e2, a, b);
    e = a + b;
    // Infinities, NaN and nothing but the lowest logit: once more, one by one.
    if (tid < n_vec && (!(fabsf(e) < INFINITY) || s != s || !(m > lowest))) {
      m = -INFINITY;
      s = e = 0.f;
      for (int pass = 0; pass < 2; ++pass) {
        const float ref = m == -INFINITY ? 0.f : m;
        for (int k = tid; k < n_vec; k += TH) {
          float f[N];
          logits_load<T>(row, base + k * N, lo, hi, -INFINITY, f);
          for (int x = 0; x < N; ++x) {
            if (pass == 0) {
              nan |= f[x] != f[x];
              m = fmaxf(m, f[x]);
            } else {
              const float d = f[x] - ref, w = ex2_approx(d * L2E);
              s += w;
              if (w != 0.f) e = fmaf(w, d, e);
            }
          }
        }
      }
    }
  }
  // --- maxima, sums of the block
  const float mine = m;
  {
    const float wm = warp_max(m);
    const float d = m - (wm == -INFINITY ? 0.f : wm), r = ex2_approx(d * L2E);
    e = warp_sum(r * fmaf(fmaxf(d, -1e30f), s, e));
    s = warp_sum(r * s);
    if (lane == 0) {
      red_s[warp][0] = wm;
      red_s[warp][1] = s;
      red_s[warp][2] = e;
    }
  }
  key_s[tid] = tid < n_vec ? (nan ? LOGIT_KEY_NAN : logit_key(mine)) : 0u;
  if (tid == 0) n_pool = 0;
  __syncthreads();
  // Joins n triples (m, S, E).
  auto join = [&](const float (*red)[3], int n, float* out) {
    float gm = -INFINITY, gs = 0.f, ge = 0.f;
    for (int w = 0; w < n; ++w) gm = fmaxf(gm, red[w][0]);
    const float ref = gm == -INFINITY ? 0.f : gm;
    for (int w = 0; w < n; ++w) {
      const float d = red[w][0] - ref, r = ex2_approx(d * L2E);
      ge += r * fmaf(fmaxf(d, -1e30f), red[w][1], red[w][2]);
      gs += r * red[w][1];
    }
    out[0] = gm;
    out[1] = gs;
    out[2] = ge;
  };
  if (tid == 32) join(red_s, LOGPROBS_WARPS, all_s);

  // --- the n largest of the block, best_s, in order
  const int active = min(TH, n_vec);          // threads with elements
  const int want = min(top, active);
  if (warp == 0 && top > 0) {
    // A bar that `want` of the maxima reach at least, and few more: the want-th of 32, each the largest of eight.
    uint32_t k[TH / 32], most = 0;
#pragma unroll
    for (int i = 0; i < TH / 32; ++i) {
      k[i] = key_s[lane + 32 * i];
      most = max(most, k[i]);
    }
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
      for (int step = size >> 1; step >= 1; step >>= 1) {
        const uint32_t other = __shfl_xor_sync(0xffffffffu, most, step);
        most = ((lane & size) == 0) == ((lane & step) == 0) ? max(most, other) : min(most, other);      // falling
      }
    uint32_t at = __shfl_sync(0xffffffffu, most, want - 1);
    // The threads above it, and those that equal it.
    int n = 0, ties = 0;
    auto count = [&]() {
      n = ties = 0;
#pragma unroll
      for (int i = 0; i < TH / 32; ++i) {
        n += k[i] > at;
        ties += k[i] == at;
      }
      n = __reduce_add_sync(0xffffffffu, n);
      ties = __reduce_add_sync(0xffffffffu, ties);
    };
    count();
    if (n + ties > LOGPROBS_SHARES) {
      // Too many: the want-th largest of all, the largest key that `want` maxima reach, bit by bit.
      at = 0;
      for (int bit = 31; bit >= 0; --bit) {
        const uint32_t test = at | (1u << bit);
        int c = 0;
#pragma unroll
        for (int i = 0; i < TH / 32; ++i) c += k[i] >= test;
        if (__reduce_add_sync(0xffffffffu, c) >= want) at = test;
      }
      count();
    }
    const bool room = n + ties <= LOGPROBS_SHARES;
    int put = 0;
#pragma unroll
    for (int i = 0; i < TH / 32; ++i) {
      const bool in = k[i] > at || (room && k[i] == at);
      const unsigned m = __ballot_sync(0xffffffffu, in);
      if (in) win_s[put + __popc(m & ((1u << lane) - 1u))] = lane + 32 * i;
      put += __popc(m);
    }
    if (lane == 0) {
      bar_s = at;
      n_above_s = n;
      n_win_s = room ? n + ties : 0;
    }
  }
  __syncthreads();
  if (top > 0) {
    const uint32_t bar = bar_s;
    const int per = (n_vec + TH - 1) / TH;              // vectors a thread, at most
    int n_win = n_win_s;
    if (n_win == 0) {
      // Of the threads whose maxima are equal those whose first such element comes first.
      n_win = want;
      const int n_above = n_above_s;
      for (int x = warp; x < TH; x += LOGPROBS_WARPS) {
        if (key_s[x] != bar) {
          if (lane == 0) first_s[x] = 0x7fffffff;
          continue;
        }
        int first = 0x7fffffff;
        for (int j = lane; j < per; j += 32) {
          const int k = x + j * TH;
          if (k >= n_vec) break;
          float f[N];
          logits_load<T>(row, base + k * N, lo, hi, 0.f, f);
#pragma unroll
          for (int y = 0; y < N; ++y) {
            const int i = base + k * N + y;
            if (i >= lo && i < hi && logit_key(f[y]) == bar) first = min(first, i);
          }
          if (first != 0x7fffffff) break;
        }
        first = __reduce_min_sync(0xffffffffu, first);
        if (lane == 0) first_s[x] = first;
      }
      __syncthreads();
      if (key_s[tid] == bar) {
        int before = 0;
        for (int x = 0; x < active; ++x) before += first_s[x] < first_s[tid];
        if (before < want - n_above) win_s[n_above + before] = tid;
      }
      __syncthreads();
    }
    // Their shares once more, two at a time by a warp: what reaches the bar (all of them, where there are fewer threads with
    // elements than elements wanted).
    auto each = [&](auto&& use) {
      for (int w = warp; w < n_win; w += 2 * LOGPROBS_WARPS) {
        for (int j = lane; j < per; j += 32) {
          float f[2][N];
          int first[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const int x = w + y * LOGPROBS_WARPS, k = x < n_win ? win_s[x] + j * TH : n_vec;
            first[y] = k < n_vec ? base + k * N : hi;
            logits_load<T>(row, first[y], lo, hi, 0.f, f[y]);
          }
#pragma unroll
          for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int x = 0; x < N; ++x) {
              const uint32_t key = logit_key(f[y][x]);
              if ((key >= bar || want < top) && first[y] + x >= lo && first[y] + x < hi) use(logit_order(key, first[y] + x));
            }
        }
      }
    };
    each([&](unsigned long long o) {
      const int at = atomicAdd(&n_pool, 1);
      if (at < LOGPROBS_ROOM) pool_s[at] = o;
    });
    __syncthreads();
    const int n = n_pool;
    if (n <= LOGPROBS_ROOM) {
      for (int c = tid; c < n; c += TH) {
        const unsigned long long o = pool_s[c];
        int before = 0;
        for (int x = 0; x < n; ++x) before += pool_s[x] > o;
        if (before < top) best_s[before] = o;
      }
    } else {
      unsigned long long last = ~0ull;
      for (int r = 0; r < top; ++r) {
        unsigned long long o = 0;
        each([&](unsigned long long x) {
          if (x < last && x > o) o = x;
        });
#pragma unroll
        for (int x = 16; x >= 1; x >>= 1) {
          const unsigned long long y = __shfl_xor_sync(0xffffffffu, o, x);
          if (y > o) o = y;
        }
        if (lane == 0) warp_best_s[warp] = o;
        __syncthreads();
        o = 0;
#pragma unroll
        for (int x = 0; x < LOGPROBS_WARPS; ++x)
          if (warp_best_s[x] > o) o = warp_best_s[x];
        if (tid == 0) best_s[r] = o;
        last = o;
        __syncthreads();
      }
    }
    __syncthreads();
  }

  // --- results
  if constexpr (CLUSTER) {
    cluster_wait_acquire();                   // all blocks have started
    auto first_block = [](const void* x) {
      uint32_t a;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_addr(x)), "r"(0));
      return a;
    };
    if (tid < p.top) {
      const unsigned long long o = tid < top ? best_s[tid] : 0ull;
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(first_block(&peer_best[rank][tid])), "l"(o) : "memory");
    }
    if (tid == 0) {
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(first_block(&peer_red[rank][0])), "f"(all_s[0]) : "memory");
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(first_block(&peer_red[rank][1])), "f"(all_s[1]) : "memory");
      asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(first_block(&peer_red[rank][2])), "f"(all_s[2]) : "memory");
    }
    cluster_arrive_release();
    if (rank != 0) return;
    cluster_wait_acquire();
    if (tid == TH - 1) join(peer_red, LOGPROBS_CLUSTER, all_s);
    if (tid < LOGPROBS_CLUSTER * p.top) {
      const unsigned long long o = peer_best[tid / p.top][tid % p.top];
      int before = 0;
      for (int r = 0; r < LOGPROBS_CLUSTER; ++r)
        for (int x = 0; x < p.top; ++x) before += peer_best[r][x] > o;
      if (o != 0 && before < p.top) best_s[before] = o;
    }
    __syncthreads();
  }
  const float gm = all_s[0], gs = all_s[1], ge = all_s[2], ls = logf(gs);
  if (tid == 0) {
    p.lp[t] = (chosen - gm) - ls;
    if (p.entropy) p.entropy[t] = ls - ge / gs;
  }
  if (tid < p.top) {
    const unsigned long long o = best_s[tid];
    p.ids[(long long)t * p.top + tid] = (int)(0xffffffffu - (uint32_t)o);
    p.top_lp[(long long)t * p.top + tid] = (key_logit((uint32_t)(o >> 32)) - gm) - ls;
  }
}

}  // namespace tova
