// Verification of drafted tokens against the target's probabilities, from given random numbers (sm_100a).
//
// A sequence's drafted tokens form a tree (a chain is one): node i carries token x_i and hangs below node parents[i],
// or below the last settled token (the root).  Row 0 of the target's probabilities p is the distribution after the
// root, row 1 + i the one after node i; row r of the draft's probabilities q is the distribution that the children of
// that node were drawn from.  The walk starts at the root.  At a node with target p and draft q its children are
// tried in index order:
//   r_0 = p, Z_0 = 1;   child with token x is accepted when   u Z_j q(x) < r_j(x);
//   rejected:           r_{j+1} = max(0, r_j - Z_j q),  Z_{j+1} = sum of r_{j+1}
// and the walk goes on at the accepted child.  Where no child is accepted the last token is drawn from r (from p where
// r is zero everywhere), by the smallest x whose running sum exceeds u_sample times the whole.  The tokens are then
// distributed as if they had been drawn from p one by one, provided each child was drawn from q.  Unnormalised
// residuals nest: r_j = max(0, p - S_j q) with S_j = Z_0 + ... + Z_{j-1}, so the kernel keeps the scalar S and never
// stores a residual.  Without q the drafts are taken as certain (q = 1 at the child's own token): r_{j+1} is r_j with
// x struck out, Z_{j+1} = Z_j - r_j(x), and no row is read before the last token is drawn.
//
// Every comparison and sum is in 64 bits (u q is exact there), so that the decisions do not depend on the order of
// the sums.  What has to be read is a few scalars along the walk and the rows where a rejection meets another child
// or the walk ends: the time is the latency of a chain of small steps.  One cluster of blocks per sequence: the
// scalars of all nodes are fetched at once at the start, every block walks the same path, and the blocks share out
// the vocabulary where a row has to be summed; partial sums travel through distributed shared memory.  A lane holds
// eight neighbouring entries of the row in registers for as long as the walk stays at the node (vocabularies up to
// 32768 entries), so a second rejection or the final draw there reads nothing, and the draw needs one scan over the
// lanes of the one warp whose stretch holds the goal.  Measured (GPU time): trees of 63 drafts, 32 sequences, 32000 tokens 14 to
// 16 us, about 2.5 us for each row sum along the longest walk; a chain of five, whose walk takes scalars and the last token
// the one sum, 6.5 us.  Larger vocabularies read a row again for every sum, a step at a time: the trees 27 us at 50000 tokens;
// a chain of five 12 us at 128256.
#pragma once

#include <cooperative_groups.h>

#include "tova_device.cuh"

namespace tova {

constexpr int VERIFY_THREADS = 256;
constexpr int VERIFY_WARPS = VERIFY_THREADS / 32;
constexpr int VERIFY_CLUSTER = 8;
constexpr int VERIFY_MAX_NODES = 1024;

struct VerifyParams {
  const void* target;         // [N+1,B,row_stride] probabilities
  const void* draft;          // the same layout, or NULL
  const int32_t* tokens;      // [N,B]
  const int32_t* parents;     // [N,B] or NULL: a chain
  const float* u;             // [N,B]
  const float* u_sample;      // [B]
  int32_t* n_accepted;        // [B]
  int32_t* path;              // [N,B] or NULL
  int32_t* tokens_out;        // [N+1,B]
  long long row_stride;
  int B, N, V;
  int vec;                    // rows start on 16-byte boundaries
};

// Dynamic shared memory: per node p(x), q(x), u (floats), token, parent, and a list of tokens.
inline size_t verify_smem_bytes(int N) { return (size_t)N * 24; }

template <typename T>
__device__ __forceinline__ float verify_load(const void* p, long long i) {
  return (float)static_cast<const T*>(p)[i];
}

constexpr int VERIFY_LANE = 8;                     // entries a lane takes at a time
constexpr int VERIFY_STEP = 32 * VERIFY_LANE;      // ... and a warp
constexpr int VERIFY_HELD = 2;                     // steps of a warp that are held in registers

// Eight entries i .. i+7 of a row, zeros from `end` on.
template <typename T>
__device__ __forceinline__ void verify_load8(const void* p, long long row, int i, int end, bool vec, float (&f)[VERIFY_LANE]) {
  const T* x = static_cast<const T*>(p) + row + i;
  if (vec && i + VERIFY_LANE <= end) {
    constexpr int N = Vec16<T>::N;
#pragma unroll
    for (int k = 0; k < VERIFY_LANE / N; ++k) {
      float g[N];
      Vec16<T>::unpack(*reinterpret_cast<const uint4*>(x + k * N), g);
#pragma unroll
      for (int e = 0; e < N; ++e) f[k * N + e] = g[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < VERIFY_LANE; ++e) f[e] = i + e < end ? (float)x[e] : 0.f;
  }
}

// A probability that counts: an entry of p that is an infinity or NaN is none, and negative ones are none either.  (The bits
// of positive finite numbers, and of 0, are the smallest.)
__device__ __forceinline__ double verify_prob(float p) { return __float_as_uint(p) < 0x7f800000u ? (double)p : 0.0; }

// The weight that the last token is drawn with, or a term of Z: max(0, p - S q).  Where p or q is not finite it is zero, so
// that every sum is finite and the draw always finds a token where there is one.  (One integer comparison of the high word, in
// place of two of 64 bits.)
__device__ __forceinline__ double verify_weight(float p, float q, double S) {
  const double w = (double)p - S * (double)q;
  return (uint32_t)__double2hiint(w) < 0x7ff00000u ? w : 0.0;
}

template <typename T>
__global__ void __launch_bounds__(VERIFY_THREADS, 2) tova_verify_kernel(const __grid_constant__ VerifyParams p) {
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  extern __shared__ __align__(16) unsigned char verify_smem[];
  float* px_s = reinterpret_cast<float*>(verify_smem);
  float* qx_s = px_s + p.N;
  float* u_s = qx_s + p.N;
  int* tok_s = reinterpret_cast<int*>(u_s + p.N);
  int* par_s = tok_s + p.N;
  int* kid_s = par_s + p.N;                       // without q: tokens of the last node's children
  __shared__ double inbox[2][VERIFY_CLUSTER];     // partial sums of the cluster's blocks, double-buffered
  __shared__ double warp_part[VERIFY_WARPS];
  __shared__ int cmd_s, node_s, count_s, last_child_s, kids_s;
  __shared__ double S_s;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.y;
  const int rank = (int)cluster.block_rank(), nc = (int)cluster.num_blocks();
  const int N = p.N, V = p.V;

  for (int i = tid; i < N; i += VERIFY_THREADS) {
    const long long at = (long long)i * p.B + b;
    int par = p.parents ? p.parents[at] : i - 1;
    if (par < -1 || par >= i) par = -2;                       // padding: never reached
    const int tok = p.tokens[at];
    const bool ok = par >= -1 && (unsigned)tok < (unsigned)V;
    const long long row = ((long long)(par + 1) * p.B + b) * p.row_stride;
    par_s[i] = par;
    tok_s[i] = tok;
    u_s[i] = p.u[at];
    px_s[i] = ok ? verify_load<T>(p.target, row + tok) : 0.f;   // a token outside the vocabulary is never accepted
    qx_s[i] = ok ? (p.draft ? verify_load<T>(p.draft, row + tok) : 1.f) : 0.f;
  }
  if (tid == 0) { kids_s = 0; node_s = -1; count_s = 0; last_child_s = -1; S_s = 0.0; cmd_s = 0; }
  cluster.sync();     // every block of the cluster runs before any writes into another's inbox

  // This block's share of the vocabulary, and every warp's share of that: contiguous, in order.
  const int per_block = ((V + nc - 1) / nc + VERIFY_LANE - 1) / VERIFY_LANE * VERIFY_LANE;
  const int v0 = min(V, rank * per_block), v1 = min(V, v0 + per_block);
  const int per_warp = ((per_block + VERIFY_WARPS - 1) / VERIFY_WARPS + VERIFY_STEP - 1) / VERIFY_STEP * VERIFY_STEP;
  const int w0 = min(v1, v0 + warp * per_warp), w1 = min(v1, w0 + per_warp);
  const int steps = per_warp / VERIFY_STEP;
  const bool held = steps <= VERIFY_HELD;
  float pr[VERIFY_HELD][VERIFY_LANE], qr[VERIFY_HELD][VERIFY_LANE];     // this lane's entries of the node's row
  int held_node = -2;
  // This lane's entries of step k: from registers, or fetched.
  auto fetch = [&](long long row, int k, bool with_q, float (&a)[VERIFY_LANE], float (&b)[VERIFY_LANE]) {
    const int i = w0 + k * VERIFY_STEP + lane * VERIFY_LANE;
    verify_load8<T>(p.target, row, i, w1, p.vec, a);
    if (with_q) verify_load8<T>(p.draft, row, i, w1, p.vec, b);
  };
  auto hold = [&](int node, bool with_q) {
    if (!held || held_node == node) return;
    const long long row = ((long long)(node + 1) * p.B + b) * p.row_stride;
#pragma unroll
    for (int k = 0; k < VERIFY_HELD; ++k)
      if (k < steps) fetch(row, k, with_q, pr[k], qr[k]);
    held_node = node;
  };
  // f(k, p entries, q entries) for every step of the warp.
  auto each_step = [&](int node, bool with_q, auto f) {
    if (held) {
      hold(node, with_q);
#pragma unroll
      for (int k = 0; k < VERIFY_HELD; ++k)
        if (k < steps) f(k, pr[k], qr[k]);
    } else {
      const long long row = ((long long)(node + 1) * p.B + b) * p.row_stride;
      for (int k = 0; k < steps; ++k) {
        fetch(row, k, with_q, pr[0], qr[0]);
        f(k, pr[0], qr[0]);
      }
    }
  };

  int turn = 0;                       // exchanges so far
  // The sum over the cluster of one value per thread, in a fixed order; the block's prefix before this warp and the
  // cluster's before this block come with it.
  auto cluster_sum = [&](double x, double& before_block, double& before_warp) -> double {
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (lane == 0) warp_part[warp] = x;
    __syncthreads();
    double block = 0.0;
    before_warp = 0.0;
    for (int i = 0; i < VERIFY_WARPS; ++i) {
      if (i == warp) before_warp = block;
      block += warp_part[i];
    }
    if (tid < nc) *cluster.map_shared_rank(&inbox[turn & 1][rank], tid) = block;
    cluster.sync();
    double all = 0.0;
    before_block = 0.0;
    for (int i = 0; i < nc; ++i) {
      if (i == rank) before_block = all;
      all += inbox[turn & 1][i];
    }
    ++turn;
    return all;
  };

  double Z = 1.0;
  for (;;) {
    // Warp 0 walks until a row's sum is needed (cmd 1) or the walk ends (cmd 2); every block does the same steps.
    if (warp == 0) {
      int node = node_s, count = count_s, from = last_child_s + 1;
      double S = S_s;
      int cmd = 0;
      if (from < node + 1) from = node + 1;     // children come after their parent
      auto next_child = [&](int start) {
        for (int i0 = start; i0 < N; i0 += 32) {
          const int i = i0 + lane;
          const unsigned m = __ballot_sync(0xffffffffu, i < N && par_s[i] == node);
          if (m) return i0 + __ffs(m) - 1;
        }
        return -1;
      };
      int c = next_child(from);
      while (cmd == 0) {
        if (c < 0) { cmd = 2; break; }
        const double qr = (double)qx_s[c];
        double r;
        if (p.draft) {
          r = verify_weight(px_s[c], qx_s[c], S);
        } else {                                 // struck out if an earlier child carried the same token
          bool again = false;
          for (int i = node + 1 + lane; i < c; i += 32) again |= par_s[i] == node && tok_s[i] == tok_s[c];
          r = __any_sync(0xffffffffu, again) ? 0.0 : verify_prob(px_s[c]);
        }
        if (r > 0.0 && (double)u_s[c] * qr * Z < r) {      // (a negative q must not pass a token without probability)
          if (rank == 0 && lane == 0) {
            if (p.path) p.path[(long long)count * p.B + b] = c;
            p.tokens_out[(long long)count * p.B + b] = tok_s[c];
          }
          ++count;
          node = c;
          S = 0.0;
          Z = 1.0;
          c = next_child(c + 1);
          continue;
        }
        const int more = next_child(c + 1);
        if (p.draft) {
          S += Z;
          if (more >= 0) cmd = 1;
          from = c;                              // the child just rejected
        } else {
          Z -= r;
        }
        if (cmd == 0) c = more;
      }
      __syncwarp();
      if (lane == 0) { cmd_s = cmd; node_s = node; count_s = count; last_child_s = from; S_s = S; }
    }
    __syncthreads();
    if (cmd_s == 2) break;
    const double S = S_s;
    double sum = 0.0, bb, bw;
    each_step(node_s, true, [&](int, const float (&a)[VERIFY_LANE], const float (&q)[VERIFY_LANE]) {
#pragma unroll
      for (int e = 0; e < VERIFY_LANE; ++e) sum += verify_weight(a[e], q[e], S);
    });
    Z = cluster_sum(sum, bb, bw);
    __syncthreads();
  }

  // The last token.
  const int node = node_s, count = count_s;
  const double S = S_s;
  const bool with_q = p.draft != nullptr && S > 0.0;     // (nothing rejected here: r is p)
  if (!p.draft) {                // tokens of the node's children, all rejected: struck out
    for (int i = node + 1 + tid; i < N; i += VERIFY_THREADS)
      if (par_s[i] == node) kid_s[atomicAdd(&kids_s, 1)] = tok_s[i];      // (in any order: they are only compared with)
    __syncthreads();
  }
  const int kids = kids_s;
  bool plain = false;            // r was zero everywhere: drawn from p
  double before_block = 0.0, before_warp = 0.0, all = 0.0, mine = 0.0;
  auto weights = [&](int k, const float (&a)[VERIFY_LANE], const float (&q)[VERIFY_LANE], double (&w)[VERIFY_LANE]) {
    const int i = w0 + k * VERIFY_STEP + lane * VERIFY_LANE;
#pragma unroll
    for (int e = 0; e < VERIFY_LANE; ++e) {
      w[e] = with_q && !plain ? verify_weight(a[e], q[e], S) : verify_prob(a[e]);
      if (!plain)
        for (int j = 0; j < kids; ++j)
          if (kid_s[j] == i + e) w[e] = 0.0;
    }
  };
  for (;;) {
    double sum = 0.0;
    each_step(node, with_q, [&](int k, const float (&a)[VERIFY_LANE], const float (&q)[VERIFY_LANE]) {
      double w[VERIFY_LANE];
      weights(k, a, q, w);
#pragma unroll
      for (int e = 0; e < VERIFY_LANE; ++e) sum += w[e];
    });
    mine = sum;
    all = cluster_sum(sum, before_block, before_warp);
    if (all > 0.0 || plain) break;
    __syncthreads();
    plain = true;
  }
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  // The warp whose stretch of the running sum holds the goal: the running sum before it is not above, the one after it
  // is.  The prefixes are added up the same way in every warp, so exactly one warp finds it (the goal lies below the
  // whole).
  float us = p.u_sample[b];
  us = us >= 0.f ? fminf(us, 0x1.fffffep-1f) : 0.f;
  const double goal = (double)us * all;
  const double lo = before_block + before_warp, hi = before_block + (before_warp + mine);
  if (mine > 0.0 && lo <= goal && goal < hi) {
    double run = lo;
    int found = -1, last_some = -1;
    each_step(node, with_q, [&](int k, const float (&a)[VERIFY_LANE], const float (&q)[VERIFY_LANE]) {
      if (found >= 0) return;
      double w[VERIFY_LANE], own = 0.0;
      weights(k, a, q, w);
#pragma unroll
      for (int e = 0; e < VERIFY_LANE; ++e) own += w[e];
      double inc = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      // this lane's entry at which the running sum passes the goal, and its last one that has any weight
      int at = -1, some = -1;
      double x = run + (inc - own);
#pragma unroll
      for (int e = 0; e < VERIFY_LANE; ++e) {
        x += w[e];
        if (w[e] > 0.0) {
          some = e;
          if (at < 0 && x > goal) at = e;
        }
      }
      const int i = w0 + k * VERIFY_STEP + lane * VERIFY_LANE;
      const unsigned m = __ballot_sync(0xffffffffu, at >= 0), n = __ballot_sync(0xffffffffu, some >= 0);
      if (m) found = __shfl_sync(0xffffffffu, i + at, __ffs(m) - 1);
      if (n) last_some = __shfl_sync(0xffffffffu, i + some, 31 - __clz(n));
      run += __shfl_sync(0xffffffffu, inc, 31);
    });
    if (found < 0) found = last_some;     // the stretch's sum in another order fell short of the goal
    if (lane == 0) p.tokens_out[(long long)count * p.B + b] = found;
  }
  if (rank == 0) {
    if (tid == 0) {
      p.n_accepted[b] = count;
      if (!(all > 0.0)) p.tokens_out[(long long)count * p.B + b] = -1;    // no probability anywhere
    }
    for (int i = count + tid; i < N; i += VERIFY_THREADS) {
      if (p.path) p.path[(long long)i * p.B + b] = -1;
      p.tokens_out[(long long)(i + 1) * p.B + b] = -1;
    }
  }
  // (No block writes into another's inbox behind the last exchange, so none has to wait for the others to leave.)
}

}  // namespace tova
