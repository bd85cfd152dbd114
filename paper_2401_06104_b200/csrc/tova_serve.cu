// Host side of the operators for sequences of different lengths declared in include/tova.h: norms with the rotation, a state
// in pages, attention of packed prompts, log probabilities.  Argument checks and launches; the work runs in the kernels of
// tova_norm_rope.cuh, tova_paged.cuh, tova_packed.cuh and tova_logprobs.cuh.
#include "../../include/tova.h"

#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "tova_host.cuh"
#include "tova_logprobs.cuh"
#include "tova_norm_rope.cuh"
#include "tova_packed.cuh"
#include "tova_packed_tc.cuh"
#include "tova_paged.cuh"

namespace {

// Launches `kern`; dependent: it may start while its predecessor in the stream ends (it waits for it itself).
template <typename... Args>
cudaError_t start(void (*kern)(Args...), dim3 grid, int threads, size_t smem, int cluster, bool dependent, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t lc{};
  lc.gridDim = grid;
  lc.blockDim = dim3((unsigned)threads);
  lc.dynamicSmemBytes = smem;
  lc.stream = st;
  cudaLaunchAttribute at[2];
  int n = 0;
  if (cluster > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = (unsigned)cluster;
    at[n].val.clusterDim.y = 1;
    at[n].val.clusterDim.z = 1;
    ++n;
  }
  if (dependent) {
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  lc.attrs = at;
  lc.numAttrs = n;
  return cudaLaunchKernelEx(&lc, kern, args...);
}

// Lets `kern` use `smem` bytes of dynamic shared memory on the current device (once per device; `done` is the kernel's own).
template <typename... Args>
cudaError_t allow_smem(void (*kern)(Args...), std::atomic<bool>* done, size_t smem) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 64 && done[dev].load(std::memory_order_acquire)) return cudaSuccess;
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess && dev < 64) done[dev].store(true, std::memory_order_release);
  return e;
}

inline size_t round_up(size_t x, size_t to) { return (x + to - 1) / to * to; }

}  // namespace

// ---------------------------------------------------------------------------
// Norms with the rotation
// ---------------------------------------------------------------------------
namespace {

// Blocks of the gradient's kernel: as many as are resident at a time, none without tokens; even shares of the tokens.
long long norm_back_blocks(const tova_rope_config& c, int32_t n_tokens, int sm_count, int* tokens_per_block) {
  const long long rows = (long long)n_tokens * c.batch, most = (long long)tova::NORM_BACK_BLOCKS * sm_count;
  *tokens_per_block = (int)((rows + most - 1) / most);
  return rows == 0 ? 0 : (rows + *tokens_per_block - 1) / *tokens_per_block;
}

template <typename T, int D>
cudaError_t norm_launch(const tova::NormRopeParams& p, const tova_rope_config& c, bool back, unsigned grid, cudaStream_t st) {
  constexpr int TH = tova::NORM_THREADS, TB = tova::NORM_BACK_THREADS, N = tova::Vec16<T>::N;
  const int mode = c.layout == TOVA_ROPE_INTERLEAVED ? tova::NORM_INTERLEAVED
                   : c.rotary_dim == c.head_dim      ? tova::NORM_HALF
                   : (c.rotary_dim / 2) % N == 0     ? tova::NORM_HALF_PART
                                                     : tova::NORM_HALF_ODD;
#define TOVA_NORM_GO(M)                                                                    \
  if (back) tova::tova_norm_rope_back_kernel<T, D, M><<<grid, TB, 0, st>>>(p);             \
  else tova::tova_norm_rope_kernel<T, D, M><<<grid, TH, 0, st>>>(p);
  if (mode == tova::NORM_HALF) {
    TOVA_NORM_GO(tova::NORM_HALF)
  } else if (mode == tova::NORM_INTERLEAVED) {
    TOVA_NORM_GO(tova::NORM_INTERLEAVED)
  } else if (mode == tova::NORM_HALF_PART) {
    TOVA_NORM_GO(tova::NORM_HALF_PART)
  } else {
    TOVA_NORM_GO(tova::NORM_HALF_ODD)
  }
#undef TOVA_NORM_GO
  return cudaGetLastError();
}
cudaError_t norm_run(const tova::NormRopeParams& p, const tova_rope_config& c, bool back, unsigned grid, cudaStream_t st) {
  if (c.dtype == TOVA_DTYPE_BF16)
    return c.head_dim == 128 ? norm_launch<__nv_bfloat16, 128>(p, c, back, grid, st) : norm_launch<__nv_bfloat16, 64>(p, c, back, grid, st);
  return c.head_dim == 128 ? norm_launch<float, 128>(p, c, back, grid, st) : norm_launch<float, 64>(p, c, back, grid, st);
}

void norm_fill(tova::NormRopeParams& p, const tova_rope* r, int32_t n_tokens, const int32_t* positions, int32_t first_pos, bool k, float eps,
               const void* qw, const void* kw) {
  const tova_rope_config& c = r->cfg;
  p.heads[0] = c.n_q_heads;
  p.heads[1] = k ? c.n_kv_heads : 0;
  const int heads[3] = {p.heads[0], p.heads[1], p.heads[0] + p.heads[1]};
  for (int i = 0; i < 3; ++i) p.magic[i] = heads[i] > 1 ? (unsigned)(((1ull << 32) + heads[i] - 1) / heads[i]) : 0;
  p.w[0] = qw; p.w[1] = kw;
  p.positions = positions;
  p.rows = (long long)n_tokens * c.batch;
  p.first_pos = first_pos;
  p.B = c.batch; p.rot = c.rotary_dim;
  p.factor = r->factor;
  p.eps = eps;
  std::copy(r->turns, r->turns + tova::ROPE_MAX_PAIRS, p.turns);
}

}  // namespace

extern "C" int tova_norm_rope_apply(const tova_rope* r, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                    const void* q_weight, const void* k_weight, float eps, int32_t n_tokens, const int32_t* positions,
                                    int32_t first_pos, void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride,
                                    void* cuda_stream) {
  if (!r) return TOVA_ERR_NULL;
  const tova_rope_config& c = r->cfg;
  if (n_tokens < 0 || !(eps >= 0.f) || !std::isfinite(eps)) return TOVA_ERR_BAD_SHAPE;
  if (n_tokens == 0) return TOVA_OK;
  if (!q || !q_out || (k == nullptr) != (k_out == nullptr)) return TOVA_ERR_NULL;
  const size_t E = dtype_bytes(c.dtype);
  const int64_t qr = (int64_t)c.n_q_heads * c.head_dim, kr = (int64_t)c.n_kv_heads * c.head_dim;
  if (!aligned16(q) || !aligned16(q_out) || !aligned16(k) || !aligned16(k_out) || !aligned16(q_weight) || !aligned16(k_weight)) return TOVA_ERR_ALIGN;
  if (q_stride < 0 || k_stride < 0 || q_out_stride < 0 || k_out_stride < 0) return TOVA_ERR_BAD_SHAPE;
  if (!stride_ok(q_stride, qr, E) || !stride_ok(q_out_stride, qr, E) || !stride_ok(k_stride, kr, E) || !stride_ok(k_out_stride, kr, E))
    return TOVA_ERR_ALIGN;
  if (!positions && (int64_t)first_pos + n_tokens - 1 > INT32_MAX) return TOVA_ERR_BAD_SHAPE;
  DeviceInfo dev;
  if (!device_info(&dev)) return TOVA_ERR_CUDA;
  tova::NormRopeParams p{};
  norm_fill(p, r, n_tokens, positions, first_pos, k != nullptr, eps, q_weight, k_weight);
  p.x[0] = q; p.x[1] = k; p.y[0] = q_out; p.y[1] = k_out;
  p.x_stride[0] = q_stride; p.x_stride[1] = k_stride;
  p.y_stride[0] = q_out_stride; p.y_stride[1] = k_out_stride;
  // One token per block while that leaves SMs idle; several share the set-up of a block beyond that.
  p.tokens_per_block = (int)std::min<long long>(tova::NORM_MAX_TOKENS, std::max<long long>(1, p.rows / (8LL * dev.sm_count)));
  const long long blocks = (p.rows + p.tokens_per_block - 1) / p.tokens_per_block;
  if (blocks > INT32_MAX) return TOVA_ERR_BAD_SHAPE;
  return launched(norm_run(p, c, false, (unsigned)blocks, static_cast<cudaStream_t>(cuda_stream)));
}

extern "C" size_t tova_norm_rope_workspace_bytes(const tova_rope* r, int32_t n_tokens) {
  DeviceInfo dev;
  if (!r || n_tokens < 0 || !device_info(&dev)) return (size_t)-1;
  // (for every number of tokens up to this one: there may be more blocks for fewer tokens, never more than are resident)
  return (size_t)std::min<long long>((long long)tova::NORM_BACK_BLOCKS * dev.sm_count, (long long)n_tokens * r->cfg.batch) * 2 * r->cfg.head_dim * sizeof(float);
}

extern "C" int tova_norm_rope_backward(const tova_rope* r, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                       const void* q_weight, const void* k_weight, float eps, int32_t n_tokens,
                                       const int32_t* positions, int32_t first_pos, const void* dq_out, int64_t dq_out_stride,
                                       const void* dk_out, int64_t dk_out_stride, void* dq, int64_t dq_stride, void* dk,
                                       int64_t dk_stride, float* dq_weight, float* dk_weight, void* workspace,
                                       size_t workspace_bytes, void* cuda_stream) {
  if (!r) return TOVA_ERR_NULL;
  const tova_rope_config& c = r->cfg;
  if (n_tokens < 0 || !(eps >= 0.f) || !std::isfinite(eps)) return TOVA_ERR_BAD_SHAPE;
  const bool keys = k != nullptr;
  if (n_tokens > 0 && (!q || !dq_out || !dq || keys != (dk_out != nullptr) || keys != (dk != nullptr))) return TOVA_ERR_NULL;
  const size_t E = dtype_bytes(c.dtype);
  const int64_t qr = (int64_t)c.n_q_heads * c.head_dim, kr = (int64_t)c.n_kv_heads * c.head_dim;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_weight) || !aligned16(k_weight) || !aligned16(dq_out) || !aligned16(dk_out) ||
      !aligned16(dq) || !aligned16(dk) || !aligned16(dq_weight) || !aligned16(dk_weight) || !aligned16(workspace))
    return TOVA_ERR_ALIGN;
  if (q_stride < 0 || k_stride < 0 || dq_out_stride < 0 || dk_out_stride < 0 || dq_stride < 0 || dk_stride < 0) return TOVA_ERR_BAD_SHAPE;
  if (!stride_ok(q_stride, qr, E) || !stride_ok(dq_out_stride, qr, E) || !stride_ok(dq_stride, qr, E) || !stride_ok(k_stride, kr, E) ||
      !stride_ok(dk_out_stride, kr, E) || !stride_ok(dk_stride, kr, E))
    return TOVA_ERR_ALIGN;
  if (!positions && n_tokens > 0 && (int64_t)first_pos + n_tokens - 1 > INT32_MAX) return TOVA_ERR_BAD_SHAPE;
  DeviceInfo dev;
  if (!device_info(&dev)) return TOVA_ERR_CUDA;
  tova::NormRopeParams p{};
  const long long blocks = norm_back_blocks(c, n_tokens, dev.sm_count, &p.tokens_per_block);
  const size_t need = (size_t)blocks * 2 * c.head_dim * sizeof(float);
  if (need > 0 && !workspace) return TOVA_ERR_NULL;
  if (workspace_bytes < need) return TOVA_ERR_WORKSPACE;
  norm_fill(p, r, n_tokens, positions, first_pos, keys, eps, q_weight, k_weight);
  p.x[0] = q; p.x[1] = k; p.dy[0] = dq_out; p.dy[1] = dk_out; p.y[0] = dq; p.y[1] = dk;
  p.x_stride[0] = q_stride; p.x_stride[1] = k_stride;
  p.dy_stride[0] = dq_out_stride; p.dy_stride[1] = dk_out_stride;
  p.y_stride[0] = dq_stride; p.y_stride[1] = dk_stride;
  p.dw_part = static_cast<float*>(workspace);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (blocks > 0)
    if (int rc = launched(norm_run(p, c, true, (unsigned)blocks, st))) return rc;
  if (!dq_weight && !dk_weight) return TOVA_OK;
  return launched(start(tova::tova_norm_rope_weights_kernel, dim3((unsigned)c.head_dim / 32, 2), 1024, 0, 1, blocks > 0, st,
                        (const float*)p.dw_part, (int)blocks, (int)c.head_dim, dq_weight, dk_weight));
}

// ---------------------------------------------------------------------------
// A state in pages
// ---------------------------------------------------------------------------
namespace {

int paged_check(const tova_paged_config* c) {
  if (!c) return TOVA_ERR_NULL;
  if (!heads_ok(c->batch, c->n_q_heads, c->n_kv_heads) || c->n_pages < 1 || c->max_pages < 1 || c->page_rows < 1 || c->page_rows > (1 << 15) ||
      (c->page_rows & (c->page_rows - 1)) != 0 || !(c->sm_scale >= 0.f) || !std::isfinite(c->sm_scale))
    return TOVA_ERR_BAD_SHAPE;
  if ((c->head_dim != 64 && c->head_dim != 128) || !known_dtype(c->dtype)) return TOVA_ERR_UNSUPPORTED;
  return TOVA_OK;
}
// Rows that a call may be bounded by: the table's, at most 2^30 (row numbers and what is added to them stay below 2^31).
bool paged_bound_ok(const tova_paged_config& c, int32_t n_live) {
  return n_live >= 0 && n_live <= (1 << 30) && n_live <= (long long)c.max_pages * c.page_rows;
}
int paged_shift(const tova_paged_config& c) {
  int s = 0;
  while ((1 << s) < c.page_rows) ++s;
  return s;
}

// How a call's rows are dealt out.
struct PagedPlan {
  int heads, hgroups, jobs;        // query heads a block takes, groups of them in a KV head, jobs of a sequence
  int splits;                      // > 0: a cluster of so many blocks a job; 0: even shares
  int blocks, least;
  bool wide_join;                  // many parts a job
  size_t acc_bytes, ml_bytes, bytes;
};
PagedPlan paged_plan(const tova_paged_config& c, int32_t n_live, int sm_count, bool up_to = false) {
  PagedPlan t{};
  const int G = c.n_q_heads / c.n_kv_heads;
  const bool bf16 = c.dtype == TOVA_DTYPE_BF16;
  t.heads = bf16 ? (G <= 8 ? 8 : 16) : (G == 1 ? 1 : G == 2 ? 2 : 4);
  t.hgroups = (G + t.heads - 1) / t.heads;
  t.jobs = c.n_kv_heads * t.hgroups;
  const long long jobs = (long long)c.batch * t.jobs, units = (n_live + tova::PAGED_UNIT - 1) / tova::PAGED_UNIT;
  const int resident = sm_count * (bf16 ? (t.heads == 8 ? 3 : 2) : t.heads == 4 ? 2 : 3);
  // Clusters, a job each, as wide as the GPU has room for, up to eight blocks: where a block has four units at most (two launches
  // take longer), or where all jobs fill the GPU that way and no block has more than 32 (with lengths that differ, even shares are
  // as fast from there on, and far faster where a few sequences are much longer than the others).  Measured, us by clusters / by
  // shares, 8 KV heads x 128: 1 x 1000 rows 7.4 / 10.6, 4 x 4000 17.4 / 20.7, 16 x 1000 17.0 / 20.9, 16 x 4000 46 / 51,
  // 64 x up to 2000 59 / 63, 64 x up to 8192 223 / 219; 1 x 8000 23 / 16.
  const long long wide = std::min<long long>(8, std::max<long long>(1, std::min<long long>(units, resident / std::max<long long>(1, jobs))));
  if (jobs <= 65535 && (units <= 4 * wide || (4 * jobs * wide >= 3LL * resident && units <= 32 * wide))) t.splits = (int)wide;
  t.least = 4;
  if (t.splits == 0 || up_to) {
    t.blocks = (int)std::min<long long>(resident, std::max<long long>(1, jobs * std::max<long long>(1, units)));
    t.acc_bytes = (size_t)t.blocks * 2 * t.heads * c.head_dim * sizeof(float);
    t.ml_bytes = (size_t)t.blocks * 2 * t.heads * sizeof(float2);
    t.bytes = t.acc_bytes + t.ml_bytes + round_up((size_t)jobs * sizeof(tova::PagedCut), 16);
    t.wide_join = t.blocks > 4 * jobs;
  }
  return t;
}

template <typename Core>
cudaError_t paged_launch(const tova::PagedParams& p, const PagedPlan& t, cudaStream_t st) {
  if (t.splits > 0)
    return start(tova::tova_paged_kernel<Core, true>, dim3((unsigned)t.splits, (unsigned)(p.B * p.jobs)), tova::PAGED_THREADS, 0, t.splits, false, st, p);
  cudaError_t e = start(tova::tova_paged_kernel<Core, false>, dim3((unsigned)t.blocks), tova::PAGED_THREADS, 0, 1, false, st, p);
  if (e != cudaSuccess) return e;
  const unsigned jobs = (unsigned)(p.B * p.jobs);
  if (t.wide_join) return start(tova::tova_paged_join_kernel<Core, true>, dim3(jobs, Core::HEADS), tova::PAGED_JOIN_THREADS, 0, 1, true, st, p);
  return start(tova::tova_paged_join_kernel<Core, false>, dim3(jobs, (Core::HEADS + 7) / 8), tova::PAGED_JOIN_THREADS, 0, 1, true, st, p);
}
template <int D>
cudaError_t paged_run(const tova::PagedParams& p, const PagedPlan& t, bool bf16, cudaStream_t st) {
  if (bf16) {
    if (t.heads == 8) return p.shift >= 4 ? paged_launch<tova::PagedMma<D, 1, false>>(p, t, st) : paged_launch<tova::PagedMma<D, 1, true>>(p, t, st);
    return p.shift >= 4 ? paged_launch<tova::PagedMma<D, 2, false>>(p, t, st) : paged_launch<tova::PagedMma<D, 2, true>>(p, t, st);
  }
  return t.heads == 1   ? paged_launch<tova::PagedAlu<D, 1>>(p, t, st)
         : t.heads == 2 ? paged_launch<tova::PagedAlu<D, 2>>(p, t, st)
                        : paged_launch<tova::PagedAlu<D, 4>>(p, t, st);
}

}  // namespace

extern "C" int tova_paged_write(const tova_paged_config* cfg, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                int32_t n_tokens, const int32_t* offsets, const int32_t* first_rows, const int32_t* page_table,
                                void* K, void* V, void* cuda_stream) {
  if (int rc = paged_check(cfg)) return rc;
  if (n_tokens < 0 || (!offsets && n_tokens > cfg->batch)) return TOVA_ERR_BAD_SHAPE;
  if (n_tokens == 0) return TOVA_OK;
  if (!k || !v || !K || !V || !page_table) return TOVA_ERR_NULL;
  if (!aligned16(k) || !aligned16(v) || !aligned16(K) || !aligned16(V)) return TOVA_ERR_ALIGN;
  if (k_stride < 0 || v_stride < 0) return TOVA_ERR_BAD_SHAPE;
  const size_t E = dtype_bytes(cfg->dtype);
  const int64_t row = (int64_t)cfg->n_kv_heads * cfg->head_dim;
  if (!stride_ok(k_stride, row, E) || !stride_ok(v_stride, row, E)) return TOVA_ERR_ALIGN;
  DeviceInfo dev;
  if (!device_info(&dev)) return TOVA_ERR_CUDA;
  tova::PagedWriteParams p{};
  p.x[0] = k; p.x[1] = v; p.y[0] = K; p.y[1] = V;
  p.x_stride[0] = k_stride * (int64_t)E / 16; p.x_stride[1] = v_stride * (int64_t)E / 16;
  p.table = page_table; p.first = first_rows; p.offsets = offsets;
  p.max_rows = (long long)cfg->max_pages * cfg->page_rows;
  p.S = cfg->batch; p.N = n_tokens; p.Hkv = cfg->n_kv_heads; p.n_pages = cfg->n_pages; p.max_pages = cfg->max_pages;
  p.shift = paged_shift(*cfg);
  const unsigned vec = (unsigned)(cfg->head_dim * E / 16), per_row = vec * (unsigned)cfg->n_kv_heads;      // vec: 8, 16 or 32
  for (p.vec_shift = 3; (1u << p.vec_shift) < vec;) ++p.vec_shift;
  // Exact for i < 2 * PAGED_WRITE_TOKENS * per_row where i * per_row < 2^32.
  p.magic = 2ull * tova::PAGED_WRITE_TOKENS * per_row * per_row < (1ull << 32) ? (unsigned)(((1ull << 32) + per_row - 1) / per_row) : 0;
  p.tokens_per_block = (int)std::min<long long>(tova::PAGED_WRITE_TOKENS, std::max<long long>(1, n_tokens / (4LL * dev.sm_count)));
  const unsigned blocks = (unsigned)((n_tokens + p.tokens_per_block - 1) / p.tokens_per_block);
  tova::tova_paged_write_kernel<<<blocks, tova::PAGED_WRITE_THREADS, 0, static_cast<cudaStream_t>(cuda_stream)>>>(p);
  return launched(cudaGetLastError());
}

extern "C" size_t tova_paged_workspace_bytes(const tova_paged_config* cfg, int32_t n_live) {
  DeviceInfo dev;
  if (paged_check(cfg) != TOVA_OK || !paged_bound_ok(*cfg, n_live) || !device_info(&dev)) return (size_t)-1;
  return paged_plan(*cfg, n_live, dev.sm_count, true).bytes;
}

extern "C" int tova_paged_attention(const tova_paged_config* cfg, const void* K, const void* V, const int32_t* page_table,
                                    const int32_t* lens, int32_t n_live, const void* q, int64_t q_stride, void* out, void* workspace,
                                    size_t workspace_bytes, void* cuda_stream) {
  if (int rc = paged_check(cfg)) return rc;
  if (!paged_bound_ok(*cfg, n_live)) return TOVA_ERR_BAD_SHAPE;
  if (!K || !V || !page_table || !lens || !q || !out) return TOVA_ERR_NULL;
  if (!aligned16(K) || !aligned16(V) || !aligned16(q) || !aligned16(out) || !aligned16(workspace)) return TOVA_ERR_ALIGN;
  if (q_stride < 0) return TOVA_ERR_BAD_SHAPE;
  if (!stride_ok(q_stride, (int64_t)cfg->n_q_heads * cfg->head_dim, dtype_bytes(cfg->dtype))) return TOVA_ERR_ALIGN;
  DeviceInfo dev;
  if (!device_info(&dev)) return TOVA_ERR_CUDA;
  const PagedPlan t = paged_plan(*cfg, n_live, dev.sm_count);
  if (t.bytes > 0 && !workspace) return TOVA_ERR_NULL;
  if (workspace_bytes < t.bytes) return TOVA_ERR_WORKSPACE;
  tova::PagedParams p{};
  p.q = q; p.K = K; p.V = V; p.table = page_table; p.lens = lens; p.out = out;
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  p.part_acc = reinterpret_cast<float*>(ws);
  p.part_ml = reinterpret_cast<float2*>(ws + t.acc_bytes);
  p.cuts = reinterpret_cast<tova::PagedCut*>(ws + t.acc_bytes + t.ml_bytes);
  p.q_stride = q_stride;
  p.B = cfg->batch; p.H = cfg->n_q_heads; p.Hkv = cfg->n_kv_heads; p.G = p.H / p.Hkv;
  p.hgroups = t.hgroups; p.jobs = t.jobs;
  p.n_pages = cfg->n_pages; p.max_pages = cfg->max_pages; p.shift = paged_shift(*cfg); p.n_live = n_live; p.least = t.least;
  const float scale = cfg->sm_scale == 0.f ? 1.f / std::sqrt((float)cfg->head_dim) : cfg->sm_scale;
  p.scale2 = scale * 1.4426950408889634f;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const bool bf16 = cfg->dtype == TOVA_DTYPE_BF16;
  return launched(cfg->head_dim == 128 ? paged_run<128>(p, t, bf16, st) : paged_run<64>(p, t, bf16, st));
}

// ---------------------------------------------------------------------------
// Attention of packed prompts
// ---------------------------------------------------------------------------
namespace {

int packed_check(const tova_packed_config* c, int32_t n_tokens) {
  if (!c) return TOVA_ERR_NULL;
  if (!heads_ok(c->n_seqs, c->n_q_heads, c->n_kv_heads) || !(c->sm_scale >= 0.f) || !std::isfinite(c->sm_scale) || n_tokens < 0 || n_tokens > (1 << 24))
    return TOVA_ERR_BAD_SHAPE;
  if ((c->head_dim != 64 && c->head_dim != 128) || !known_dtype(c->dtype)) return TOVA_ERR_UNSUPPORTED;
  return TOVA_OK;
}

struct PackedPlan {
  bool pairs;                  // bf16: an item is two heads, not two tiles of tokens
  int rows, room, heads;       // tokens of a list's entry, the most entries there can be, items (fp32: blocks) of each
  bool list;                   // entries in order of their work
  size_t bytes;
};
PackedPlan packed_plan(const tova_packed_config& c, int32_t n_tokens, int sm_count) {
  PackedPlan t{};
  const bool bf16 = c.dtype == TOVA_DTYPE_BF16;
  t.pairs = bf16 && (c.n_q_heads / c.n_kv_heads) % 2 == 0;
  t.rows = !bf16 ? tova::PACKED_ALU_ROWS : t.pairs ? 128 : 256;
  t.room = n_tokens / t.rows + std::min(c.n_seqs, n_tokens);
  t.heads = t.pairs ? c.n_q_heads / 2 : c.n_q_heads;
  // (a block that finds its own tile walks through the sequences, 32 at a time)
  t.list = (long long)t.room * t.heads > sm_count || c.n_seqs > 256;
  t.bytes = t.list ? 16 + (size_t)t.room * sizeof(int4) : 0;
  return t;
}

template <int D>
cudaError_t packed_launch_alu(const tova::PackedParams& p, const PackedPlan& t, cudaStream_t st) {
  static std::atomic<bool> done[64];
  constexpr int smem = tova::packed_alu_smem<D>();
  const cudaError_t e = allow_smem(tova::tova_packed_alu_kernel<float, D>, done, smem);
  if (e != cudaSuccess) return e;
  return start(tova::tova_packed_alu_kernel<float, D>, dim3((unsigned)t.room, (unsigned)p.H), tova::PACKED_ALU_THREADS, smem, 1, t.list, st, p);
}

template <int D>
cudaError_t packed_launch_tc(const tova::PackedParams& p, const PackedPlan& t, int sm_count, cudaStream_t st) {
  static std::atomic<bool> done[64];
  using S = tova::PackedTcShape<D>;
  const cudaError_t e = allow_smem(tova::tova_packed_tc_kernel<D>, done, S::SMEM);
  if (e != cudaSuccess) return e;
  // q, k, v as [N, heads, D] in boxes of 128 tokens of one head x 64 components.
  CUtensorMap map[3];
  const void* base[3] = {p.q, p.k, p.v};
  const int64_t stride[3] = {p.q_stride, p.k_stride, p.v_stride};
  for (int i = 0; i < 3; ++i) {
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)(i == 0 ? p.H : p.Hkv), (cuuint64_t)p.N};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)stride[i] * 2};
    const cuuint32_t box[3] = {64, 1, 128};
    if (encode_map(&map[i], const_cast<void*>(base[i]), 3, dims, strides, box) != TOVA_OK) return cudaErrorInvalidValue;
  }
  const long long items = (long long)t.room * t.heads;
  const unsigned grid = (unsigned)(t.list ? std::min<long long>(items, sm_count) : items);
  return start(tova::tova_packed_tc_kernel<D>, dim3(grid), S::THREADS, S::SMEM, 1, t.list, st, p, map[0], map[1], map[2]);
}

}  // namespace

extern "C" size_t tova_packed_workspace_bytes(const tova_packed_config* cfg, int32_t n_tokens) {
  DeviceInfo dev;
  if (packed_check(cfg, n_tokens) != TOVA_OK || !device_info(&dev)) return (size_t)-1;
  return packed_plan(*cfg, n_tokens, dev.sm_count).bytes;
}

extern "C" int tova_packed_attention(const tova_packed_config* cfg, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                     const void* v, int64_t v_stride, int32_t n_tokens, const int32_t* offsets, void* out,
                                     void* workspace, size_t workspace_bytes, void* cuda_stream) {
  if (int rc = packed_check(cfg, n_tokens)) return rc;
  if (n_tokens == 0) return TOVA_OK;
  if (!q || !k || !v || !offsets || !out) return TOVA_ERR_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(workspace)) return TOVA_ERR_ALIGN;
  if (q_stride < 0 || k_stride < 0 || v_stride < 0) return TOVA_ERR_BAD_SHAPE;
  const size_t E = dtype_bytes(cfg->dtype);
  const int64_t qr = (int64_t)cfg->n_q_heads * cfg->head_dim, kr = (int64_t)cfg->n_kv_heads * cfg->head_dim;
  if (!stride_ok(q_stride, qr, E) || !stride_ok(k_stride, kr, E) || !stride_ok(v_stride, kr, E)) return TOVA_ERR_ALIGN;
  DeviceInfo dev;
  if (!device_info(&dev)) return TOVA_ERR_CUDA;
  const PackedPlan t = packed_plan(*cfg, n_tokens, dev.sm_count);
  if (t.bytes > 0 && !workspace) return TOVA_ERR_NULL;
  if (workspace_bytes < t.bytes) return TOVA_ERR_WORKSPACE;
  tova::PackedParams p{};
  p.q = q; p.k = k; p.v = v; p.out = out; p.offsets = offsets;
  p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride;
  p.S = cfg->n_seqs; p.N = n_tokens; p.H = cfg->n_q_heads; p.Hkv = cfg->n_kv_heads; p.G = p.H / p.Hkv;
  const float scale = cfg->sm_scale == 0.f ? 1.f / std::sqrt((float)cfg->head_dim) : cfg->sm_scale;
  p.scale2 = scale * 1.4426950408889634f;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  p.pairs = t.pairs;
  if (n_tokens == 1) p.q_stride = qr, p.k_stride = kr, p.v_stride = kr;      // (no second row: any stride will do)
  if (t.list) {
    int* n_list = static_cast<int*>(workspace);
    int4* list = reinterpret_cast<int4*>(static_cast<unsigned char*>(workspace) + 16);
    tova::tova_packed_plan_kernel<<<1, tova::PACKED_PLAN_THREADS, 0, st>>>(p, t.rows, list, n_list, t.room);
    if (int rc = launched(cudaGetLastError())) return rc;
    p.list = list;
    p.n_list = n_list;
  }
  if (cfg->dtype == TOVA_DTYPE_BF16)
    return launched(cfg->head_dim == 128 ? packed_launch_tc<128>(p, t, dev.sm_count, st) : packed_launch_tc<64>(p, t, dev.sm_count, st));
  return launched(cfg->head_dim == 128 ? packed_launch_alu<128>(p, t, st) : packed_launch_alu<64>(p, t, st));
}

// ---------------------------------------------------------------------------
// Log probabilities
// ---------------------------------------------------------------------------
extern "C" int tova_token_logprobs(const tova_logprobs_config* cfg, const void* logits, int32_t n_tokens, const int32_t* tokens,
                                   float* logprobs, float* entropy, int32_t* top_ids, float* top_logprobs, void* cuda_stream) {
  if (!cfg) return TOVA_ERR_NULL;
  if (cfg->vocab < 1 || cfg->vocab > (1 << 24) || cfg->n_top < 0 || cfg->n_top > tova::LOGPROBS_MAX_TOP || cfg->n_top > cfg->vocab ||
      (cfg->row_stride != 0 && cfg->row_stride < cfg->vocab) || n_tokens < 0 || n_tokens > (1 << 24))
    return TOVA_ERR_BAD_SHAPE;
  if (!known_dtype(cfg->dtype)) return TOVA_ERR_UNSUPPORTED;
  if (n_tokens == 0) return TOVA_OK;
  if (!logits || !tokens || !logprobs || (cfg->n_top > 0 && (!top_ids || !top_logprobs))) return TOVA_ERR_NULL;
  if (!aligned16(logits)) return TOVA_ERR_ALIGN;
  DeviceInfo dev;
  if (!device_info(&dev)) return TOVA_ERR_CUDA;
  tova::LogprobsParams p{};
  p.x = logits; p.tokens = tokens; p.lp = logprobs; p.entropy = entropy; p.ids = top_ids; p.top_lp = top_logprobs;
  p.row_stride = cfg->row_stride ? cfg->row_stride : cfg->vocab;
  p.T = n_tokens; p.V = cfg->vocab; p.top = cfg->n_top;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  // A cluster a row while rows are too few to give every SM one, and long enough to be shared out.
  const bool cluster = n_tokens <= dev.sm_count / 2 && cfg->vocab >= 4096;
  const int blocks = n_tokens * (cluster ? tova::LOGPROBS_CLUSTER : 1), size = cluster ? tova::LOGPROBS_CLUSTER : 1;
  constexpr int TH = tova::LOGPROBS_THREADS;
  if (cfg->dtype == TOVA_DTYPE_BF16)
    return launched(cluster ? start(tova::tova_logprobs_kernel<__nv_bfloat16, true>, dim3((unsigned)blocks), TH, 0, size, false, st, p)
                            : start(tova::tova_logprobs_kernel<__nv_bfloat16, false>, dim3((unsigned)blocks), TH, 0, size, false, st, p));
  return launched(cluster ? start(tova::tova_logprobs_kernel<float, true>, dim3((unsigned)blocks), TH, 0, size, false, st, p)
                          : start(tova::tova_logprobs_kernel<float, false>, dim3((unsigned)blocks), TH, 0, size, false, st, p));
}
