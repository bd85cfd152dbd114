// Host side of the operators around the decode step declared in include/tova.h: rotary positions, the 8-bit state,
// attention of drafted tokens, their verification.  Argument checks and launches; the work runs in the kernels of
// tova_rope.cuh, tova_quant.cuh, tova_tree.cuh and tova_verify.cuh.
#include "../../include/tova.h"

#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <new>
#include <type_traits>

#include "tova_quant.cuh"
#include "tova_rope.cuh"
#include "tova_tree.cuh"
#include "tova_tree_mma.cuh"
#include "tova_tree_tc.cuh"
#include "tova_verify.cuh"

// tova_api.cu
int encode_state_map(CUtensorMap* map, void* base, const tova_config& cfg, int box_rows, long long rows_per_head);
int encode_map(CUtensorMap* map, void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box);

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool known_dtype(int32_t t) { return t == TOVA_DTYPE_FP32 || t == TOVA_DTYPE_BF16; }
inline size_t dtype_bytes(int32_t t) { return t == TOVA_DTYPE_BF16 ? 2 : 4; }

// Batch and heads as everywhere in the library (tova_config).
inline bool heads_ok(int32_t batch, int32_t hq, int32_t hkv) {
  return batch >= 1 && batch <= 65535 && hkv >= 1 && hq >= hkv && hq <= 4096 && hq % hkv == 0;
}

// A row stride in elements: 0 = contiguous; else at least a row, and whole 16-byte vectors.
inline bool stride_ok(int64_t& s, int64_t row, size_t elem) {
  if (s == 0) s = row;
  return s >= row && (s * (int64_t)elem) % 16 == 0;
}

struct DeviceInfo {
  int sm_count;
};

// SM count of the current device, looked up once per device.
bool device_info(DeviceInfo* out) {
  static std::atomic<int> sms[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
  int n = sms[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) return false;
    sms[dev].store(n, std::memory_order_relaxed);
  }
  out->sm_count = n;
  return true;
}

inline int launched(cudaError_t e) { return e == cudaSuccess ? TOVA_OK : TOVA_ERR_CUDA; }

}  // namespace

// ---------------------------------------------------------------------------
// Rotary positions
// ---------------------------------------------------------------------------
struct tova_rope {
  tova_rope_config cfg;
  double turns[tova::ROPE_MAX_PAIRS];   // w_i / 2 pi
  float factor;                         // m
};

extern "C" int tova_rope_init(tova_rope** out, const tova_rope_config* cfg) {
  if (!out) return TOVA_ERR_NULL;
  *out = nullptr;
  if (!cfg) return TOVA_ERR_NULL;
  tova_rope_config c = *cfg;
  if (c.rotary_dim == 0) c.rotary_dim = c.head_dim;
  if (c.base == 0.0) c.base = 10000.0;
  if (c.factor == 0.0 || c.scaling == TOVA_ROPE_PLAIN) c.factor = 1.0;
  if ((c.head_dim != 64 && c.head_dim != 128) || !known_dtype(c.dtype) || (c.layout != TOVA_ROPE_HALF && c.layout != TOVA_ROPE_INTERLEAVED) ||
      c.scaling < TOVA_ROPE_PLAIN || c.scaling > TOVA_ROPE_BANDS)
    return TOVA_ERR_UNSUPPORTED;
  if (!heads_ok(c.batch, c.n_q_heads, c.n_kv_heads) || c.rotary_dim < 2 || c.rotary_dim > c.head_dim || c.rotary_dim % 2 != 0 ||
      !(c.base > 1.0) || !std::isfinite(c.base) || !(c.factor >= 1.0) || !std::isfinite(c.factor) || !(c.amplitude >= 0.0) ||
      !std::isfinite(c.amplitude) || !(c.blend_low >= 0.0) || !(c.blend_high >= 0.0) || !std::isfinite(c.blend_low) || !std::isfinite(c.blend_high))
    return TOVA_ERR_BAD_SHAPE;
  const bool blends = c.scaling == TOVA_ROPE_YARN || c.scaling == TOVA_ROPE_BANDS;
  const double low = c.blend_low > 0.0 ? c.blend_low : 1.0;
  const double high = c.blend_high > 0.0 ? c.blend_high : (c.scaling == TOVA_ROPE_YARN ? 32.0 : 4.0);
  if (blends && (c.original_context < 1 || !(high > low))) return TOVA_ERR_BAD_SHAPE;
  if (c.scaling == TOVA_ROPE_NTK && c.rotary_dim == 2) return TOVA_ERR_BAD_SHAPE;

  const double two_pi = 6.283185307179586476925286766559;
  const int half = c.rotary_dim / 2;
  const double rot = c.rotary_dim;
  double base = c.base, m = 1.0;
  if (c.scaling == TOVA_ROPE_NTK) base *= std::pow(c.factor, rot / (rot - 2.0));
  double ramp_lo = 0.0, ramp_hi = 0.0;
  if (c.scaling == TOVA_ROPE_YARN) {
    auto pair_of = [&](double turns) { return rot * std::log(c.original_context / (turns * two_pi)) / (2.0 * std::log(base)); };
    ramp_lo = std::floor(pair_of(high));
    ramp_hi = std::ceil(pair_of(low));
    // The bounds are held to the pairs' indices, unless the whole ramp lies before the first pair (then all pairs turn less
    // than `low` times) or behind: held there too, it would run backwards.
    if (ramp_hi >= 0.0 && ramp_lo <= rot - 1.0) {
      ramp_lo = std::max(ramp_lo, 0.0);
      ramp_hi = std::min(ramp_hi, rot - 1.0);
    }
    if (ramp_hi == ramp_lo) ramp_hi += 0.001;
    m = c.factor > 1.0 ? 0.1 * std::log(c.factor) + 1.0 : 1.0;
  }
  tova_rope* r = new (std::nothrow) tova_rope();
  if (!r) return TOVA_ERR_CUDA;
  for (int i = 0; i < half; ++i) {
    double w = std::pow(base, -2.0 * i / rot);
    if (c.scaling == TOVA_ROPE_LINEAR) {
      w /= c.factor;
    } else if (c.scaling == TOVA_ROPE_YARN) {
      const double ramp = std::min(1.0, std::max(0.0, (i - ramp_lo) / (ramp_hi - ramp_lo)));
      w = w / c.factor * ramp + w * (1.0 - ramp);
    } else if (c.scaling == TOVA_ROPE_BANDS) {
      const double per_context = c.original_context * w / two_pi;   // original_context / wavelength
      if (per_context < low) w /= c.factor;
      else if (per_context <= high) {
        const double s = (per_context - low) / (high - low);
        w = (1.0 - s) * w / c.factor + s * w;
      }
    }
    r->turns[i] = w / two_pi;
  }
  r->factor = (float)(c.amplitude > 0.0 ? c.amplitude : m);
  r->cfg = c;
  *out = r;
  return TOVA_OK;
}

extern "C" int tova_rope_apply(const tova_rope* r, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                               int32_t n_tokens, const int32_t* positions, int32_t first_pos, int32_t inverse, void* q_out,
                               int64_t q_out_stride, void* k_out, int64_t k_out_stride, void* cuda_stream) {
  if (!r) return TOVA_ERR_NULL;
  const tova_rope_config& c = r->cfg;
  if (n_tokens < 0) return TOVA_ERR_BAD_SHAPE;
  if (n_tokens == 0) return TOVA_OK;
  if (!q || !q_out || (k == nullptr) != (k_out == nullptr)) return TOVA_ERR_NULL;
  const size_t E = dtype_bytes(c.dtype);
  const int64_t qr = (int64_t)c.n_q_heads * c.head_dim, kr = (int64_t)c.n_kv_heads * c.head_dim;
  if (!aligned16(q) || !aligned16(q_out) || !aligned16(k) || !aligned16(k_out)) return TOVA_ERR_ALIGN;
  if (q_stride < 0 || k_stride < 0 || q_out_stride < 0 || k_out_stride < 0) return TOVA_ERR_BAD_SHAPE;
  if (!stride_ok(q_stride, qr, E) || !stride_ok(q_out_stride, qr, E) || !stride_ok(k_stride, kr, E) || !stride_ok(k_out_stride, kr, E))
    return TOVA_ERR_ALIGN;
  if (!positions && (int64_t)first_pos + n_tokens - 1 > INT32_MAX) return TOVA_ERR_BAD_SHAPE;
  DeviceInfo dev;
  if (!device_info(&dev)) return TOVA_ERR_CUDA;

  tova::RopeParams p{};
  p.x[0] = q; p.x[1] = k; p.y[0] = q_out; p.y[1] = k_out;
  p.x_stride[0] = q_stride; p.x_stride[1] = k_stride;
  p.y_stride[0] = q_out_stride; p.y_stride[1] = k_out_stride;
  p.heads[0] = c.n_q_heads;
  p.heads[1] = k ? c.n_kv_heads : 0;
  p.positions = positions;
  p.rows = (long long)n_tokens * c.batch;
  p.first_pos = first_pos;
  p.B = c.batch; p.D = c.head_dim; p.rot = c.rotary_dim;
  p.factor = r->factor;
  p.sign = inverse ? -1.f : 1.f;
  std::copy(r->turns, r->turns + tova::ROPE_MAX_PAIRS, p.turns);
  // One token per block while that leaves SMs idle; several share the set-up of a block beyond that.
  p.tokens_per_block = (int)std::min<long long>(tova::ROPE_MAX_TOKENS, std::max<long long>(1, p.rows / (8LL * dev.sm_count)));
  const long long blocks = (p.rows + p.tokens_per_block - 1) / p.tokens_per_block;
  if (blocks > INT32_MAX) return TOVA_ERR_BAD_SHAPE;
  const int N = c.dtype == TOVA_DTYPE_BF16 ? 8 : 4;
  const bool half = c.layout == TOVA_ROPE_HALF;
  const bool vec = half ? (c.rotary_dim / 2) % N == 0 : c.rotary_dim % N == 0;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const unsigned g = (unsigned)blocks;
  constexpr int TH = tova::ROPE_THREADS;
  if (c.dtype == TOVA_DTYPE_BF16) {
    if (half) {
      if (vec) tova::tova_rope_kernel<__nv_bfloat16, true, true><<<g, TH, 0, st>>>(p);
      else tova::tova_rope_kernel<__nv_bfloat16, true, false><<<g, TH, 0, st>>>(p);
    } else {
      if (vec) tova::tova_rope_kernel<__nv_bfloat16, false, true><<<g, TH, 0, st>>>(p);
      else tova::tova_rope_kernel<__nv_bfloat16, false, false><<<g, TH, 0, st>>>(p);
    }
  } else {
    if (half) {
      if (vec) tova::tova_rope_kernel<float, true, true><<<g, TH, 0, st>>>(p);
      else tova::tova_rope_kernel<float, true, false><<<g, TH, 0, st>>>(p);
    } else {
      if (vec) tova::tova_rope_kernel<float, false, true><<<g, TH, 0, st>>>(p);
      else tova::tova_rope_kernel<float, false, false><<<g, TH, 0, st>>>(p);
    }
  }
  return launched(cudaGetLastError());
}

extern "C" int tova_rope_destroy(tova_rope* r) {
  if (!r) return TOVA_ERR_NULL;
  delete r;
  return TOVA_OK;
}

// ---------------------------------------------------------------------------
// The 8-bit state
// ---------------------------------------------------------------------------
namespace {

int quant_check(const tova_quant_config* c, int32_t n_tokens, const int32_t* slots, int32_t first_slot) {
  if (!c) return TOVA_ERR_NULL;
  if (c->batch < 1 || c->batch > 65535 || c->n_kv_heads < 1 || c->n_kv_heads > 65535 || c->capacity < 1 || c->capacity > (1 << 24) || n_tokens < 0)
    return TOVA_ERR_BAD_SHAPE;
  if ((c->head_dim != 64 && c->head_dim != 128) || !known_dtype(c->dtype) || (c->format != TOVA_FORMAT_INT8 && c->format != TOVA_FORMAT_E4M3))
    return TOVA_ERR_UNSUPPORTED;
  if (!slots && n_tokens > 0 && (first_slot < 0 || (int64_t)first_slot + n_tokens > c->capacity)) return TOVA_ERR_BAD_SHAPE;
  return TOVA_OK;
}

// Tokens per block: as many as still give every SM a few blocks.
int quant_tokens_per_block(const tova_quant_config& c, int32_t n_tokens, int sm_count) {
  int n = tova::QUANT_MAX_TOKENS;
  while (n > 1 && (long long)((n_tokens + n - 1) / n) * c.batch < 4LL * sm_count) n /= 2;
  return n;
}

template <typename T, int D, int FMT>
void quant_launch(const tova::QuantParams& p, bool write, dim3 grid, cudaStream_t st) {
  if (write) tova::tova_quant_write_kernel<T, D, FMT><<<grid, tova::QUANT_THREADS, 0, st>>>(p);
  else tova::tova_quant_read_kernel<T, D, FMT><<<grid, tova::QUANT_THREADS, 0, st>>>(p);
}
template <typename T, int D>
void quant_launch_f(const tova::QuantParams& p, int format, bool write, dim3 grid, cudaStream_t st) {
  if (format == TOVA_FORMAT_INT8) quant_launch<T, D, tova::FORMAT_INT8>(p, write, grid, st);
  else quant_launch<T, D, tova::FORMAT_E4M3>(p, write, grid, st);
}
int quant_run(const tova_quant_config& c, tova::QuantParams& p, bool write, void* cuda_stream) {
  DeviceInfo dev;
  if (!device_info(&dev)) return TOVA_ERR_CUDA;
  p.B = c.batch; p.Hkv = c.n_kv_heads; p.cap = c.capacity;
  p.tokens_per_block = quant_tokens_per_block(c, p.T, dev.sm_count);
  const dim3 grid((unsigned)((p.T + p.tokens_per_block - 1) / p.tokens_per_block), (unsigned)c.batch);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (c.dtype == TOVA_DTYPE_BF16) {
    if (c.head_dim == 128) quant_launch_f<__nv_bfloat16, 128>(p, c.format, write, grid, st);
    else quant_launch_f<__nv_bfloat16, 64>(p, c.format, write, grid, st);
  } else {
    if (c.head_dim == 128) quant_launch_f<float, 128>(p, c.format, write, grid, st);
    else quant_launch_f<float, 64>(p, c.format, write, grid, st);
  }
  return launched(cudaGetLastError());
}

}  // namespace

extern "C" int tova_quant_write(const tova_quant_config* cfg, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                                int32_t n_tokens, const int32_t* slots, int32_t first_slot, void* k_codes, float* k_scale,
                                void* v_codes, float* v_scale, void* cuda_stream) {
  if (int rc = quant_check(cfg, n_tokens, slots, first_slot)) return rc;
  if (n_tokens == 0) return TOVA_OK;
  if (!k || !v || !k_codes || !k_scale || !v_codes || !v_scale) return TOVA_ERR_NULL;
  if (!aligned16(k) || !aligned16(v) || !aligned16(k_codes) || !aligned16(v_codes) || !aligned16(k_scale) || !aligned16(v_scale))
    return TOVA_ERR_ALIGN;
  if (k_stride < 0 || v_stride < 0) return TOVA_ERR_BAD_SHAPE;
  const int64_t row = (int64_t)cfg->n_kv_heads * cfg->head_dim;
  if (!stride_ok(k_stride, row, dtype_bytes(cfg->dtype)) || !stride_ok(v_stride, row, dtype_bytes(cfg->dtype))) return TOVA_ERR_ALIGN;
  tova::QuantParams p{};
  p.x[0] = k; p.x[1] = v;
  p.x_stride[0] = k_stride; p.x_stride[1] = v_stride;
  p.codes[0] = k_codes; p.codes[1] = v_codes;
  p.scale[0] = k_scale; p.scale[1] = v_scale;
  p.slots = slots; p.first_slot = first_slot; p.T = n_tokens;
  return quant_run(*cfg, p, true, cuda_stream);
}

extern "C" int tova_quant_read(const tova_quant_config* cfg, const void* k_codes, const float* k_scale, const void* v_codes,
                               const float* v_scale, int32_t n_tokens, const int32_t* slots, int32_t first_slot, void* k,
                               void* v, void* cuda_stream) {
  if (int rc = quant_check(cfg, n_tokens, slots, first_slot)) return rc;
  if (n_tokens == 0 || (!k && !v)) return TOVA_OK;
  if ((k && (!k_codes || !k_scale)) || (v && (!v_codes || !v_scale))) return TOVA_ERR_NULL;
  if (!aligned16(k) || !aligned16(v) || !aligned16(k_codes) || !aligned16(v_codes) || !aligned16(k_scale) || !aligned16(v_scale))
    return TOVA_ERR_ALIGN;
  tova::QuantParams p{};
  p.y[0] = k; p.y[1] = v;
  p.codes[0] = const_cast<void*>(k_codes); p.codes[1] = const_cast<void*>(v_codes);
  p.scale[0] = const_cast<float*>(k_scale); p.scale[1] = const_cast<float*>(v_scale);
  p.slots = slots; p.first_slot = first_slot; p.T = n_tokens;
  return quant_run(*cfg, p, false, cuda_stream);
}

// ---------------------------------------------------------------------------
// Attention of drafted tokens
// ---------------------------------------------------------------------------
namespace {

int tree_check(const tova_tree_config* c, int32_t n_live, int32_t n_nodes) {
  if (!c) return TOVA_ERR_NULL;
  if (!heads_ok(c->batch, c->n_q_heads, c->n_kv_heads) || c->capacity < 1 || c->capacity > (1 << 24) || !(c->sm_scale >= 0.f) ||
      !std::isfinite(c->sm_scale) || n_live < 0 || n_live > c->capacity || n_nodes < 0 || n_nodes > tova::TREE_MAX_NODES ||
      (long long)c->batch * c->n_kv_heads > 65535)
    return TOVA_ERR_BAD_SHAPE;
  if ((c->head_dim != 64 && c->head_dim != 128) || !known_dtype(c->dtype) || c->format < TOVA_FORMAT_PLAIN || c->format > TOVA_FORMAT_E4M3)
    return TOVA_ERR_UNSUPPORTED;
  return TOVA_OK;
}

// Which kernel serves a call and how its columns are cut.
enum : int { TREE_ALU, TREE_MMA_16, TREE_MMA_32, TREE_MMA_64, TREE_TC_1, TREE_TC_2 };
struct TreePlan {
  int kernel, row_blocks, splits, split_cols;
  int blocks, group, row_rounds, least;      // tcgen05 kernel
  bool cluster;                  // the runs' blocks join by themselves
  size_t ml_bytes, acc_bytes, bytes;   // workspace: maxima and sums, weighted sums (and the tcgen05 kernel's list of cuts)
};

// up_to: the workspace is to do for every length up to n_live (fewer tiles can make more runs: 150 tiles for at most 148 runs
// are 75 of two, 148 are 148 of one).
TreePlan tree_plan(const tova_tree_config& c, int32_t n_live, int32_t n_nodes, int sm_count, bool up_to = false) {
  TreePlan t{};
  const int M = n_nodes * (c.n_q_heads / c.n_kv_heads);
  size_t part_rows;
  if (c.dtype == TOVA_DTYPE_BF16 && M > 64) {
    // More than 64 rows: the contractions, not the state's bytes, set the pace of a warp-level kernel.
    // Two row tiles a block from 129 rows on; 8-bit states one (see the kernel).
    const bool one = M <= 128 || c.format != TOVA_FORMAT_PLAIN;
    t.kernel = one ? TREE_TC_1 : TREE_TC_2;
    t.splits = 1;
    const int rows = (one ? 1 : 2) * tova::TREE_TC_ROWS, row_blocks = (M + rows - 1) / rows;
    t.row_rounds = (row_blocks + sm_count - 1) / sm_count;
    t.group = (row_blocks + t.row_rounds - 1) / t.row_rounds;
    t.blocks = sm_count / t.group * t.group;
    t.least = 4;                 // tiles of 128 columns: less than that does not pay for a block's set-up
    part_rows = (size_t)2 * t.blocks * rows;
  } else {
    int rows = M <= 4 ? 4 : M <= 16 ? 16 : 64, cols = tova::TREE_ALU_COLS;       // fp32: the plain-ALU kernel
    if (c.dtype == TOVA_DTYPE_BF16) {
      t.kernel = M <= 16 ? TREE_MMA_16 : M <= 32 ? TREE_MMA_32 : TREE_MMA_64;
      rows = 64;
      cols = 64;                 // a tile of four warps
    }
    t.row_blocks = (M + rows - 1) / rows;
    const long long whole = (long long)t.row_blocks * c.batch * c.n_kv_heads;
    const int all_tiles = std::max(1, (n_live + cols - 1) / cols);
    int tiles = all_tiles;
    // Runs of columns for two rounds of resident blocks (two per SM), but none shorter than two tiles unless the GPU
    // would stay half empty.
    const int resident = 2 * sm_count, shortest = whole * (tiles / 2) < resident ? 1 : 2;
    long long want = (2LL * resident + whole - 1) / whole;
    const long long most = want;
    want = std::max(1LL, std::min<long long>(want, tiles / shortest));
    // Up to eight runs join in a cluster.  A call with more runs gets eight, too, where they are then at most four tiles
    // long: that is less time than the second kernel takes.
    if (t.kernel != TREE_ALU && want > 1 && (want <= tova::TREE_CLUSTER_MAX || tiles <= 4 * tova::TREE_CLUSTER_MAX)) {
      t.cluster = true;
      cols *= 2;                 // a tile of eight warps
      tiles = (tiles + 1) / 2;
      want = std::min<long long>(std::min<long long>(want, tova::TREE_CLUSTER_MAX), tiles);
    }
    const int per = (int)((tiles + want - 1) / want);
    t.split_cols = per * cols;
    t.splits = (tiles + per - 1) / per;
    t.cluster = t.cluster && t.splits > 1;
    if (t.splits > 1 && !t.cluster) t.splits += 1;      // a run of its own for the drafts: it does not wait for a run of rows
    // A shorter state makes at most as many runs as it has tiles, and joins them in a cluster where it has few.
    const bool merges = most > 1 && all_tiles > 1 && (t.kernel == TREE_ALU || (most > tova::TREE_CLUSTER_MAX && all_tiles > 4 * tova::TREE_CLUSTER_MAX));
    const long long runs = up_to ? (merges ? std::min<long long>(most, all_tiles) + 1 : 0) : t.splits > 1 && !t.cluster ? t.splits : 0;
    part_rows = (size_t)runs * c.batch * c.n_kv_heads * M;
  }
  t.ml_bytes = (part_rows * sizeof(float2) + 255) / 256 * 256;
  t.acc_bytes = part_rows * c.head_dim * sizeof(float);
  t.bytes = t.ml_bytes + t.acc_bytes + t.blocks * sizeof(tova::TreeTcCut);
  return t;
}

inline dim3 tree_grid(const tova::TreeParams& p, const TreePlan& t) {
  return dim3((unsigned)t.row_blocks, (unsigned)t.splits, (unsigned)(p.B * p.Hkv));
}

template <typename... Args>
cudaError_t tree_start(void (*kern)(Args...), std::atomic<bool>* configured, size_t smem, int threads, dim3 grid, int cluster_y,
                       cudaStream_t st, const Args&... args) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (!configured[dev & 63]) {
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, 100);
    if (e != cudaSuccess) return e;
    configured[dev & 63] = true;
  }
  cudaLaunchConfig_t lc{};
  lc.gridDim = grid;
  lc.blockDim = dim3((unsigned)threads);
  lc.dynamicSmemBytes = smem;
  lc.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = 1;
  at[0].val.clusterDim.y = (unsigned)cluster_y;
  at[0].val.clusterDim.z = 1;
  lc.attrs = at;
  lc.numAttrs = cluster_y > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&lc, kern, args...);
}

template <typename T, int D>
cudaError_t tree_merge(const tova::TreeParams& p, cudaStream_t st) {
  const long long rows = (long long)p.B * p.Hkv * p.M;
  cudaLaunchConfig_t lc{};
  constexpr int ROWS = tova::TREE_MERGE_THREADS / 32;
  lc.gridDim = dim3((unsigned)((rows + ROWS - 1) / ROWS));
  lc.blockDim = dim3(tova::TREE_MERGE_THREADS);
  lc.stream = st;
  cudaLaunchAttribute at[1];      // its blocks may come up while the first kernel's last ones still run
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at;
  lc.numAttrs = 1;
  return cudaLaunchKernelEx(&lc, tova::tova_tree_merge_kernel<T, D>, p);
}

template <int D, int FMT, int MT, int WR, bool CLUSTER>
cudaError_t tree_start_mma_c(const tova::TreeParams& p, const TreePlan& t, cudaStream_t st) {
  static std::atomic<bool> configured[64];
  using S = tova::TreeMmaShape<D, FMT, MT, WR, CLUSTER ? 8 : 4>;
  return tree_start(tova::tova_tree_mma_kernel<D, FMT, MT, WR, CLUSTER>, configured, S::SMEM, S::THREADS, tree_grid(p, t),
                    CLUSTER ? t.splits : 1, st, p);
}
template <int D, int FMT, int MT, int WR>
cudaError_t tree_start_mma(const tova::TreeParams& p, const TreePlan& t, cudaStream_t st) {
  return t.cluster && t.splits > 1 ? tree_start_mma_c<D, FMT, MT, WR, true>(p, t, st) : tree_start_mma_c<D, FMT, MT, WR, false>(p, t, st);
}

template <int D, int FMT, int NT>
cudaError_t tree_run_tc(const tova::TreeParams& p, const TreePlan& t, cudaStream_t st) {
  static std::atomic<bool> configured[64];
  using S = tova::TreeTcShape<D, FMT, NT>;
  // Tiled views of a bf16 state in boxes of 128 rows; where they cannot be had (fewer rows, 2^31 or more) the kernel
  // copies every tile as it copies a sequence's last.
  CUtensorMap map_k{}, map_v{}, map_q{};
  tova::TreeParams q = p;
  const long long rows = (long long)p.B * p.Hkv * p.cap;
  if (FMT == tova::FORMAT_PLAIN && rows >= tova::TREE_TC_COLS && rows < (1LL << 31)) {
    tova_config c{};
    c.batch = p.B; c.n_kv_heads = p.Hkv; c.capacity = p.cap; c.head_dim = D;
    q.tiled = encode_state_map(&map_k, const_cast<void*>(p.K), c, tova::TREE_TC_COLS, 0) == TOVA_OK &&
              encode_state_map(&map_v, const_cast<void*>(p.V), c, tova::TREE_TC_COLS, 0) == TOVA_OK;
  }
  // q as [N, B * H, D] in boxes of 128 / G nodes x one KV head's G query heads, where G divides 128.
  if (tova::TREE_TC_ROWS % p.G == 0) {
    const cuuint64_t heads = (cuuint64_t)p.B * p.H;
    const cuuint64_t dims[3] = {(cuuint64_t)D, heads, (cuuint64_t)p.N};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, heads * D * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)p.G, (cuuint32_t)(tova::TREE_TC_ROWS / p.G)};
    q.q_tiled = encode_map(&map_q, const_cast<void*>(p.q), 3, dims, strides, box) == TOVA_OK;
  }
  cudaError_t e = tree_start(tova::tova_tree_tc_kernel<D, FMT, NT>, configured, S::SMEM, S::THREADS, dim3((unsigned)t.blocks), 1, st, q, map_k, map_v, map_q);
  if (e != cudaSuccess) return e;
  constexpr int JOIN_ROWS = tova::TREE_TC_JOIN_THREADS / 32;
  cudaLaunchConfig_t lc{};
  lc.gridDim = dim3((unsigned)t.blocks, (unsigned)((std::min(p.M, NT * tova::TREE_TC_ROWS) + JOIN_ROWS - 1) / JOIN_ROWS));
  lc.blockDim = dim3(tova::TREE_TC_JOIN_THREADS);
  lc.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at;
  lc.numAttrs = 1;
  return cudaLaunchKernelEx(&lc, tova::tova_tree_tc_join_kernel<D, NT>, p);
}

template <int D, int FMT, int R>
cudaError_t tree_start_alu(const tova::TreeParams& p, const TreePlan& t, cudaStream_t st) {
  static std::atomic<bool> configured[64];
  return tree_start(tova::tova_tree_alu_kernel<D, FMT, R>, configured, tova::tree_alu_smem_bytes<D, R>(), tova::TREE_ALU_THREADS,
                    tree_grid(p, t), 1, st, p);
}

template <typename T, int D, int FMT>
cudaError_t tree_launch(const tova::TreeParams& p, const TreePlan& t, cudaStream_t st) {
  cudaError_t e;
  if constexpr (std::is_same<T, float>::value) {
    e = p.M <= 4    ? tree_start_alu<D, FMT, 4>(p, t, st)
        : p.M <= 16 ? tree_start_alu<D, FMT, 16>(p, t, st)
                    : tree_start_alu<D, FMT, 64>(p, t, st);
  } else {
    switch (t.kernel) {
      case TREE_MMA_16: e = tree_start_mma<D, FMT, 1, 1>(p, t, st); break;
      case TREE_MMA_32: e = tree_start_mma<D, FMT, 1, 2>(p, t, st); break;
      case TREE_MMA_64: e = tree_start_mma<D, FMT, 2, 2>(p, t, st); break;
      case TREE_TC_1: return tree_run_tc<D, FMT, 1>(p, t, st);
      default:
        if constexpr (FMT == tova::FORMAT_PLAIN) return tree_run_tc<D, FMT, 2>(p, t, st);
        return cudaErrorInvalidValue;
    }
  }
  if (e != cudaSuccess || t.splits == 1 || t.cluster) return e;
  return tree_merge<T, D>(p, st);
}
template <typename T, int D>
cudaError_t tree_launch_f(int format, const tova::TreeParams& p, const TreePlan& t, cudaStream_t st) {
  switch (format) {
    case TOVA_FORMAT_PLAIN: return tree_launch<T, D, tova::FORMAT_PLAIN>(p, t, st);
    case TOVA_FORMAT_INT8: return tree_launch<T, D, tova::FORMAT_INT8>(p, t, st);
    default: return tree_launch<T, D, tova::FORMAT_E4M3>(p, t, st);
  }
}

}  // namespace

extern "C" size_t tova_tree_workspace_bytes(const tova_tree_config* cfg, int32_t n_live, int32_t n_nodes) {
  DeviceInfo dev;
  if (tree_check(cfg, n_live, n_nodes) != TOVA_OK || !device_info(&dev)) return (size_t)-1;
  return n_nodes ? tree_plan(*cfg, n_live, n_nodes, dev.sm_count, true).bytes : 0;
}

extern "C" int tova_tree_attention(const tova_tree_config* cfg, const void* K, const void* V, const float* k_scale,
                                   const float* v_scale, const int32_t* lens, int32_t n_live, const void* q, const void* k,
                                   const void* v, int32_t n_nodes, const int32_t* parents, void* out, void* workspace,
                                   size_t workspace_bytes, void* cuda_stream) {
  if (int rc = tree_check(cfg, n_live, n_nodes)) return rc;
  if (n_nodes == 0) return TOVA_OK;
  if (!K || !V || !q || !k || !v || !out) return TOVA_ERR_NULL;
  if (cfg->format != TOVA_FORMAT_PLAIN && (!k_scale || !v_scale)) return TOVA_ERR_NULL;
  if (!aligned16(K) || !aligned16(V) || !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(workspace) ||
      !aligned16(k_scale) || !aligned16(v_scale))
    return TOVA_ERR_ALIGN;
  DeviceInfo dev;
  if (!device_info(&dev)) return TOVA_ERR_CUDA;
  const TreePlan t = tree_plan(*cfg, n_live, n_nodes, dev.sm_count);
  if (t.bytes > 0 && !workspace) return TOVA_ERR_NULL;
  if (workspace_bytes < t.bytes) return TOVA_ERR_WORKSPACE;

  tova::TreeParams p{};
  p.q = q; p.k_new = k; p.v_new = v; p.K = K; p.V = V;
  p.k_scale = k_scale; p.v_scale = v_scale;
  p.lens = lens; p.parents = parents; p.out = out;
  p.part_ml = static_cast<float2*>(workspace);
  p.part_acc = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + t.ml_bytes);
  p.cuts = static_cast<unsigned char*>(workspace) + t.ml_bytes + t.acc_bytes;
  p.N = n_nodes; p.B = cfg->batch; p.H = cfg->n_q_heads; p.Hkv = cfg->n_kv_heads;
  p.G = p.H / p.Hkv; p.M = p.N * p.G; p.cap = cfg->capacity; p.n_live = n_live;
  p.splits = t.splits; p.split_cols = t.split_cols;
  p.group = t.group; p.row_rounds = t.row_rounds; p.least = t.least;
  const float scale = cfg->sm_scale == 0.f ? 1.f / std::sqrt((float)cfg->head_dim) : cfg->sm_scale;
  p.scale2 = scale * 1.4426950408889634f;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (cfg->dtype == TOVA_DTYPE_BF16)
    return launched(cfg->head_dim == 128 ? tree_launch_f<__nv_bfloat16, 128>(cfg->format, p, t, st)
                                         : tree_launch_f<__nv_bfloat16, 64>(cfg->format, p, t, st));
  return launched(cfg->head_dim == 128 ? tree_launch_f<float, 128>(cfg->format, p, t, st)
                                       : tree_launch_f<float, 64>(cfg->format, p, t, st));
}

// ---------------------------------------------------------------------------
// Verification of drafted tokens
// ---------------------------------------------------------------------------
extern "C" int tova_verify_draft(const tova_verify_config* cfg, const void* target, const void* draft, const int32_t* tokens,
                                 const int32_t* parents, const float* u, const float* u_sample, int32_t* n_accepted,
                                 int32_t* path, int32_t* tokens_out, void* cuda_stream) {
  if (!cfg) return TOVA_ERR_NULL;
  if (cfg->batch < 1 || cfg->batch > 65535 || cfg->n_nodes < 0 || cfg->n_nodes > tova::VERIFY_MAX_NODES || cfg->vocab < 1 ||
      cfg->vocab > (1 << 24) || (cfg->row_stride != 0 && cfg->row_stride < cfg->vocab))
    return TOVA_ERR_BAD_SHAPE;
  if (!known_dtype(cfg->dtype)) return TOVA_ERR_UNSUPPORTED;
  if (!target || !u_sample || !n_accepted || !tokens_out || (cfg->n_nodes > 0 && (!tokens || !u))) return TOVA_ERR_NULL;
  if (!aligned16(target) || !aligned16(draft)) return TOVA_ERR_ALIGN;
  tova::VerifyParams p{};
  p.target = target; p.draft = draft; p.tokens = tokens; p.parents = parents;
  p.u = u; p.u_sample = u_sample;
  p.n_accepted = n_accepted; p.path = path; p.tokens_out = tokens_out;
  p.row_stride = cfg->row_stride ? cfg->row_stride : cfg->vocab;
  p.B = cfg->batch; p.N = cfg->n_nodes; p.V = cfg->vocab;
  p.vec = (p.row_stride * dtype_bytes(cfg->dtype)) % 16 == 0;

  cudaLaunchConfig_t lc{};
  lc.gridDim = dim3(tova::VERIFY_CLUSTER, (unsigned)cfg->batch);
  lc.blockDim = dim3(tova::VERIFY_THREADS);
  lc.dynamicSmemBytes = tova::verify_smem_bytes(cfg->n_nodes);
  lc.stream = static_cast<cudaStream_t>(cuda_stream);
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = tova::VERIFY_CLUSTER;
  at[0].val.clusterDim.y = 1;
  at[0].val.clusterDim.z = 1;
  lc.attrs = at;
  lc.numAttrs = 1;
  return launched(cfg->dtype == TOVA_DTYPE_BF16 ? cudaLaunchKernelEx(&lc, tova::tova_verify_kernel<__nv_bfloat16>, p)
                                                : cudaLaunchKernelEx(&lc, tova::tova_verify_kernel<float>, p));
}
