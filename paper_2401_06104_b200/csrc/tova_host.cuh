// Host-side helpers shared by the operators' entry points: argument checks, the current device, the rotation's handle.
#pragma once

#include "../../include/tova.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "tova_rope.cuh"

// tova_api.cu
int encode_state_map(CUtensorMap* map, void* base, const tova_config& cfg, int box_rows, long long rows_per_head);
int encode_map(CUtensorMap* map, void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box);

namespace tova_host {

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
inline bool device_info(DeviceInfo* out) {
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

}  // namespace tova_host
using namespace tova_host;

// Frequencies and factor of a rotation.
struct tova_rope {
  tova_rope_config cfg;
  double turns[tova::ROPE_MAX_PAIRS];   // w_i / 2 pi
  float factor;                         // m
};
