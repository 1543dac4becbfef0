// What the host side of include/lssvm_cache.h hands to its kernels.
#pragma once

#include "lssvm_cache.h"

#include <hip/hip_runtime.h>

namespace lssvm {

// Strides in elements: token and head, or page and head.
struct Stride2 {
  int64_t outer, head;
};

struct RotaryArgs {
  const void* x;
  void* out;
  Stride2 xs, os;
  int64_t tokens;
  int heads, dim, pairs;
  const void* positions;
  const double* freqs;
  float scale;
  int dtype;
  bool wide_positions, interleaved, transpose;
};
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream);

struct AppendArgs {
  lssvm_cache c;
  RotaryArgs k;   // x, strides, tokens, positions, frequencies of the new keys
  const void* v;
  Stride2 vs;
  const int32_t* offsets;
};
hipError_t launch_append(const AppendArgs& a, hipStream_t stream);

struct AttentionArgs;   // attention.h
size_t attention_workspace(const lssvm_cache& c, int64_t tokens, int heads, bool accumulate);
hipError_t launch_attention(AttentionArgs a, void* workspace, hipStream_t stream);

struct EvictArgs {
  lssvm_cache from, to;
  int budget, recent;
  int32_t* kept;
};
hipError_t launch_evict(const EvictArgs& a, hipStream_t stream);

// ------------------------------------------------------------- device -------
#ifdef __HIP_DEVICE_COMPILE__
#define LSSVM_DEV __device__ __forceinline__
#else
#define LSSVM_DEV __device__ inline
#endif

using bf16_t = __bf16;
using f16_t = _Float16;

// N values of T that need be aligned to one of them only (global loads and stores
// of up to 16 bytes take any such address on gfx950).
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Loose {
  T v[N];
};
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);   // values in 16 bytes

// Keys that sequence s has, as the kernels count them.
LSSVM_DEV int cache_length(const lssvm_cache& c, int s) {
  const int64_t most = c.columns * c.page;
  const int64_t n = c.lengths[s];
  return (int)(n < 0 ? 0 : n < most ? n : most);
}

// The page of key j, or -1 for a hole; *slot is its place there.
LSSVM_DEV int cache_page(const lssvm_cache& c, int s, int j, int* slot) {
  const uint32_t size = (uint32_t)c.page, column = (uint32_t)j / size;
  *slot = (int)((uint32_t)j - column * size);
  const int32_t p = c.table[s * c.table_stride + column];
  return p >= 0 && p < c.pages ? p : -1;
}

LSSVM_DEV int64_t clip(int64_t v, int64_t most) { return v < 0 ? 0 : v < most ? v : most; }

}  // namespace lssvm
