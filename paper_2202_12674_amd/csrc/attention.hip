// Attention of new tokens over a paged cache (include/lssvm_cache.h).
#include "cache_internal.h"

#include <algorithm>

namespace lssvm {
namespace {

// One wave per row and head: 64 keys at a time, a key's score on a lane, with the
// running maximum and sum of the softmax; then the values, four of a head on a lane.
// Sums are fp32, exponents of two.
constexpr int kRows = 4;   // rows a block
template <typename T>
__global__ void __launch_bounds__(64 * kRows) k_attention(AttentionArgs a, float* lse) {
  __shared__ float q[kRows][256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t = (int64_t)blockIdx.x * kRows + wave;
  const int h = blockIdx.y, group = a.heads / (int)a.c.heads, hk = h / group;
  const int dim = (int)a.c.dim;
  if (t >= a.tokens) return;
  int s = 0;
  while (s + 1 < a.c.sequences && a.offsets[s + 1] <= t) ++s;
  const int64_t first = clip(a.offsets[s], a.tokens), end = clip(a.offsets[s + 1], a.tokens);
  if (t < first || t >= end) return;
  const int L = cache_length(a.c, s);
  const int64_t seen = a.causal ? L - (end - first) + (t - first) + 1 : L;
  const int keys = (int)(seen < 0 ? 0 : seen);
  const T* qr = static_cast<const T*>(a.q) + t * a.qs.outer + h * a.qs.head;
  for (int i = lane; i < dim; i += 64) q[wave][i] = (float)qr[i];

  float m = -INFINITY, l = 0.0f, o[4] = {0, 0, 0, 0};
  for (int j0 = 0; j0 < keys; j0 += 64) {
    int slot = 0;
    const int page = j0 + lane < keys ? cache_page(a.c, s, j0 + lane, &slot) : -1;
    float x = -INFINITY;
    if (page >= 0) {
      const T* k = static_cast<const T*>(a.c.k) + page * a.c.k_stride[0] + hk * a.c.k_stride[1] +
                   slot * a.c.k_stride[2];
      float sum = 0.0f;
      for (int i = 0; i < dim; ++i) sum += q[wave][i] * (float)k[i];
      x = sum * a.scale2;
    }
    float top = x;
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float next = fmaxf(m, top), base = next == -INFINITY ? 0.0f : next;
    const float p = __builtin_amdgcn_exp2f(x - base), old = __builtin_amdgcn_exp2f(m - base);
    m = next;
    l = l * old + p;   // of this lane's keys
    for (int i = 0; i < 4; ++i) o[i] *= old;
    for (int jj = 0; jj < 64; ++jj) {
      const int pj = __shfl(page, jj), sj = __shfl(slot, jj);
      const float w = __shfl(p, jj);
      if (pj < 0) continue;
      const T* v = static_cast<const T*>(a.c.v) + pj * a.c.v_stride[0] + hk * a.c.v_stride[1] +
                   sj * a.c.v_stride[2];
      for (int i = 0; i < 4; ++i)
        if (4 * lane + i < dim) o[i] += w * (float)v[4 * lane + i];
    }
  }
  for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d);
  T* y = static_cast<T*>(a.out) + t * a.os.outer + h * a.os.head;
  for (int i = 0; i < 4; ++i)
    if (4 * lane + i < dim) y[4 * lane + i] = (T)(l == 0.0f ? 0.0f : o[i] / l);
  if (lse && lane == 0) lse[t * a.heads + h] = l == 0.0f ? INFINITY : m + log2f(l);
}

// One thread per key and head: the weights of all its rows, from the sums above.
template <typename T>
__global__ void __launch_bounds__(256) k_weights(AttentionArgs a, const float* lse) {
  const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int hk = blockIdx.y, s = blockIdx.z, group = a.heads / (int)a.c.heads;
  const int dim = (int)a.c.dim, L = cache_length(a.c, s);
  if (j >= L) return;
  int slot;
  const int page = cache_page(a.c, s, (int)j, &slot);
  if (page < 0) return;
  const int64_t first = clip(a.offsets[s], a.tokens), end = clip(a.offsets[s + 1], a.tokens);
  const T* k = static_cast<const T*>(a.c.k) + page * a.c.k_stride[0] + hk * a.c.k_stride[1] +
               slot * a.c.k_stride[2];
  float gain = 0.0f;
  for (int64_t t = first; t < end; ++t) {
    if (a.causal && j > L - (end - first) + (t - first)) continue;
    for (int h = hk * group; h < (hk + 1) * group; ++h) {
      const T* q = static_cast<const T*>(a.q) + t * a.qs.outer + h * a.qs.head;
      float sum = 0.0f;
      for (int i = 0; i < dim; ++i) sum += (float)q[i] * (float)k[i];
      gain += __builtin_amdgcn_exp2f(sum * a.scale2 - lse[t * a.heads + h]);
    }
  }
  const float old = a.c.weight[page * a.c.weight_stride[0] + hk * a.c.weight_stride[1] + slot];
  a.weight_out[page * a.ws.outer + hk * a.ws.head + slot] = old + gain;
}

template <typename T>
hipError_t launch(const AttentionArgs& a, float* lse, hipStream_t stream) {
  if (a.tokens > 0)
    k_attention<T><<<dim3((unsigned)((a.tokens + kRows - 1) / kRows), (unsigned)a.heads),
                     64 * kRows, 0, stream>>>(a, a.accumulate ? lse : nullptr);
  if (a.accumulate)
    k_weights<T><<<dim3((unsigned)((a.c.columns * a.c.page + 255) / 256), (unsigned)a.c.heads,
                        (unsigned)a.c.sequences),
                   256, 0, stream>>>(a, lse);
  return hipGetLastError();
}

}  // namespace

size_t attention_workspace(const lssvm_cache&, int64_t tokens, int heads, bool accumulate) {
  return 256 + (accumulate ? (size_t)tokens * heads * sizeof(float) : 0);
}

hipError_t launch_attention(const AttentionArgs& a, void* workspace, hipStream_t stream) {
  float* lse = static_cast<float*>(workspace);
  if (a.c.dtype == LSSVM_BF16) return launch<bf16_t>(a, lse, stream);
  if (a.c.dtype == LSSVM_F16) return launch<f16_t>(a, lse, stream);
  return launch<float>(a, lse, stream);
}

}  // namespace lssvm
