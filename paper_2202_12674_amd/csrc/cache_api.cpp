// Host side of include/lssvm_cache.h: argument checks and launches.
#include "attention.h"
#include "lssvm_error.h"

#include <algorithm>
#include <cmath>

namespace lssvm {
namespace {

constexpr int64_t kMaxHeads = 65535;
constexpr int64_t kMaxTokens = (int64_t(1) << 31) - 1;
// A launch's grid has less than 2^32 threads along each of its sides.
constexpr int64_t kMaxKeys = int64_t(1) << 29;      // of a sequence
constexpr int64_t kMaxRows = int64_t(1) << 30;      // tokens x heads
constexpr int64_t kMaxValues = int64_t(1) << 33;    // ... x dim
constexpr int64_t kMaxTables = int64_t(1) << 22;    // sequences x heads of a cache
constexpr int64_t kMaxSlotStride = int64_t(1) << 24;
constexpr int64_t kMaxStride = int64_t(1) << 40;

#define CACHE_TRY(expr)              \
  do {                               \
    int rc_ = (expr);                \
    if (rc_ != LSSVM_OK) return rc_; \
  } while (0)

int bad(const char* what) { return fail(LSSVM_EINVAL, "%s", what); }

int launched(hipError_t e) {
  return e == hipSuccess ? LSSVM_OK : fail(LSSVM_EHIP, "launch failed: %s", hipGetErrorString(e));
}

int64_t element(int32_t dtype) { return dtype == LSSVM_F32 ? 4 : 2; }

bool known(int32_t dtype) {
  return dtype == LSSVM_F32 || dtype == LSSVM_BF16 || dtype == LSSVM_F16;
}

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// Whether rows of `width` values at the given strides overlap nowhere: from the
// smallest stride up, each steps over all that lies within it.
bool apart(const int64_t* stride, const int64_t* count, int n, int64_t width) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + n, [&](int a, int b) { return stride[a] < stride[b]; });
  int64_t span = width;
  for (int i = 0; i < n; ++i) {
    const int k = order[i];
    if (count[k] == 1) continue;
    if (stride[k] < span) return false;
    span = stride[k] * (count[k] - 1) + span;
  }
  return true;
}

bool strides_in_range(const int64_t* stride, int n) {
  for (int i = 0; i < n; ++i)
    if (stride[i] < 0 || stride[i] > kMaxStride) return false;
  return true;
}

int check_cache(const lssvm_cache* c) {
  if (!c) return bad("cache is NULL");
  if (!known(c->dtype)) return bad("cache: dtype must be LSSVM_F32, LSSVM_BF16 or LSSVM_F16");
  if (!c->k || !c->v || !c->table || !c->lengths) return bad("cache: a NULL array");
  if (c->dim < 8 || c->dim > 256 || c->dim % 8)
    return fail(LSSVM_EINVAL, "cache: dim must be a multiple of 8 in 8 .. 256, not %lld",
                (long long)c->dim);
  if (c->pages < 1 || c->pages > kMaxTokens || c->heads < 1 || c->heads > kMaxHeads ||
      c->page < 1 || c->page > kMaxTokens || c->sequences < 1 || c->sequences > kMaxHeads)
    return bad("cache: pages, heads, page or sequences out of range");
  if (c->columns < 1 || c->columns > kMaxTokens || c->columns * c->page > kMaxKeys)
    return bad("cache: columns * page must be 1 .. 2^29");
  if (c->sequences * c->heads > kMaxTables) return bad("cache: more than 2^22 sequences x heads");
  if (c->table_stride < c->columns && c->sequences > 1)
    return bad("cache: table_stride must be at least columns");
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return bad("cache: k and v must be 16-byte aligned");
  const int64_t count[3] = {c->pages, c->heads, c->page};
  for (const int64_t* st : {c->k_stride, c->v_stride}) {
    if (!strides_in_range(st, 3) || (c->page > 1 && st[2] > kMaxSlotStride))
      return bad("cache: a stride out of range");
    for (int i = 0; i < 3; ++i)
      if (count[i] > 1 && st[i] * element(c->dtype) % 16)
        return bad("cache: rows of k and v must begin on 16 bytes");
    if (!apart(st, count, 3, c->dim)) return bad("cache: rows of k or v overlap");
  }
  if (c->weight && (!strides_in_range(c->weight_stride, 2) ||
                    !apart(c->weight_stride, count, 2, c->page)))
    return bad("cache: rows of weight overlap");
  return LSSVM_OK;
}

int check_rows(const char* name, const void* p, const int64_t* stride) {
  if (!p || !stride) return fail(LSSVM_EINVAL, "%s or its strides are NULL", name);
  if (!strides_in_range(stride, 2)) return fail(LSSVM_EINVAL, "%s: a stride out of range", name);
  return LSSVM_OK;
}

int check_out(const char* name, const void* p, const int64_t* stride, int64_t tokens,
              int64_t heads, int64_t dim) {
  CACHE_TRY(check_rows(name, p, stride));
  const int64_t count[2] = {tokens, heads};
  if (!apart(stride, count, 2, dim)) return fail(LSSVM_EINVAL, "%s: rows overlap", name);
  return LSSVM_OK;
}

// Whether rows at a and b may share a value; those at b are apart. Of equal strides, as of
// views of one array, it is known: rows i tokens and j heads from each other do if that
// leaves less than a row between their starts, and since a stride steps over all that lies
// within it, only the two multiples next to the distance can. Else it goes by all that
// lies between the first and the last value.
bool overlap(const void* a, const int64_t* as, const void* b, const int64_t* bs, int64_t tokens,
             int64_t heads, int64_t dim, int64_t size) {
  const auto span = [&](const int64_t* s) {
    return (s[0] * (tokens - 1) + s[1] * (heads - 1) + dim) * size;
  };
  const int64_t apart_by = reinterpret_cast<intptr_t>(b) - reinterpret_cast<intptr_t>(a);
  if (apart_by >= span(as) || -apart_by >= span(bs)) return false;
  if (apart_by % size || (tokens > 1 && as[0] != bs[0]) || (heads > 1 && as[1] != bs[1]))
    return true;
  struct { int64_t stride, count; } outer{bs[0], tokens}, inner{bs[1], heads};
  if (outer.count == 1 || (inner.count > 1 && outer.stride < inner.stride))
    std::swap(outer, inner);
  const auto near = [](auto d, int64_t left, auto use) {   // (of a single row, its own place)
    if (d.count == 1) return use(left);
    const int64_t low = left / d.stride - (left % d.stride < 0);
    for (int64_t n = low; n <= low + 1; ++n)
      if (std::abs(n) < d.count && use(left - n * d.stride)) return true;
    return false;
  };
  return near(outer, apart_by / size, [&](int64_t left) {
    return near(inner, left, [&](int64_t rest) { return std::abs(rest) < dim; });
  });
}

int check_sizes(int64_t tokens, int64_t heads, int64_t dim) {
  if (tokens < 0 || tokens > kMaxTokens) return bad("tokens must be 0 .. 2^31 - 1");
  if (heads < 1 || heads > kMaxHeads) return bad("heads must be 1 .. 65535");
  if (tokens * heads > kMaxRows || tokens * heads * dim > kMaxValues)
    return bad("more than 2^30 rows (tokens x heads) or 2^33 values");
  return LSSVM_OK;
}

int check_angles(const void* positions, int32_t position_bytes, const double* freqs,
                 int64_t pairs, int64_t dim, int64_t tokens, double scale) {
  if (pairs < 0 || 2 * pairs > dim) return bad("pairs must be 0 .. dim / 2");
  if (pairs > 0 && tokens > 0 && (!positions || !freqs)) return bad("positions or freqs is NULL");
  if (pairs > 0 && position_bytes != 4 && position_bytes != 8)
    return bad("position_bytes must be 4 or 8");
  if (pairs > 0 && (!aligned(positions, position_bytes) || !aligned(freqs, 8)))
    return bad("positions or freqs is not aligned");
  if (!std::isfinite((float)scale)) return bad("scale must be finite in single precision");
  return LSSVM_OK;
}

RotaryArgs rotary_args(const void* x, const int64_t* xs, int64_t tokens, int64_t heads,
                       int64_t dim, const void* positions, int32_t position_bytes,
                       const double* freqs, int64_t pairs, double scale, int32_t interleaved) {
  RotaryArgs a{};
  a.x = x;
  a.xs = {xs[0], xs[1]};
  a.tokens = tokens;
  a.heads = (int)heads;
  a.dim = (int)dim;
  a.pairs = (int)pairs;
  a.positions = positions;
  a.freqs = freqs;
  a.scale = (float)scale;
  a.wide_positions = position_bytes == 8;
  a.interleaved = interleaved != 0;
  return a;
}

}  // namespace
}  // namespace lssvm

using namespace lssvm;

extern "C" {

int lssvm_rotary_frequencies(int64_t pairs, double base, int32_t scaling, double factor,
                             double original, double* freqs, double* scale) {
  clear_error();
  if (pairs < 1 || pairs > (int64_t(1) << 20)) return bad("pairs must be 1 .. 2^20");
  if (!(base > 0) || !std::isfinite(base)) return bad("base must be positive and finite");
  if (!(factor >= 1) || !std::isfinite(factor)) return bad("factor must be finite and >= 1");
  if (scaling < LSSVM_ROPE_PLAIN || scaling > LSSVM_ROPE_YARN) return bad("unknown scaling");
  if (scaling == LSSVM_ROPE_YARN && !(original > 0 && std::isfinite(original)))
    return bad("original must be positive and finite");
  if (!freqs || !scale) return bad("freqs or scale is NULL");
  if (scaling == LSSVM_ROPE_NTK && pairs > 1)
    base *= std::pow(factor, (double)pairs / (double)(pairs - 1));
  for (int64_t i = 0; i < pairs; ++i) {
    double f = std::pow(base, -(double)i / (double)pairs);
    if (scaling == LSSVM_ROPE_LINEAR) f /= factor;
    if (scaling == LSSVM_ROPE_YARN) {
      const double turns = original * f / (2.0 * M_PI);
      const double keep = std::min(1.0, std::max(0.0, (turns - 1.0) / (32.0 - 1.0)));
      f = f / factor * (1.0 - keep) + f * keep;
    }
    freqs[i] = f;
  }
  *scale = scaling == LSSVM_ROPE_YARN ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return LSSVM_OK;
}

int lssvm_rotary(const void* x, const int64_t* x_stride, void* out, const int64_t* out_stride,
                 int64_t tokens, int64_t heads, int64_t dim, const void* positions,
                 int32_t position_bytes, const double* freqs, int64_t pairs, double scale,
                 int32_t interleaved, int32_t transpose, int32_t dtype, void* stream) {
  clear_error();
  if (!known(dtype)) return bad("dtype must be LSSVM_F32, LSSVM_BF16 or LSSVM_F16");
  if (dim < 1 || dim > kMaxHeads) return bad("dim must be 1 .. 65535");
  CACHE_TRY(check_sizes(tokens, heads, dim));
  CACHE_TRY(check_angles(positions, position_bytes, freqs, pairs, dim, tokens, scale));
  if (tokens == 0) return LSSVM_OK;
  CACHE_TRY(check_rows("x", x, x_stride));
  CACHE_TRY(check_out("out", out, out_stride, tokens, heads, dim));
  const int64_t size = element(dtype);
  if (!aligned(x, size) || !aligned(out, size)) return bad("x or out is not aligned");
  if (x == out) {
    if ((tokens > 1 && x_stride[0] != out_stride[0]) || (heads > 1 && x_stride[1] != out_stride[1]))
      return bad("in place, x and out need the same strides");
  } else if (overlap(x, x_stride, out, out_stride, tokens, heads, dim, size)) {
    return bad("x and out overlap");
  }
  RotaryArgs a = rotary_args(x, x_stride, tokens, heads, dim, positions, position_bytes, freqs,
                             pairs, scale, interleaved);
  a.out = out;
  a.os = {out_stride[0], out_stride[1]};
  a.transpose = transpose != 0;
  a.dtype = dtype;
  return launched(launch_rotary(a, static_cast<hipStream_t>(stream)));
}

int lssvm_cache_append(const lssvm_cache* cache, const void* k, const int64_t* k_stride,
                       const void* v, const int64_t* v_stride, int64_t tokens,
                       const int32_t* offsets, const void* positions, int32_t position_bytes,
                       const double* freqs, int64_t pairs, double scale, int32_t interleaved,
                       void* stream) {
  clear_error();
  CACHE_TRY(check_cache(cache));
  CACHE_TRY(check_sizes(tokens, cache->heads, cache->dim));
  CACHE_TRY(check_angles(positions, position_bytes, freqs, pairs, cache->dim, tokens,
                         scale));
  if (!offsets) return bad("offsets is NULL");
  if (tokens == 0) return LSSVM_OK;
  CACHE_TRY(check_rows("k", k, k_stride));
  CACHE_TRY(check_rows("v", v, v_stride));
  const int64_t size = element(cache->dtype);
  if (!aligned(k, size) || !aligned(v, size)) return bad("k or v is not aligned");
  AppendArgs a{};
  a.c = *cache;
  a.k = rotary_args(k, k_stride, tokens, cache->heads, cache->dim, positions, position_bytes,
                    freqs, pairs, scale, interleaved);
  a.v = v;
  a.vs = {v_stride[0], v_stride[1]};
  a.offsets = offsets;
  return launched(launch_append(a, static_cast<hipStream_t>(stream)));
}

size_t lssvm_attention_workspace_bytes(const lssvm_cache* cache, int64_t tokens, int64_t heads,
                                       int32_t accumulate) {
  clear_error();
  if (check_cache(cache) != LSSVM_OK || check_sizes(tokens, heads, cache->dim) != LSSVM_OK ||
      heads % cache->heads)
    return 0;
  return attention_workspace(*cache, tokens, (int)heads, accumulate != 0);
}

int lssvm_attention(const lssvm_cache* cache, const void* q, const int64_t* q_stride,
                    int64_t tokens, int64_t heads, const int32_t* offsets, double scale,
                    int32_t causal, int32_t accumulate, float* weight_out,
                    const int64_t* weight_out_stride, void* out, const int64_t* out_stride,
                    void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  CACHE_TRY(check_cache(cache));
  CACHE_TRY(check_sizes(tokens, heads, cache->dim));
  if (heads % cache->heads)
    return fail(LSSVM_EINVAL, "heads (%lld) must be a multiple of the cache's (%lld)",
                (long long)heads, (long long)cache->heads);
  if (!offsets) return bad("offsets is NULL");
  const float scale2 = (float)(scale * 1.4426950408889634074);   // exponents are of two
  if (!std::isfinite(scale2)) return bad("scale must be finite in single precision");
  AttentionArgs a{};
  if (accumulate) {
    if (!cache->weight) return bad("accumulate needs a cache with weights");
    a.weight_out = weight_out ? weight_out : cache->weight;
    const int64_t* st = weight_out ? weight_out_stride : cache->weight_stride;
    const int64_t count[2] = {cache->pages, cache->heads};
    if (!st || !strides_in_range(st, 2) || !apart(st, count, 2, cache->page))
      return bad("weight_out: strides missing or out of range, or rows overlap");
    a.ws = {st[0], st[1]};
  }
  if (tokens > 0) {
    CACHE_TRY(check_rows("q", q, q_stride));
    CACHE_TRY(check_out("out", out, out_stride, tokens, heads, cache->dim));
    const int64_t size = element(cache->dtype);
    if (!aligned(q, size) || !aligned(out, size)) return bad("q or out is not aligned");
    if (overlap(q, q_stride, out, out_stride, tokens, heads, cache->dim, size))
      return bad("q and out overlap");
    a.qs = {q_stride[0], q_stride[1]};
    a.os = {out_stride[0], out_stride[1]};
  }
  const size_t need = attention_workspace(*cache, tokens, (int)heads, accumulate != 0);
  if (!workspace || !aligned(workspace, 256)) return bad("workspace must be 256-byte aligned");
  if (workspace_bytes < need)
    return fail(LSSVM_EINVAL, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
  if (tokens == 0 && !accumulate) return LSSVM_OK;
  a.c = *cache;
  a.q = q;
  a.out = out;
  a.tokens = tokens;
  a.heads = (int)heads;
  a.group = (int)(heads / cache->heads);
  a.offsets = offsets;
  a.scale2 = scale2;
  a.causal = causal != 0;
  a.accumulate = accumulate != 0;
  return launched(launch_attention(a, workspace, static_cast<hipStream_t>(stream)));
}

int lssvm_cache_evict(const lssvm_cache* from, const lssvm_cache* to, int64_t budget,
                      int64_t recent, int32_t* kept, void* stream) {
  clear_error();
  CACHE_TRY(check_cache(from));
  CACHE_TRY(check_cache(to));
  if (!from->weight || !to->weight) return bad("both caches need weights");
  if (from->heads != to->heads || from->page != to->page || from->dim != to->dim ||
      from->dtype != to->dtype || from->sequences != to->sequences)
    return bad("the caches' heads, page, dim, dtype and sequences must be the same");
  if (from->lengths == to->lengths || from->table == to->table)
    return bad("the caches need tables and lengths of their own");
  if (budget < 1 || budget > to->columns * to->page)
    return bad("budget must be 1 .. the target's columns * page");
  if (recent < 0) return bad("recent must be >= 0");
  if (!kept) return bad("kept is NULL");
  EvictArgs a{};
  a.from = *from;
  a.to = *to;
  a.budget = (int)budget;
  a.recent = (int)std::min(recent, budget);
  a.kept = kept;
  return launched(launch_evict(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
