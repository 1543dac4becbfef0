// Kernels around a paged key/value cache (include/lssvm_cache.h): rotary positions,
// writing new tokens, eviction by weight. All of them move memory; what they compute
// hides behind that.
#include "cache_internal.h"

#include <algorithm>

namespace lssvm {
namespace {

constexpr int kThreads = 256;
// Blocks of one launch, whose grid has less than 2^32 threads along a side; what needs
// more goes in pieces.
constexpr int64_t kMostBlocks = 1 << 23;

// ------------------------------------------------------ rotary positions ----

// cos and sin of `angle`, to about an ulp of fp32: the quarter turns are taken off in
// fp64 (pi/2 in two parts), so that positions of millions lose nothing; what is left is
// at most pi/4, where the Taylor polynomials of degree 9 and 10 are off by 2e-9 and 2e-10.
// From kFarAngle = 2^45 on the rounding of k shows in what is left (turn_far).
constexpr double kFarAngle = 35184372088832.0;
LSSVM_DEV void turn(double angle, float* c, float* s) {
  const double k = rint(angle * 0.63661977236758134308);
  double rest = fma(-k, 1.57079632679489655800, angle);
  rest = fma(-k, 6.12323399573676603587e-17, rest);
  const float r = (float)rest, q = r * r;
  const float sr = r + r * q * (-1.0f / 6 + q * (1.0f / 120 + q * (-1.0f / 5040 + q * (1.0f / 362880))));
  const float cr = 1.0f + q * (-0.5f + q * (1.0f / 24 + q * (-1.0f / 720 + q * (1.0f / 40320 +
                                                                             q * (-1.0f / 3628800)))));
  // of k, the last two bits
  const int quarter = (int)(k - 4.0 * floor(0.25 * k));
  const float a = quarter & 1 ? sr : cr, b = quarter & 1 ? cr : sr;
  *c = quarter == 1 || quarter == 2 ? -a : a;
  *s = quarter >= 2 ? -b : b;
}

// A head's values are handled in chunks of 16 bytes: first those of the turned part
// (half layout: 16 bytes from either half), then those that are copied.
template <typename T>
__host__ __device__ inline int pair_chunks(int pairs, bool interleaved) {
  const int v = interleaved ? kVec<T> / 2 : kVec<T>;
  return (pairs + v - 1) / v;
}
template <typename T>
__host__ __device__ inline int copy_chunks(int values) {
  return (values + kVec<T> - 1) / kVec<T>;
}

LSSVM_DEV double position(const RotaryArgs& a, int64_t t) {
  return a.wide_positions ? (double)static_cast<const int64_t*>(a.positions)[t]
                          : (double)static_cast<const int32_t*>(a.positions)[t];
}

// The factors of the pairs of chunk `at` (of its last pair behind the last one).
template <typename T, bool INTER>
struct Factors {
  static constexpr int N = INTER ? kVec<T> / 2 : kVec<T>;
  float c[N], s[N];
  // false if an angle is too far for them
  LSSVM_DEV bool set(const RotaryArgs& a, int64_t t, int at) {
    double f[N];
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = a.freqs[min(at * N + i, a.pairs - 1)];
    const double p = position(a, t);
    bool near = true;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      near &= fabs(p * f[i]) < kFarAngle;
      turn(p * f[i], &c[i], &s[i]);
      c[i] *= a.scale;
      s[i] *= a.transpose ? -a.scale : a.scale;
    }
    return near;
  }
};

// The pairs of chunk `at` of every groups-th head, with sincos, which reduces angles of
// any size: a path of its own, so that the others' registers and code do not grow by it
// (within `turn` small calls took 0.6 us more).
template <typename T, bool INTER>
LSSVM_DEV void turn_far(const RotaryArgs& a, int64_t t, int at, const T* x, T* y, int64_t y_head,
                        int group, int groups) {
  constexpr int N = Factors<T, INTER>::N;
#pragma unroll 1
  for (int i = at * N; i < min(at * N + N, a.pairs); ++i) {
    double ds, dc;
    sincos(position(a, t) * a.freqs[i], &ds, &dc);
    const float c = (float)dc * a.scale, s = (float)ds * (a.transpose ? -a.scale : a.scale);
    const int m = INTER ? 2 * i : i, n = INTER ? 2 * i + 1 : i + a.pairs;
#pragma unroll 1
    for (int h = group; h < a.heads; h += groups) {
      const float p = (float)x[h * a.xs.head + m], q = (float)x[h * a.xs.head + n];
      y[h * y_head + m] = (T)(p * c - q * s);
      y[h * y_head + n] = (T)(q * c + p * s);
    }
  }
}

// Chunk `at` of the pairs of one head: read, turned, written. All of it is read before
// any is written, so y may be x.
template <typename T, bool INTER>
struct Pairs {
  static constexpr int N = Factors<T, INTER>::N, W = kVec<T>;
  typedef T vec __attribute__((ext_vector_type(W)));
  vec a, b;   // interleaved: a alone
  static LSSVM_DEV vec get(const T* x) {
    return __builtin_bit_cast(vec, *reinterpret_cast<const Loose<T, W>*>(x));
  }
  static LSSVM_DEV void put(T* y, vec v) {
    *reinterpret_cast<Loose<T, W>*>(y) = __builtin_bit_cast(Loose<T, W>, v);
  }
  LSSVM_DEV void read(const T* x, int at, int pairs) {
    const int left = pairs - at * N;
    x += at * (INTER ? W : N);
    if (left >= N) {
      a = get(x);
      if constexpr (!INTER) b = get(x + pairs);
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const bool in = (INTER ? i / 2 : i) < left;
        a[i] = in ? x[i] : (T)0.0f;
        if constexpr (!INTER) b[i] = in ? x[i + pairs] : (T)0.0f;
      }
    }
  }
  LSSVM_DEV void turn(const Factors<T, INTER>& f) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (INTER) {
        const float p = (float)a[2 * i], q = (float)a[2 * i + 1];
        a[2 * i] = (T)(p * f.c[i] - q * f.s[i]);
        a[2 * i + 1] = (T)(q * f.c[i] + p * f.s[i]);
      } else {
        const float p = (float)a[i], q = (float)b[i];
        a[i] = (T)(p * f.c[i] - q * f.s[i]);
        b[i] = (T)(q * f.c[i] + p * f.s[i]);
      }
    }
  }
  LSSVM_DEV void write(T* y, int at, int pairs) const {
    const int left = pairs - at * N;
    y += at * (INTER ? W : N);
    if (left >= N) {
      put(y, a);
      if constexpr (!INTER) put(y + pairs, b);
    } else {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        if ((INTER ? i / 2 : i) >= left) break;
        y[i] = a[i];
        if constexpr (!INTER) y[i + pairs] = b[i];
      }
    }
  }
};

// Copies chunk `at` of `n` values.
template <typename T>
LSSVM_DEV void copy_chunk(const T* x, T* y, int at, int n) {
  constexpr int W = kVec<T>;
  x += at * W;
  y += at * W;
  const int left = n - at * W;
  if (left >= W) {
    *reinterpret_cast<Loose<T, W>*>(y) = *reinterpret_cast<const Loose<T, W>*>(x);
  } else {
    for (int i = 0; i < left; ++i) y[i] = x[i];
  }
}

// Heads that a thread handles one after the other with the same factors: as many as
// leave `enough` threads, since a chunk's sines cost more than its 16 bytes, and a
// few tokens need the threads more. Rotation alone wants eight times what the chip
// holds, to even out its end (16384 tokens x 32 heads x 128, 1/4, 1/2, 1 and 2 x 2^20
// threads: 65, 51, 45 and 42 us); an appending thread first looks up where its token
// goes, and half as many as the chip holds do best (9 x 2048 tokens x 8 heads x 128,
// 1/4, 1/2, 1 and 2 x 2^20: 24, 23, 27 and 47 us).
constexpr int64_t kRotaryThreads = 2 << 20, kAppendThreads = 1 << 19;
inline int heads_per_thread(int64_t tokens, int chunks, int heads, int64_t enough) {
  const int64_t threads = tokens * chunks * heads;
  return (int)std::max<int64_t>(1, std::min<int64_t>(heads, threads / enough));
}

// v / by and the rest; in 32 bits where they do.
LSSVM_DEV int64_t split(int64_t v, int by, int* rest) {
  const int64_t q = v >> 32 ? v / by : (int64_t)((uint32_t)v / (uint32_t)by);
  *rest = (int)(v - q * by);
  return q;
}

// Measured: bf16, 16384 tokens x 32 heads x 128, 268 MB, in 42 us (6.3 TB/s, in part from
// the cache behind the L2s); fp32, 3001 x 12 x 80, 23 MB, in 6.3 us.
template <typename T, bool INTER>
__global__ void __launch_bounds__(kThreads) k_rotary(RotaryArgs a, int chunks, int turned,
                                                     int groups) {
  int at, group;
  const int64_t t = split(split((int64_t)blockIdx.x * kThreads + threadIdx.x, chunks, &at),
                          groups, &group);
  if (t >= a.tokens) return;
  const T* x = static_cast<const T*>(a.x) + t * a.xs.outer;
  T* y = static_cast<T*>(a.out) + t * a.os.outer;
  if (at >= turned) {
    for (int h = group; h < a.heads; h += groups)
      copy_chunk(x + h * a.xs.head + 2 * a.pairs, y + h * a.os.head + 2 * a.pairs, at - turned,
                 a.dim - 2 * a.pairs);
    return;
  }
  // the next head is read before this one is written
  Pairs<T, INTER> now, next;
  now.read(x + group * a.xs.head, at, a.pairs);
  Factors<T, INTER> f;
  if (!f.set(a, t, at)) {
    turn_far<T, INTER>(a, t, at, x, y, a.os.head, group, groups);
    return;
  }
  for (int h = group; h < a.heads; h += groups) {
    if (h + groups < a.heads) next.read(x + (h + groups) * a.xs.head, at, a.pairs);
    now.turn(f);
    now.write(y + h * a.os.head, at, a.pairs);
    now = next;
  }
}

template <typename F>
hipError_t by_dtype(int dtype, F f) {
  if (dtype == LSSVM_BF16) return f(bf16_t{});
  if (dtype == LSSVM_F16) return f(f16_t{});
  return f(float{});
}

// -------------------------------------------------------- cache append ------

// One chunk of a new token's key or value per thread, for some of its heads. Measured: 9
// x 2048 tokens x 8 heads x 128, 110 MB, in 24 us (4.6 TB/s); 64 tokens in 5.3 us, a
// chain of loads (offsets, length, page).
template <typename T, bool INTER>
__global__ void __launch_bounds__(kThreads) k_append(AppendArgs a, unsigned from_block,
                                                     int chunks, int turned, int copied,
                                                     int groups) {
  // every `stride`-th offset, so that the search for a token's sequence is one in LDS
  __shared__ int32_t some[kThreads];
  const int sequences = (int)a.c.sequences, stride = (sequences + kThreads - 1) / kThreads;
  const int held = (sequences + stride - 1) / stride;
  if ((int)threadIdx.x < held) some[threadIdx.x] = a.offsets[threadIdx.x * stride];
  __syncthreads();
  int at, group;
  const int64_t item = (int64_t)(from_block + blockIdx.x) * kThreads + threadIdx.x;
  const int64_t t = split(split(item, chunks, &at), groups, &group);
  if (t >= a.k.tokens) return;
  const T* xk = static_cast<const T*>(a.k.x) + t * a.k.xs.outer;
  const T* xv = static_cast<const T*>(a.v) + t * a.vs.outer;
  Factors<T, INTER> f;
  Pairs<T, INTER> pairs;
  bool near = true;
  if (at < turned) {
    pairs.read(xk + group * a.k.xs.head, at, a.k.pairs);
    near = f.set(a.k, t, at);
  }
  // the sequence: the last whose first token is not behind t
  int lo = 0, hi = held;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (some[mid] <= t) lo = mid; else hi = mid;
  }
  lo *= stride;
  hi = min(lo + stride, sequences);
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.offsets[mid] <= t) lo = mid; else hi = mid;
  }
  const int64_t first = clip(a.offsets[lo], a.k.tokens), end = clip(a.offsets[lo + 1], a.k.tokens);
  if (t < first || t >= end) return;
  const int64_t j = cache_length(a.c, lo) - (end - t);
  if (j < 0) return;
  int slot;
  const int page = cache_page(a.c, lo, (int)j, &slot);
  if (page < 0) return;
  T* k = static_cast<T*>(a.c.k) + page * a.c.k_stride[0] + slot * a.c.k_stride[2];
  T* v = static_cast<T*>(a.c.v) + page * a.c.v_stride[0] + slot * a.c.v_stride[2];
  if (!near) {
    turn_far<T, INTER>(a.k, t, at, xk, k, a.c.k_stride[1], group, groups);
    return;
  }
  for (int h = group; h < a.k.heads; h += groups) {
    if (at < turned) {
      if (h != group) pairs.read(xk + h * a.k.xs.head, at, a.k.pairs);
      pairs.turn(f);
      pairs.write(k + h * a.c.k_stride[1], at, a.k.pairs);
    } else if (at < turned + copied) {
      copy_chunk(xk + h * a.k.xs.head + 2 * a.k.pairs, k + h * a.c.k_stride[1] + 2 * a.k.pairs,
                 at - turned, a.k.dim - 2 * a.k.pairs);
    } else {
      copy_chunk(xv + h * a.vs.head, v + h * a.c.v_stride[1], at - turned - copied, a.k.dim);
    }
    if (at == chunks - 1 && a.c.weight)
      a.c.weight[page * a.c.weight_stride[0] + h * a.c.weight_stride[1] + slot] = 0.0f;
  }
}

// ------------------------------------------------------------- eviction -----

// Floats as integers of the same order: -0 as 0, NaN below all.
LSSVM_DEV uint32_t weight_order(float w) {
  if (w != w) return 0;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kSelectKeys = 24 * 1024;   // keys of a sequence that LDS holds: 96 KB

// One head of one sequence: the border, the m-th largest weight of the keys before
// the recent ones, by four rounds over 8 bits of the ordered integers each; then the
// kept indices in order, every wave a run of its own.
__global__ void __launch_bounds__(kSelectThreads) k_evict_select(EvictArgs a) {
  extern __shared__ uint32_t held[];
  __shared__ uint32_t bins[256];
  __shared__ uint32_t border, above;
  __shared__ int count_over[kSelectWaves], count_equal[kSelectWaves];
  const int s = blockIdx.x, h = blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int L = cache_length(a.from, s);
  const int n = min(L, a.budget);
  const int recent = min(n, a.recent), old = L - recent, m = n - recent;
  int32_t* kept = a.kept + ((int64_t)s * a.from.heads + h) * a.budget;
  for (int i = n + tid; i < a.budget; i += kSelectThreads) kept[i] = -1;
  if (h == 0 && tid == 0) a.to.lengths[s] = n;
  for (int i = tid; i < recent; i += kSelectThreads) kept[m + i] = old + i;
  if (m == 0) return;

  const bool fits = old <= kSelectKeys;
  auto fetch = [&](int j) -> uint32_t {
    int slot;
    const int p = cache_page(a.from, s, j, &slot);
    return p < 0 ? 0
                 : weight_order(a.from.weight[p * a.from.weight_stride[0] +
                                              h * a.from.weight_stride[1] + slot]);
  };
  if (fits)
    for (int j = tid; j < old; j += kSelectThreads) held[j] = fetch(j);
  auto key = [&](int j) -> uint32_t { return fits ? held[j] : fetch(j); };

  if (tid == 0) border = 0, above = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) bins[tid] = 0;
    __syncthreads();
    const uint32_t known = border, mask = shift == 24 ? 0 : 0xFFFFFFFFu << (shift + 8);
    for (int j = tid; j < old; j += kSelectThreads) {
      const uint32_t u = key(j);
      if ((u & mask) == known) atomicAdd(&bins[(u >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid < 64) {   // from the largest value down: four bins a lane
      uint32_t c[4], sum = 0;
      for (int i = 0; i < 4; ++i) c[i] = bins[255 - 4 * lane - i], sum += c[i];
      uint32_t before = sum;
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(before, d);
        if (lane >= d) before += o;
      }
      before = above + before - sum;
      for (int i = 0; i < 4; ++i) {
        if (before < (uint32_t)m && before + c[i] >= (uint32_t)m) {
          border = known | ((uint32_t)(255 - 4 * lane - i) << shift);
          above = before;
        }
        before += c[i];
      }
    }
    __syncthreads();
  }
  const uint32_t edge = border;
  const int equals = m - (int)above;   // of those at the border, so many first ones

  const int run = ((old + kSelectWaves - 1) / kSelectWaves + 63) & ~63;
  const int j0 = wave * run, j1 = min(old, j0 + run);
  int over = 0, equal = 0;
  for (int j = j0 + lane; j < j1; j += 64) {
    const uint32_t u = key(j);
    over += u > edge;
    equal += u == edge;
  }
  for (int d = 32; d; d >>= 1) over += __shfl_xor(over, d), equal += __shfl_xor(equal, d);
  if (lane == 0) count_over[wave] = over, count_equal[wave] = equal;
  __syncthreads();
  over = equal = 0;
  for (int w = 0; w < wave; ++w) over += count_over[w], equal += count_equal[w];
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int j = j0; j < j1; j += 64) {
    const bool in = j + lane < j1;
    const uint32_t u = in ? key(j + lane) : 0;
    const bool o = in && u > edge, e = in && u == edge;
    const uint64_t bo = __ballot(o), be = __ballot(e);
    const int mine = equal + __popcll(be & below);
    if (o || (e && mine < equals))
      kept[over + __popcll(bo & below) + min(mine, equals)] = j + lane;
    over += __popcll(bo);
    equal += __popcll(be);
  }
}

// Rows of keys and values, 16 bytes of each per thread and row. Measured: 6144 of 12288
// keys x 8 heads x 128 of 32 sequences, 1.6 GB, in 326 us (5.0 TB/s, as a large copy); the
// selection before it 22 us.
constexpr int kCopyRows = 4;   // rows in flight per thread
__global__ void __launch_bounds__(kThreads) k_evict_copy(EvictArgs a, int from_row, int lanes,
                                                         int size) {
  const int s = blockIdx.z, h = blockIdx.y;
  const int n = min(cache_length(a.from, s), a.budget);
  const int rows = kThreads / lanes;   // rows that a block moves at once
  const int row = threadIdx.x / lanes, at = threadIdx.x % lanes;
  if (row >= rows) return;
  const int32_t* kept = a.kept + ((int64_t)s * a.from.heads + h) * a.budget;
  const int first = from_row + blockIdx.x * rows * kCopyRows + row;
  const char* src[2][kCopyRows];
  char* dst[2][kCopyRows];
  bool move[kCopyRows], hole[kCopyRows];
#pragma unroll
  for (int r = 0; r < kCopyRows; ++r) {
    const int i = first + r * rows;
    move[r] = i < n;
    hole[r] = false;
    if (!move[r]) continue;
    int from_slot, to_slot;
    const int to = cache_page(a.to, s, i, &to_slot);
    const int from = cache_page(a.from, s, kept[i], &from_slot);
    move[r] = to >= 0;
    hole[r] = from < 0;
    auto place = [&](const int64_t* st, int p, int slot) {
      return (p * st[0] + h * st[1] + slot * st[2]) * size + 16 * at;
    };
    src[0][r] = static_cast<const char*>(a.from.k) + place(a.from.k_stride, from, from_slot);
    src[1][r] = static_cast<const char*>(a.from.v) + place(a.from.v_stride, from, from_slot);
    dst[0][r] = static_cast<char*>(a.to.k) + place(a.to.k_stride, to, to_slot);
    dst[1][r] = static_cast<char*>(a.to.v) + place(a.to.v_stride, to, to_slot);
    if (at == 0 && move[r])
      a.to.weight[to * a.to.weight_stride[0] + h * a.to.weight_stride[1] + to_slot] =
          hole[r] ? 0.0f
                  : a.from.weight[from * a.from.weight_stride[0] + h * a.from.weight_stride[1] +
                                  from_slot];
  }
  uint4 w[2][kCopyRows];
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int r = 0; r < kCopyRows; ++r)
      w[x][r] = move[r] && !hole[r] ? *reinterpret_cast<const uint4*>(src[x][r]) : uint4{};
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int r = 0; r < kCopyRows; ++r)
      if (move[r]) *reinterpret_cast<uint4*>(dst[x][r]) = w[x][r];
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream) {
  return by_dtype(a.dtype, [&](auto type) {
    using T = decltype(type);
    const int turned = pair_chunks<T>(a.pairs, a.interleaved);
    const bool in_place = a.x == a.out;
    const int chunks = turned + (in_place ? 0 : copy_chunks<T>(a.dim - 2 * a.pairs));
    if (chunks == 0) return hipSuccess;
    const int each = heads_per_thread(a.tokens, chunks, a.heads, kRotaryThreads);
    const int groups = (a.heads + each - 1) / each;
    const int64_t items = a.tokens * groups * chunks;
    const dim3 grid((unsigned)((items + kThreads - 1) / kThreads));
    if (a.interleaved)
      k_rotary<T, true><<<grid, kThreads, 0, stream>>>(a, chunks, turned, groups);
    else
      k_rotary<T, false><<<grid, kThreads, 0, stream>>>(a, chunks, turned, groups);
    return hipGetLastError();
  });
}

hipError_t launch_append(const AppendArgs& a, hipStream_t stream) {
  return by_dtype(a.c.dtype, [&](auto type) {
    using T = decltype(type);
    const int turned = pair_chunks<T>(a.k.pairs, a.k.interleaved);
    const int copied = copy_chunks<T>(a.k.dim - 2 * a.k.pairs);
    const int chunks = turned + copied + copy_chunks<T>(a.k.dim);
    const int each = heads_per_thread(a.k.tokens, chunks, a.k.heads, kAppendThreads);
    const int groups = (a.k.heads + each - 1) / each;
    const int64_t items = a.k.tokens * groups * chunks, blocks = (items + kThreads - 1) / kThreads;
    hipError_t e = hipSuccess;
    for (int64_t from = 0; from < blocks && e == hipSuccess; from += kMostBlocks) {
      const dim3 grid((unsigned)std::min(blocks - from, kMostBlocks));
      if (a.k.interleaved)
        k_append<T, true><<<grid, kThreads, 0, stream>>>(a, (unsigned)from, chunks, turned, copied,
                                                         groups);
      else
        k_append<T, false><<<grid, kThreads, 0, stream>>>(a, (unsigned)from, chunks, turned, copied,
                                                          groups);
      e = hipGetLastError();
    }
    return e;
  });
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t stream) {
  const int64_t most = a.from.columns * a.from.page;
  const size_t lds = 4 * (size_t)std::min<int64_t>(most, kSelectKeys);
  hipError_t e = hipSuccess;
  if (lds > 32 * 1024 &&
      (e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_evict_select),
                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)) !=
          hipSuccess)
    return e;
  k_evict_select<<<dim3((unsigned)a.from.sequences, (unsigned)a.from.heads), kSelectThreads, lds,
                   stream>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const int size = a.from.dtype == LSSVM_F32 ? 4 : 2;
  const int lanes = (int)a.from.dim * size / 16, rows = kThreads / lanes * kCopyRows;
  const int64_t n = std::min<int64_t>(a.budget, most), piece = rows * kMostBlocks;
  for (int64_t row = 0; row < n; row += piece) {
    const int64_t blocks = (std::min(n - row, piece) + rows - 1) / rows;
    k_evict_copy<<<dim3((unsigned)blocks, (unsigned)a.from.heads, (unsigned)a.from.sequences),
                   kThreads, 0, stream>>>(a, (int)row, lanes, size);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return e;
}

}  // namespace lssvm
