// What the attention kernels share: how calls are laid out over workgroups, the rows
// of a tile, the key ranges of a split, and small vector helpers.
#pragma once

#include "cache_internal.h"

#include <algorithm>
#include <type_traits>

namespace lssvm {

// How one call is laid out. A tile is `rows` rows of one sequence and key/value head
// (row r is token r / group, head r % group of the group); its keys may be split over
// `splits` workgroups, whose parts one more launch joins.
struct AttentionPlan {
  bool few;          // tiles of 16 rows, keys streamed through registers
  bool wide;         // ... by eight waves in place of four
  int rows;          // rows per tile
  int64_t tiles;     // at most so many tiles of one head
  int splits;
  int64_t pitch;     // stored scores per row (few rows with weights), else 0
};

struct AttentionArgs {
  lssvm_cache c;
  const void* q;
  void* out;
  Stride2 qs, os;
  int64_t tokens;
  int heads, group;
  const int32_t* offsets;
  float scale2;   // scale * log2(e): exponents are of two
  bool causal, accumulate;
  float* weight_out;
  Stride2 ws;
  AttentionPlan plan;
  // workspace
  float* lse;          // per row: log2 of the sum of exponentials (with weights)
  float* part;         // splits x rows x dim: sums of one split, and
  float2* part_ml;     // ... its maximum and sum of exponentials; the latter negative where
                       // keys are seen, but all with scores of minus infinity
  float* scores;       // rows x pitch
};

// Keys per step of either kernel, and the fewest steps of a split.
template <typename T>
constexpr int few_keys = sizeof(T) == 2 ? 32 : 16;
template <typename T>
constexpr int chunk_keys = sizeof(T) == 2 ? 64 : 32;
constexpr int kFewLeast = 4, kChunkLeast = 4;

// Probabilities are 2^(score - maximum so far), at most 1 (few rows) or 2^8 (chunks, whose
// maximum may lag). For the product they take the stored type, of which fp16 has a short
// range: 2^-14 is its least normal number, where a cache of many keys needs weights far
// below that. So fp16 ones are lifted by kLift exponents, up to the top of the range; and
// those that still lie below 2^kFaint are multiplied apart, kFar exponents higher, in steps
// that have any. Full rounding then holds down to 2^-50 of the largest weight. Sums are
// lifted alike, maxima lowered by as much where they leave a kernel. 2 x 2048 rows over
// 8192 keys, 16/4 heads of 128: 409 us with scores of deviation 1.5, where hardly a step
// has faint ones; 618 with 6, where most have (bf16 383, 389). 64 single tokens over
// 16384 keys: 706 either way.
template <typename T>
constexpr bool kShort = std::is_same_v<T, f16_t>;
template <typename T>
constexpr int few_lift = kShort<T> ? 15 : 0;     // two parts: the low one 2^11 below the high
constexpr int kFewFaint = -10, kFewFar = 25;
template <typename T>
constexpr int chunk_lift = kShort<T> ? 7 : 0;
constexpr int kChunkFaint = -14, kChunkFar = 29;

// Sums of values up to the largest of their type overflow where their mean does not. Sums
// of up to kSafeSum are joined as they are (512 of them are finite); where one is larger
// or not finite, the keys are gone over again, with values that are not finite apart and
// probabilities so much smaller that sums over `keys` of them stay in range. (fp16 values
// cannot get there.)
constexpr float kSafeSum = 5.192296858534828e33f;   // 2^112
template <typename T>
__device__ inline float lowered(int lift, int most, int keys) {
  return kShort<T> ? lift : -(float)(most + 33 - __clz(keys));   // p <= 2^most
}
// ------------------------------------------------------------- device -------

struct Tile {
  int s, length, n;      // sequence, its keys and rows (tokens)
  int64_t first;         // its first token
  int row0, rows;        // first row of the tile, rows of it that exist
  int keys;              // keys that some row of the tile sees
};

// Keys that row r (of the sequence) sees.
LSSVM_DEV int seen_keys(const AttentionArgs& a, const Tile& t, int r) {
  const int k = a.causal ? t.length - t.n + r / a.group + 1 : t.length;
  return k > 0 ? k : 0;
}

LSSVM_DEV void sequence_rows(const AttentionArgs& a, int s, int64_t* first, int* n) {
  *first = clip(a.offsets[s], a.tokens);
  const int64_t end = clip(a.offsets[s + 1], a.tokens);
  *n = end > *first ? (int)(end - *first) : 0;
}

// The index-th tile over all sequences, found by a wave with a sequence per lane;
// false behind the last. The result is uniform over the wave.
LSSVM_DEV bool find_tile(const AttentionArgs& a, int64_t index, int rows, Tile* t) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int base = 0; base < a.c.sequences; base += 64) {
    int64_t first = 0;
    int n = 0, length = 0;
    if (base + lane < a.c.sequences) {
      sequence_rows(a, base + lane, &first, &n);
      length = cache_length(a.c, base + lane);
    }
    const int64_t mine = ((int64_t)n * a.group + rows - 1) / rows;
    int64_t to = mine;
    for (int d = 1; d < 64; d <<= 1) {
      const int64_t o = __shfl_up(to, d);
      if (lane >= d) to += o;
    }
    const uint64_t behind = __ballot(before + to > index);
    if (behind) {
      const int at = __ffsll((unsigned long long)behind) - 1;
      const int64_t skipped = before + __shfl(to - mine, at);
      t->s = __builtin_amdgcn_readfirstlane(base + at);
      first = __shfl(first, at);
      t->first = (int64_t)__builtin_amdgcn_readfirstlane((int)(first >> 32)) << 32 |
                 (uint32_t)__builtin_amdgcn_readfirstlane((int)first);
      t->n = __builtin_amdgcn_readfirstlane(__shfl(n, at));
      t->length = __builtin_amdgcn_readfirstlane(__shfl(length, at));
      t->row0 = __builtin_amdgcn_readfirstlane((int)(index - skipped) * rows);
      t->rows = min(rows, t->n * a.group - t->row0);
      t->keys = seen_keys(a, *t, t->row0 + t->rows - 1);
      return true;
    }
    before += __shfl(to, 63);
  }
  return false;
}

// What workgroup blockIdx.x of a grid of work_groups() does: tile, split and head; false
// for the few too many. Workgroups go to the XCDs in turn, so every eighth takes the
// next piece of work: an XCD works on neighbouring tiles, which read the same keys.
inline int64_t work_groups(const AttentionArgs& a) {
  return (a.plan.tiles * a.plan.splits * a.c.heads + 7) / 8 * 8;
}
LSSVM_DEV bool find_work(const AttentionArgs& a, int64_t* tile, int* split, int* head) {
  const int64_t count = a.plan.tiles * a.plan.splits * a.c.heads, each = (count + 7) / 8;
  const int64_t work = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  if ((blockIdx.x >> 3) >= each || work >= count) return false;
  const int64_t pair = work / a.plan.tiles;
  *tile = work - pair * a.plan.tiles;
  *head = (int)(pair / a.plan.splits);
  *split = (int)(pair - (int64_t)*head * a.plan.splits);
  return true;
}

// Blocks of `block` keys per split, of which a tile uses ceil(blocks / per): short
// sequences use fewer splits than the call has, none of fewer than `least` blocks.
LSSVM_DEV int split_blocks(int keys, int block, int splits, int least) {
  const int blocks = (keys + block - 1) / block;
  return max((blocks + splits - 1) / splits, least);
}

// The larger of x in this lane and in the lanes 32 (16) apart.
LSSVM_DEV float max_across_32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
LSSVM_DEV float max_across_16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// Zeros, for loads that have nothing else to load.
static __device__ const u32x4 kNothing[1] = {};

// A load that is known to be from global memory, where the compiler cannot tell.
template <typename V, typename T>
LSSVM_DEV V load_global(const T* p) {
  return *reinterpret_cast<const __attribute__((address_space(1))) V*>(
      reinterpret_cast<uintptr_t>(p));
}

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// A word of one or two values of T with zeros where they are not finite, and a word of
// codes for those: small numbers of which sums of up to 63 tell how many infinities of
// either sign and NaNs there were. Times kCodeNan they count as NaNs: what is not finite
// gives that under a weight of exactly 0.
constexpr float kCodePlus = 1.0f, kCodeMinus = 64.0f, kCodeNan = 4096.0f;
template <typename T>
LSSVM_DEV u32x2 take_wild(uint32_t word) {
  typedef T tn __attribute__((ext_vector_type(4 / sizeof(T))));
  tn x = __builtin_bit_cast(tn, word), c{};
#pragma unroll
  for (int i = 0; i < 4 / (int)sizeof(T); ++i) {
    const float v = (float)x[i];
    if (__builtin_isfinite(v)) continue;
    c[i] = (T)(v != v ? kCodeNan : v > 0 ? kCodePlus : kCodeMinus);
    x[i] = (T)0.0f;
  }
  return u32x2{__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, c)};
}
LSSVM_DEV float decode_wild(float sum) {
  const int c = (int)sum;
  const bool plus = c & 63, minus = c >> 6 & 63, nan = c >= 4096;
  return nan || (plus && minus) ? __builtin_nanf("") : plus ? INFINITY : minus ? -INFINITY : 0.0f;
}

}  // namespace lssvm
