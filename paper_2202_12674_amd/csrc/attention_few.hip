// Attention of few rows per sequence (single tokens, and up to a few) over a paged
// cache: include/lssvm_cache.h.
#include "attention.h"

#include <climits>

namespace lssvm {
namespace {

// Third word of a raw buffer resource (32-bit data, no swizzle, no stride).
constexpr int kBufferWord3 = 0x00020000;
typedef const __attribute__((address_space(4))) int32_t* const_i32;

// The matrix cores on 16 keys x 16 rows.
template <typename T>
struct Mfma16;
template <>
struct Mfma16<bf16_t> {
  static LSSVM_DEV f32x4 mul(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mfma16<f16_t> {
  static LSSVM_DEV f32x4 mul(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mfma16<float> {
  // 16 contraction places as four products of 4
  static LSSVM_DEV f32x4 mul(u32x4 a, u32x4 b, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0,
                                               0, 0);
    return c;
  }
};

// What follows from the type and the width. Lane (m, g) = (lane % 16, lane / 16).
// Products run over 16-byte chunks of a row: chunk 4c + g is lane group g's share of
// step c, for keys and queries alike. Values: lane m holds CE consecutive ones of each
// of NC parts of a row, value 16 CE part + CE m + e; keys 16b + 4g + i, which is where
// the scores of its column stand, so that they never change lanes.
template <typename T, int D>
struct Shape {
  static constexpr int VE = kVec<T>;
  static constexpr int KEYS = few_keys<T>;               // of a step
  static constexpr int KB = KEYS / 16;                   // ... blocks of 16
  static constexpr int KC = D / (4 * VE);                // 16-byte chunks of a key per lane
  static constexpr int CE = D % (16 * VE) == 0 ? VE      // values of a chunk
                            : D / 16 < VE      ? D / 16
                                               : 2;
  static constexpr int CW = CE * (int)sizeof(T) / 4;     // ... in words
  static constexpr int NC = D / (16 * CE);
  static_assert(NC * 16 * CE == D && KC * 4 * VE == D, "whole parts and chunks");
  static constexpr int VR = 4 * KB;                      // rows of values per lane
};

// One tile of 16 rows against one split of its keys. Every wave takes 32 (fp32: 16)
// keys at a time straight from memory into registers, scores S^T = K Q^T, keeps the
// running maximum and sum of every row and adds O^T += V^T P^T. The values come in
// rows and are needed in columns: 8 x 8 of them are transposed by byte permutes, in
// fp32 the operand is a row already. Probabilities enter the 16-bit product as two
// 16-bit parts, since the matrix cores have the time (the kernel waits for memory).
// The waves' sums are joined in LDS.
//
// Keys of the next step are loaded as soon as the scores are formed, values as soon
// as the product is issued, so that a wave has loads in flight all the time. BLOCKS:
// the pages hold whole runs of 16 keys, whose page is then looked up once.
//
// Measured (bf16, 128 wide, 8 heads of a group of 4): 64 rows over 16384 keys each, 3.1
// GB, in 540 us, 5.7 TB/s (a large copy moves 5.1); with scores kept for the weights 665
// us, for 100 MB of them: stores among the loads cost more than their bytes, however
// they are laid out or hinted. 1 row over 1500 keys: 7 us, a chain of five dependent
// loads (offsets, page, keys, values, join) on 8 x 12 workgroups. A workgroup alone on
// its CU reads 60 GB/s, which is why short caches too are split.
//
// (Two waves a SIMD are asked for where they fit, since the second sweep, which hardly a
// call makes, else takes registers enough to leave one: 64 single tokens over 3001 keys
// in fp16 157 us in place of 145.)
template <typename T, int D, bool BLOCKS, int kWaves>
__global__ void __launch_bounds__(64 * kWaves, D <= 128 ? 2 : 1) k_attention_few(AttentionArgs a) {
  using S = Shape<T, D>;
  constexpr int VE = S::VE, KB = S::KB, KEYS = S::KEYS, KC = S::KC, CE = S::CE, CW = S::CW,
                NC = S::NC, VR = S::VR;
  constexpr bool HALF = sizeof(T) == 2;
  __shared__ float sum_o[kWaves][16][D];
  __shared__ float sum_m[kWaves][16], sum_l[kWaves][16];

  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int64_t tile;
  int hk, split;
  Tile t;
  if (!find_work(a, &tile, &split, &hk) || !find_tile(a, tile, 16, &t)) return;
  const int per = split_blocks(t.keys, KEYS, a.plan.splits, kFewLeast);
  const int blocks = (t.keys + KEYS - 1) / KEYS;
  const int used = max(1, (blocks + per - 1) / per);
  if (split >= used) return;
  const int block0 = split * per, block1 = min(blocks, block0 + per);
  const int dim = (int)a.c.dim;

  // this lane's row, its queries and the keys it sees
  const int r = t.row0 + min(m, t.rows - 1);
  const int token = r / a.group, head = hk * a.group + r % a.group;
  const int64_t row = (t.first + token) * a.heads + head;
  const int lim = m < t.rows ? seen_keys(a, t, r) : 0;
  const int all_see = seen_keys(a, t, t.row0);   // keys that every row sees
  u32x4 qf[KC];
  {
    const T* q = static_cast<const T*>(a.q) + (t.first + token) * a.qs.outer + head * a.qs.head;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      const int at = (4 * c + g) * VE;
      qf[c] = u32x4{};
      if (at < dim)
        qf[c] = __builtin_bit_cast(u32x4, *reinterpret_cast<const Loose<T, VE>*>(q + at));
    }
  }

  const T* kbase = static_cast<const T*>(a.c.k) + hk * a.c.k_stride[1];
  const T* vbase = static_cast<const T*>(a.c.v) + hk * a.c.v_stride[1];
  const int ks = (int)a.c.k_stride[2], vs = (int)a.c.v_stride[2];

  // Where a step's keys are: page and slot of every 16 of them (or of this lane's one)
  // and how many keys of the split follow from there. The pages' numbers are checked
  // when they have arrived.
  constexpr int RUNS = BLOCKS ? KB : 1;
  struct Place {
    int page[RUNS], slot[RUNS], left[RUNS];
  };
  const int size = (int)a.c.page, end = min(t.length, block1 * KEYS);
  int column[RUNS], slot[RUNS], key[RUNS];   // of the next step to be located
  const int columns_on = kWaves * KEYS / size, slots_on = kWaves * KEYS - columns_on * size;
  auto locate = [&]() {
    Place p;
#pragma unroll
    for (int b = 0; b < RUNS; ++b) {
      const int64_t at = t.s * a.c.table_stride + min(column[b], (int)a.c.columns - 1);
      if constexpr (BLOCKS)
        p.page[b] = reinterpret_cast<const_i32>(reinterpret_cast<uintptr_t>(a.c.table))[at];
      else
        p.page[b] = a.c.table[at];
      p.slot[b] = slot[b];
      p.left[b] = end - key[b];
      key[b] += kWaves * KEYS;
      column[b] += columns_on;
      slot[b] += slots_on;
      if (slot[b] >= size) slot[b] -= size, ++column[b];
    }
    return p;
  };
  // Rows of a run through a buffer as long as they are: what lies behind it, and chunks
  // behind the width, are read as zeros. Other keys are read one by one, zeros for them
  // from a place of their own; no load hangs on a branch.
  const int bytes = (int)sizeof(T);
  int ko[BLOCKS ? KC : 1], vo[BLOCKS ? 4 : 1][NC];
  if constexpr (BLOCKS) {
#pragma unroll
    for (int c = 0; c < KC; ++c)
      ko[c] = (4 * c + g) * VE < dim ? (m * ks + (4 * c + g) * VE) * bytes : INT_MIN;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int part = 0; part < NC; ++part) {
        const int d = 16 * CE * part + CE * m;
        vo[i][part] = d < dim ? ((4 * g + i) * vs + d) * bytes : INT_MIN;
      }
  }
  auto run = [&](const T* base, int64_t page_stride, int stride, const Place& p, int b) {
    const bool ok = p.page[b] >= 0 && p.page[b] < a.c.pages && p.left[b] > 0;
    const T* at = base + (int64_t)(ok ? p.page[b] : 0) * page_stride + (int64_t)p.slot[b] * stride;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(at), (short)0,
                                             ok ? min(p.left[b], 16) * stride * bytes : 0,
                                             kBufferWord3);
  };
  auto one = [&](const T* base, int64_t page_stride, int stride, const Place& p, int from) {
    const int page = __shfl(p.left[0] > 0 ? p.page[0] : -1, from), at = __shfl(p.slot[0], from);
    return page >= 0 && page < a.c.pages ? base + page * page_stride + (int64_t)at * stride
                                         : nullptr;
  };
  const T* nothing = reinterpret_cast<const T*>(kNothing);
  u32x4 kf[KB][KC];
  auto load_keys = [&](const Place& p) {
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      if constexpr (BLOCKS) {
        const auto r = run(kbase, a.c.k_stride[0], ks, p, b);
#pragma unroll
        for (int c = 0; c < KC; ++c)
          kf[b][c] = __builtin_amdgcn_raw_buffer_load_b128(r, ko[c], 0, 0);
      } else {
        const T* k = one(kbase, a.c.k_stride[0], ks, p, 16 * b + m);
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const int at = (4 * c + g) * VE;
          kf[b][c] = load_global<u32x4>(k && at < dim ? k + at : nothing);
        }
      }
    }
  };
  typedef uint32_t vword __attribute__((ext_vector_type(CW)));
  vword vf[VR][NC];
  auto load_values = [&](const Place& p) {
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      if constexpr (BLOCKS) {
        const auto r = run(vbase, a.c.v_stride[0], vs, p, b);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int part = 0; part < NC; ++part) {
            if constexpr (CW == 4)
              vf[4 * b + i][part] = __builtin_amdgcn_raw_buffer_load_b128(r, vo[i][part], 0, 0);
            else
              vf[4 * b + i][part] = __builtin_amdgcn_raw_buffer_load_b64(r, vo[i][part], 0, 0);
          }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const T* v = one(vbase, a.c.v_stride[0], vs, p, 16 * b + 4 * g + i);
#pragma unroll
          for (int part = 0; part < NC; ++part) {
            const int at = 16 * CE * part + CE * m;
            vf[4 * b + i][part] = load_global<vword>(v && at < dim ? v + at : nothing);
          }
        }
      }
    }
  };

  f32x4 o[NC * CE];
  float top, l;
  bool met = false;   // whether this lane's row sees any of the lane's keys
  const float lift_again = lowered<T>(few_lift<T>, 0, t.keys);

  // O^T += V^T p for the step's values: `hi` and `lo` are the 16-bit parts of p, in fp32
  // p itself. WILD: values that are not finite are left out of that, and enter as
  // codes times whether the row sees the key, `see` (as a vector of T, or fp32), where a
  // key of score minus infinity makes any of them a NaN.
  uint32_t picks[2] = {0x05040100u, 0x07060302u};   // the even, the odd values of two words
  auto add_values = [&](auto with_wild, u32x4 hi, u32x4 lo, u32x4 see, f32x4 p) {
    constexpr bool WILD = decltype(with_wild)::value;
#pragma unroll
    for (int part = 0; part < NC; ++part)
#pragma unroll
      for (int e = 0; e < CE; ++e) {
        f32x4& acc = o[part * CE + e];
        u32x4 v;
        if constexpr (HALF) {
#pragma unroll
          for (int u = 0; u < 4; ++u)
            v[u] = __builtin_amdgcn_perm(vf[2 * u + 1][part][e / 2], vf[2 * u][part][e / 2],
                                         picks[e & 1]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = vf[i][part][e];
        }
        if constexpr (WILD) {
          u32x4 code;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const u32x2 taken = take_wild<T>(v[u]);
            v[u] = taken[0], code[u] = taken[1];
          }
          f32x4 sum{};
          if constexpr (HALF) {
            sum = Mfma16<T>::mul(code, see, sum);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              sum = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(code[i]),
                                                         __uint_as_float(see[i]), sum, 0, 0, 0);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[i] += decode_wild(sum[i]);
        }
        if constexpr (HALF) {
          acc = Mfma16<T>::mul(v, hi, acc);
          acc = Mfma16<T>::mul(v, lo, acc);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i]), p[i], acc, 0, 0, 0);
        }
      }
  };

  auto sweep = [&](auto with_wild) {
    const float lift = decltype(with_wild)::value ? lift_again : few_lift<T>;
#pragma unroll
    for (int e = 0; e < NC * CE; ++e) o[e] = f32x4{};
    top = -INFINITY, l = 0.0f;
    int block = block0 + wave;
#pragma unroll
    for (int b = 0; b < RUNS; ++b) {
      key[b] = block * KEYS + (BLOCKS ? 16 * b : lane & (KEYS - 1));
      column[b] = (int)((uint32_t)key[b] / (uint32_t)size);
      slot[b] = key[b] - column[b] * size;
    }
    // (pages are looked up before the loads of a step: loads return in order)
    Place now = locate(), next = locate();
    load_keys(now), load_values(now);
    for (; block < block1; block += kWaves) {
      const int j0 = block * KEYS;
      f32x4 s[KB];
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        s[b] = f32x4{};
#pragma unroll
        for (int c = 0; c < KC; ++c) s[b] = Mfma16<T>::mul(kf[b][c], qf[c], s[b]);
      }
      // holes, by key of this lane (bit 4b + i), or none
      bool whole = true;
      uint32_t there = 0xFFu;
      if constexpr (BLOCKS) {
#pragma unroll
        for (int b = 0; b < KB; ++b)
          if (now.page[b] < 0 || now.page[b] >= a.c.pages)
            there &= ~(0xFu << (4 * b)), whole = false;
      } else {
        const uint64_t ok = __ballot(now.page[0] >= 0 && now.page[0] < a.c.pages);
        whole = ok == ~(uint64_t)0;
        there = (uint32_t)(ok >> (4 * g)) & 0xFu;
        if constexpr (KB == 2) there |= ((uint32_t)(ok >> (16 + 4 * g)) & 0xFu) << 4;
      }
      const Place after = locate();
      load_keys(next);

      const bool masked = !whole || j0 + KEYS > all_see;
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[b][i] *= a.scale2;
      if (masked) {
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * b + i >= lim - j0 - 4 * g || !(there >> (4 * b + i) & 1))
              s[b][i] = -INFINITY;
            else
              met = true;
      } else {
        met = true;
      }
      if (a.plan.pitch && m < t.rows) {
#pragma unroll
        for (int b = 0; b < KB; ++b)
          *reinterpret_cast<f32x4*>(a.scores + row * a.plan.pitch + j0 + 16 * b + 4 * g) = s[b];
      }
      float high = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
      if constexpr (KB == 2)
        high = fmaxf(high, fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
      high = max_across_32(max_across_16(high));
      if (__any(high > top)) {
        const float grown = fmaxf(top, high);
        const float old = __builtin_amdgcn_exp2f(top - (grown == -INFINITY ? 0.0f : grown));
        top = grown;
        l *= old;
#pragma unroll
        for (int e = 0; e < NC * CE; ++e) o[e] *= old;
      }
      const float base = top == -INFINITY ? 0.0f : top - lift;
      f32x4 p[KB];
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[b][i] = __builtin_amdgcn_exp2f(s[b][i] - base);
          l += p[b][i];
        }
      // fp16: the least p that is not 0, as bits less one, tells whether any is faint
      const float faint = __builtin_ldexpf(1.0f, kFewFaint);
      bool far = false;
      if constexpr (kShort<T>) {
        uint32_t least = ~0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) least = min(least, __float_as_uint(p[i / 4][i % 4]) - 1);
        far = __any(least < __float_as_uint(faint) - 1);
      }
      const bool parted = far;   // the faint ones go first, then the others
#pragma unroll 1
      do {
        if constexpr (kShort<T>)   // (or all of the transposed values are kept over the loop)
          asm volatile("" : "+s"(picks[0]), "+s"(picks[1]));
        u32x4 hi{}, lo{}, see{};
        if constexpr (HALF) {
          typedef T t8 __attribute__((ext_vector_type(8)));
          t8 h, d;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float x = p[i / 4][i % 4];
            if (kShort<T> && parted)
              x = (x < faint) != far ? 0.0f
                  : far              ? __builtin_amdgcn_exp2f(s[i / 4][i % 4] - base + kFewFar)
                                     : x;
            h[i] = (T)x;
            d[i] = (T)(x - (float)h[i]);
          }
          hi = __builtin_bit_cast(u32x4, h);
          lo = __builtin_bit_cast(u32x4, d);
        }
        if constexpr (decltype(with_wild)::value) {
          auto seen = [&](int b, int i) {
            const bool sees =
                !masked || (16 * b + i < lim - j0 - 4 * g && (there >> (4 * b + i) & 1));
            return far || !sees ? 0.0f : s[b][i] == -INFINITY ? kCodeNan : 1.0f;
          };
          if constexpr (HALF) {
            typedef T t8 __attribute__((ext_vector_type(8)));
            t8 h;
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = (T)seen(i / 4, i % 4);
            see = __builtin_bit_cast(u32x4, h);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) see[i] = __float_as_uint(seen(0, i));
          }
        }
        if (far)
#pragma unroll
          for (int e = 0; e < NC * CE; ++e) o[e] *= __builtin_ldexpf(1.0f, kFewFar);
        add_values(with_wild, hi, lo, see, p[0]);
        if (!far) break;
#pragma unroll
        for (int e = 0; e < NC * CE; ++e) o[e] *= __builtin_ldexpf(1.0f, -kFewFar);
        far = false;
      } while (kShort<T>);
      load_values(next);
      now = next;
      next = after;
    }
    top -= lift;   // as the sums are lifted
  };
  // A value that is not finite makes its product with any probability so, zeros of rows
  // that do not see it among them: then the wave's keys are gone over once more, with
  // such values apart (and where sums of finite ones come near their end).
  sweep(std::false_type{});
  bool safe = true;
#pragma unroll
  for (int e = 0; e < NC * CE; ++e)
#pragma unroll
    for (int i = 0; i < 4; ++i) safe &= fabsf(o[e][i]) < kSafeSum;
  if (__any(!safe)) sweep(std::true_type{});

  // join the waves' sums
  // no softmax, unless other waves or splits have one
  if (met && top == -INFINITY && l == 0.0f) l = -1.0f;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (g == 0) sum_m[wave][m] = top, sum_l[wave][m] = l;
  __syncthreads();
  float most = sum_m[0][m];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) most = fmaxf(most, sum_m[w][m]);
  const float base = most == -INFINITY ? 0.0f : most;
  const float mine = __builtin_amdgcn_exp2f(top - base);
  if (m < t.rows) {
#pragma unroll
    for (int part = 0; part < NC; ++part)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < CE; ++e)
          sum_o[wave][m][16 * CE * part + CE * (4 * g + i) + e] = o[part * CE + e][i] * mine;
  }
  __syncthreads();
  const bool last = used == 1;
  const int64_t rows = a.tokens * a.heads;
  for (int x = threadIdx.x; x < t.rows * (D / 4); x += 64 * kWaves) {
    const int y = x / (D / 4), d = x % (D / 4) * 4;
    if (d >= dim) continue;
    f32x4 v = *reinterpret_cast<const f32x4*>(&sum_o[0][y][d]);
    float high = sum_m[0][y];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
      v += *reinterpret_cast<const f32x4*>(&sum_o[w][y][d]);
      high = fmaxf(high, sum_m[w][y]);
    }
    float total = 0.0f;
    bool any = false;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      total +=
          sum_l[w][y] * __builtin_amdgcn_exp2f(sum_m[w][y] - (high == -INFINITY ? 0.0f : high));
      any |= sum_l[w][y] < 0.0f;
    }
    if (total == 0.0f && any) total = last ? __builtin_nanf("") : -1.0f;
    const int tok = (t.row0 + y) / a.group, h = hk * a.group + (t.row0 + y) % a.group;
    const int64_t at = (t.first + tok) * a.heads + h;
    if (last) {
      const float inv = total == 0.0f ? 0.0f : 1.0f / total;
      T* out = static_cast<T*>(a.out) + (t.first + tok) * a.os.outer + h * a.os.head + d;
      Loose<T, 4> w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w.v[i] = (T)(total == 0.0f ? 0.0f : v[i] * inv);
      *reinterpret_cast<Loose<T, 4>*>(out) = w;
      if (a.lse && d == 0) a.lse[at] = total == 0.0f ? INFINITY : high + __builtin_amdgcn_logf(total);
    } else {
      *reinterpret_cast<f32x4*>(a.part + (split * rows + at) * dim + d) = v;
      if (d == 0) a.part_ml[split * rows + at] = float2{high, total};
    }
  }
}

template <typename T, int D>
hipError_t launch_width(const AttentionArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)work_groups(a));
  const bool blocks = a.c.page % 16 == 0;
  if constexpr (D <= 128) {   // (eight waves have too few registers for more)
    if (a.plan.wide) {
      if (blocks)
        k_attention_few<T, D, true, 8><<<grid, 512, 0, stream>>>(a);
      else
        k_attention_few<T, D, false, 8><<<grid, 512, 0, stream>>>(a);
      return hipGetLastError();
    }
  }
  if (blocks)
    k_attention_few<T, D, true, 4><<<grid, 256, 0, stream>>>(a);
  else
    k_attention_few<T, D, false, 4><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const AttentionArgs& a, hipStream_t stream) {
  if (a.c.dim <= 64) return launch_width<T, 64>(a, stream);
  // (in 16 bits narrower parts would take more loads than the padding costs)
  if constexpr (sizeof(T) == 4)
    if (a.c.dim <= 96) return launch_width<T, 96>(a, stream);
  if (a.c.dim <= 128) return launch_width<T, 128>(a, stream);
  return launch_width<T, 256>(a, stream);
}

}  // namespace

hipError_t launch_attention_few(const AttentionArgs& a, hipStream_t stream) {
  if (a.c.dtype == LSSVM_BF16) return launch_type<bf16_t>(a, stream);
  if (a.c.dtype == LSSVM_F16) return launch_type<f16_t>(a, stream);
  return launch_type<float>(a, stream);
}

}  // namespace lssvm
