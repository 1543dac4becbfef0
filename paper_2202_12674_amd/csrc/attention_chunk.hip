// Attention of chunks of new tokens over a paged cache (include/lssvm_cache.h), and the
// weights that its rows give to the keys.
#include "attention.h"

namespace lssvm {
namespace {

constexpr int kWaves = 4;
constexpr int kWeightBlocks = 2;   // of 32 keys that a workgroup sums the weights of

typedef __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;

// 32 x 32 products over two 16-byte chunks: lane l has chunk l / 32 of row l % 32 of
// either operand.
template <typename T>
LSSVM_DEV f32x16 mul32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (std::is_same_v<T, bf16_t>) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else if constexpr (std::is_same_v<T, f16_t>) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0,
                                               0, 0);
    return c;
  }
}

// Row (or key) of register i of a 32 x 32 result in lane half h.
LSSVM_DEV constexpr int result_row(int i, int h) { return 8 * (i / 4) + 4 * h + i % 4; }

template <typename T>
LSSVM_DEV u32x4 load_loose(const T* p) {
  return __builtin_bit_cast(u32x4, *reinterpret_cast<const Loose<T, kVec<T>>*>(p));
}

// Keeps a value whole and in its registers here: the compiler else takes the results
// apart between the steps and moves them all back every time.
template <typename V>
LSSVM_DEV void pin(V& v) {
  asm volatile("" : "+v"(v));
}

// use(n, read(n)) and side(n) for n < N, with the reads (of LDS) four ahead, in just
// this order: left alone, the compiler waits for every read. `side` is vector work that
// runs while the matrix cores are busy with `use`.
template <int N, typename R, typename U, typename W>
LSSVM_DEV void read_ahead(R read, U use, W side) {
  constexpr int AHEAD = N < 4 ? N : 4;
  decltype(read(0)) f[AHEAD];
#pragma unroll
  for (int n = 0; n < AHEAD; ++n) f[n] = read(n);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    __builtin_amdgcn_sched_barrier(0);
    use(n, f[n % AHEAD]);
    if (n + AHEAD < N) f[n % AHEAD] = read(n + AHEAD);
    side(n);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// Kinds of values, and the values of a word that are of one: finite ones as they are,
// others as 1. `lost` are all that are not finite, under scores of minus infinity.
enum class Kind { finite, plus, minus, nan, lost };
LSSVM_DEV float wild_value(Kind kind) {
  return kind == Kind::plus ? INFINITY : kind == Kind::minus ? -INFINITY : __builtin_nanf("");
}
template <typename T>
LSSVM_DEV uint32_t only_kind(uint32_t word, Kind kind) {
  typedef T tn __attribute__((ext_vector_type(4 / sizeof(T))));
  tn x = __builtin_bit_cast(tn, word);
#pragma unroll
  for (int i = 0; i < 4 / (int)sizeof(T); ++i) {
    const float v = (float)x[i];
    const Kind k = __builtin_isfinite(v) ? Kind::finite
                   : v != v              ? Kind::nan
                   : v > 0               ? Kind::plus
                                         : Kind::minus;
    if (k != kind && (kind != Kind::lost || k == Kind::finite))
      x[i] = (T)0.0f;
    else if (k != Kind::finite)
      x[i] = (T)1.0f;
  }
  return __builtin_bit_cast(uint32_t, x);
}

constexpr int pow2_from(int v) {
  int p = 1;
  while (p < v) p *= 2;
  return p;
}

template <typename T, int D>
struct Chunk {
  static constexpr int VE = kVec<T>;
  static constexpr int KEYS = chunk_keys<T>;                     // of a step
  static constexpr int NB = KEYS / 32;
  static constexpr int ROW = pow2_from(D * (int)sizeof(T));      // bytes of a row in LDS
  static constexpr int CH = ROW / 16;                            // its 16-byte chunks
  static constexpr int KC = D / (2 * VE);                        // chunks of a row per lane
  static constexpr int DB = D / 32;
  static constexpr int LOADS = KEYS * CH / (64 * kWaves);        // chunks per thread and tile
  // rows that a thread moves are NEXT apart, at one chunk under the swizzle
  static constexpr int NEXT = 64 * kWaves / CH, TURN = NEXT < 8 ? NEXT - 1 : 7;
  // 16-bit values, in columns: every column's keys in 128 bytes
  static constexpr bool HALF = sizeof(T) == 2;
  static constexpr int VBYTES = HALF ? D * 2 * KEYS : KEYS * ROW;
  static constexpr int VUNITS = KEYS / 4 * (D / VE);             // 4 keys x 16 bytes
  static constexpr int VU = (VUNITS + 64 * kWaves - 1) / (64 * kWaves);
};

// Chunks of a row (keys, and fp32 values) stand in LDS at chunk ^ (row & TURN): reads of
// keys go down the rows at one chunk, and 8 rows in a row are spread over the banks.
// 16-bit values in columns: 8 keys of column d, of its 8 times as many, start here. Reads
// go down 32 columns, writes down every eighth.
LSSVM_DEV int column_at(int d, int keys8) { return d * 128 + 16 * (keys8 ^ ((d ^ (d >> 3)) & 7)); }

// One tile of 128 rows against one split of its keys. A step's keys and values go
// from memory into LDS past the registers, one step ahead, and every wave takes 32
// rows over them: scores S^T = K Q^T, so that a row's scores are a lane's (and the
// lane's 32 away); the running maximum and sum; and O^T += V^T P^T, whose operand P^T
// the scores already are, register for register, if V^T's keys are taken in the same
// order. 16-bit values pass through registers on their way to LDS and are transposed
// there once, 4 keys x 8 values per thread, so that a lane reads 8 keys of its column
// in one piece; fp32 ones are read singly and stay in rows.
// 16-bit types: p is rounded to the stored type for the product, half a step of it,
// as the values themselves were; its sum is taken before that. (In two parts, as for few
// rows, the result's error is 1.7e-3 in place of 2.3e-3, and the time of the case below
// 2.08 ms in place of 1.57.) fp16 has too short a range for that: small ones are
// multiplied apart (attention.h).
//
// Measured: bf16, 4 x 2048 rows x 32 heads over 16384 keys, 128 wide: 1.57 to 1.69 ms on
// different cards, 780 to 837 TFLOP/s (a large library product reaches 1107). The matrix
// cores are busy for 36% of it; without loading (the same tile over and over) the form of
// 1.69 ms took 1.33, and there a step of two workgroups is 2.1 us of which the two
// products make 0.75, the exponentials 0.3, and the rest waits in turn: for LDS, the
// maximum, the barrier. Two blocks of 32 rows per wave, half a step apart in one
// instruction stream, took 2.9 ms: the results do not fit the registers that vector
// instructions reach, and moving them costs more than the overlap gives.
template <typename T, int D>
__global__ void __launch_bounds__(64 * kWaves, D > 128 ? 1 : 2)
    k_attention_chunk(AttentionArgs a) {
  using S = Chunk<T, D>;
  constexpr int VE = S::VE, KEYS = S::KEYS, NB = S::NB, ROW = S::ROW, CH = S::CH, KC = S::KC,
                DB = S::DB, LOADS = S::LOADS, VU = S::VU;
  constexpr bool HALF = S::HALF;
  // two buffers, as objects of their own: the compiler holds reads of the one only then
  // apart from loads into the other, and else waits for those before every read
  __shared__ __attribute__((aligned(16))) char kt0[KEYS * ROW], kt1[KEYS * ROW];
  __shared__ __attribute__((aligned(16))) char vt0[S::VBYTES], vt1[S::VBYTES];
  auto kt = [&](auto buf) -> char(&)[KEYS * ROW] {
    if constexpr (buf == 0) return kt0; else return kt1;
  };
  auto vt = [&](auto buf) -> char(&)[S::VBYTES] {
    if constexpr (buf == 0) return vt0; else return vt1;
  };
  constexpr std::integral_constant<int, 0> even{};
  constexpr std::integral_constant<int, 1> odd{};
  __shared__ int64_t key_at[4][KEYS], value_at[4][KEYS];   // rows of a step, -1: none
  __shared__ uint64_t there[4];

  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  int64_t tile;
  int hk, split;
  Tile t;
  if (!find_work(a, &tile, &split, &hk) || !find_tile(a, tile, 32 * kWaves, &t)) return;
  const int per = split_blocks(t.keys, KEYS, a.plan.splits, kChunkLeast);
  const int blocks = (t.keys + KEYS - 1) / KEYS;
  const int used = max(1, (blocks + per - 1) / per);
  if (split >= used) return;
  const int block0 = split * per, block1 = min(blocks, block0 + per);
  const int dim = (int)a.c.dim, chunks = dim / VE;

  // this lane's rows. Queries carry the sign of the scale (none if it is 0), so that
  // the largest score is the largest product.
  const float scale2 = a.scale2 == 0.0f ? 1.0f : fabsf(a.scale2);
  const uint32_t sign = a.scale2 < 0.0f ? (HALF ? 0x80008000u : 0x80000000u) : 0;
  const uint32_t keep = a.scale2 == 0.0f ? 0 : ~0u;
  auto turned = [&](u32x4 q) { return (q ^ sign) & keep; };
  u32x4 qf[KC];
  int lim;
  int all_see = t.length, some_see = 0;   // keys that every (any) row of the wave sees
  const int y = wave * 32 + c, r = t.row0 + min(y, t.rows - 1);
  lim = y < t.rows ? seen_keys(a, t, r) : 0;
  const int tok = r / a.group, head = hk * a.group + r % a.group;
  const T* q = static_cast<const T*>(a.q) + (t.first + tok) * a.qs.outer + head * a.qs.head;
#pragma unroll
  for (int k = 0; k < KC; ++k)
    qf[k] = 2 * k + h < chunks ? turned(load_loose(q + (2 * k + h) * VE)) : u32x4{};
  {
    const int y = wave * 32;
    if (y < t.rows) {
      all_see = seen_keys(a, t, t.row0 + y);
      some_see = seen_keys(a, t, t.row0 + min(y + 32, t.rows) - 1);
    }
  }

  const T* kbase = static_cast<const T*>(a.c.k) + hk * a.c.k_stride[1];
  const T* vbase = static_cast<const T*>(a.c.v) + hk * a.c.v_stride[1];

  constexpr uint64_t every = ~(uint64_t)0 >> (64 - KEYS);

  // a lane's key of a step: its page is looked up and, later, checked and written down
  // for all waves
  auto look_up = [&](int block) {
    const int j = min(block * KEYS + (lane & (KEYS - 1)), t.length - 1);
    return a.c.table[t.s * a.c.table_stride + (uint32_t)j / (uint32_t)a.c.page];
  };
  auto write_down = [&](int block, int page) {
    const int at = (block - block0) & 3, j = block * KEYS + (lane & (KEYS - 1));
    const int slot = (int)((uint32_t)j % (uint32_t)a.c.page);
    const bool ok = j < t.length && page >= 0 && page < a.c.pages;
    if (lane < KEYS) {
      key_at[at][lane] = ok ? page * a.c.k_stride[0] + slot * a.c.k_stride[2] : -1;
      value_at[at][lane] = ok ? page * a.c.v_stride[0] + slot * a.c.v_stride[2] : -1;
    }
    const uint64_t all = __ballot(ok);
    if (lane == 0) there[at] = all;
  };
  // Keys that are not there and chunks behind the width are loaded as zeros from a place
  // of their own: a load behind a branch would be waited for at its end.
  const T* nothing = reinterpret_cast<const T*>(kNothing);
  // 16-bit values on their way: unit x of a step is chunk x % (D / 8) of the 4 keys from
  // 4 (x / (D / 8))
  u32x4 vr[HALF ? VU : 1][4];
  auto load = [&](int block, auto buf) {
    const int at = (block - block0) & 3;
    const int row = threadIdx.x / CH, place = threadIdx.x % CH;   // and 256 / CH rows on
    const int kc = place ^ (row & S::TURN);
    if constexpr (HALF) {
#pragma unroll
      for (int u = 0; u < VU; ++u) {
        const int x = u * 64 * kWaves + (int)threadIdx.x, ch = x % (D / VE), kg = x / (D / VE);
        int64_t from[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) from[i] = value_at[at][(4 * kg + i) & (KEYS - 1)];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          vr[u][i] = load_global<u32x4>(
              from[i] >= 0 && ch < chunks ? vbase + from[i] + ch * VE : nothing);
      }
    }
    int64_t from[LOADS];
#pragma unroll
    for (int u = 0; u < LOADS; ++u) from[u] = key_at[at][row + u * S::NEXT];
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const T* k = from[u] >= 0 && kc < chunks ? kbase + from[u] + kc * VE : nothing;
      __builtin_amdgcn_global_load_lds((gptr_t)k, (lptr_t)(&kt(buf)[(u * kWaves + wave) * 1024]),
                                       16, 0, 0);
    }
    if constexpr (!HALF) {
#pragma unroll
      for (int u = 0; u < LOADS; ++u) from[u] = value_at[at][row + u * S::NEXT];
#pragma unroll
      for (int u = 0; u < LOADS; ++u) {
        const T* v = from[u] >= 0 && kc < chunks ? vbase + from[u] + kc * VE : nothing;
        __builtin_amdgcn_global_load_lds(
            (gptr_t)v, (lptr_t)(&vt(buf)[(u * kWaves + wave) * 1024]), 16, 0, 0);
      }
    }
  };
  auto store_values = [&](auto buf) {
#pragma unroll
    for (int u = 0; u < VU; ++u) {
      const int x = u * 64 * kWaves + (int)threadIdx.x, ch = x % (D / VE), kg = x / (D / VE);
      if (x >= S::VUNITS) continue;
      // keys 16 t + 8 y + 4 h .. + 3 stand behind each other for y = 0, 1
      const int keys8 = 2 * (kg / 4) + kg % 2, y = kg / 2 % 2;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t pick = e & 1 ? 0x07060302u : 0x05040100u;
        const u32x2 w{__builtin_amdgcn_perm(vr[u][1][e / 2], vr[u][0][e / 2], pick),
                      __builtin_amdgcn_perm(vr[u][3][e / 2], vr[u][2][e / 2], pick)};
        *reinterpret_cast<u32x2*>(&vt(buf)[column_at(8 * ch + e, keys8) + 8 * y]) = w;
      }
    }
  };

  f32x16 o[DB];
  float top, l;

  // Lane offsets of the 8 chunks (key and value) of a step, whose other parts are constant:
  // chunk 2x + h under the swizzle is 2x ^ (h ^ swizzle).
  int ko[4], vo[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    ko[x] = c * ROW + 16 * ((2 * x + h) ^ (c & S::TURN));
    vo[x] = column_at(c, 2 * x + h);
  }

  // One pass over the keys. Pass 0 is the only one unless values are not finite; the
  // others count only the values of one kind (below).
  f32x16 s[NB];
  float base, lift;
  bool met = false;     // whether this lane's row sees any of the lane's keys
  bool taken = false;   // whether the pass without values that are not finite met any
  auto sweep = [&](int pass) {
    const Kind kind = (Kind)(pass - 1);
    lift = pass == 0 ? chunk_lift<T> : lowered<T>(chunk_lift<T>, 8, t.keys);
    const bool counts = pass > 1;
    // scores: products of keys and queries, one block of 32 keys after the other
    auto read_key = [&](auto buf, int n) {
      const int b = n / KC, k = n % KC;
      return *reinterpret_cast<const u32x4*>(&kt(buf)[ko[k % 4] + 32 * b * ROW + 128 * (k / 4)]);
    };
    auto score = [&](int n, u32x4 kf) {
      const int b = n / KC, k = n % KC;
      s[b] = mul32<T>(kf, qf[k], k == 0 ? f32x16{} : s[b]);
    };
    // four maxima of block b's scores
    float highs[4];
    auto look_at = [&](int b) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        highs[i % 4] = b == 0 && i < 4 ? s[b][i] : fmaxf(highs[i % 4], s[b][i]);
    };
    // masks the scores, brings the maximum and what hangs on it up to date. The maximum
    // may stay up to 2^8 behind: p is then that much larger than 1.
    float low;   // fp16: the least score that is seen
    auto settle = [&](int block) {
      const int j0 = block * KEYS;
      low = INFINITY;
      const uint64_t ok = there[(block - block0) & 3];
      const uint64_t ok_h = ok >> (4 * h);   // of key k + 4 h
      const int left = lim - j0 - 4 * h;
      if (counts || (ok & every) != every || j0 + KEYS > all_see) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int k = 32 * b + result_row(i, 0);
            const bool sees = k < left && (ok_h >> k & 1);
            if (counts)   // p = 1
              s[b][i] = kind != Kind::lost || s[b][i] == -INFINITY ? 0.0f : -INFINITY;
            if constexpr (kShort<T>) low = sees ? fminf(low, s[b][i]) : low;
            if (!sees) s[b][i] = -INFINITY;
            met |= sees;
          }
          look_at(b);
        }
      } else {
        met = true;
        look_at(NB - 1);
        if constexpr (kShort<T>)
#pragma unroll
          for (int i = 0; i < 16 * NB; ++i) low = fminf(low, s[i / 16][i % 16]);
      }
      const float high =
          max_across_32(fmaxf(fmaxf(highs[0], highs[1]), fmaxf(highs[2], highs[3])));
      if (!counts && __any((high - top) * scale2 > 8.0f)) {
        const float grown = fmaxf(top, high);
        const float old =
            __builtin_amdgcn_exp2f((top - (grown == -INFINITY ? 0.0f : grown)) * scale2);
        top = grown;
        l *= old;
#pragma unroll
        for (int b = 0; b < DB; ++b) {
          o[b] *= old;
          pin(o[b]);
        }
      }
      base = counts || top == -INFINITY ? 0.0f : lift - top * scale2;
    };
    auto power = [&](int i) {   // p of score i
      return __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 16][i % 16], scale2, base));
    };
    // 16-bit types: p in pairs, as the second product takes them
    uint32_t pairs[HALF ? 8 * NB : 1];
    auto make_pairs = [&](int from, int to) {
      if constexpr (HALF) {
        typedef T t2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int x = from; x < to; ++x) {
          const float p = power(2 * x), q = power(2 * x + 1);
          l += p + q;
          pin(l);
          pairs[x] = __builtin_bit_cast(uint32_t, t2{(T)p, (T)q});
          pin(pairs[x]);
        }
      }
    };
    auto read_column = [&](auto buf, int n) {
      // (columns 32 apart differ in bit 2 of the swizzle)
      const int step = n / DB, b = n % DB;
      return *reinterpret_cast<const u32x4*>(&vt(buf)[vo[step ^ (2 * (b & 1))] + 32 * 128 * b]);
    };
    auto add = [&](int n, u32x4 v) {
      const int step = n / DB, b = n % DB;
      const u32x4 p{pairs[4 * step], pairs[4 * step + 1], pairs[4 * step + 2],
                    pairs[4 * step + 3]};
      o[b] = mul32<T>(v, p, o[b]);
    };
    // fp16: the step's probabilities below 2^kChunkFaint, and none of them after that
    auto add_faint = [&](auto buf) {
      if constexpr (kShort<T>) {
        typedef T t2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int b = 0; b < DB; ++b) o[b] *= __builtin_ldexpf(1.0f, kChunkFar);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          uint32_t far[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            t2 w;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float power = __builtin_fmaf(s[n][2 * x + e], scale2, base);
              const bool faint = power < (float)kChunkFaint;
              const float p = faint ? __builtin_amdgcn_exp2f(power + kChunkFar) : 0.0f;
              l += p * __builtin_ldexpf(1.0f, -kChunkFar);
              w[e] = (T)p;
              if (faint) s[n][2 * x + e] = -INFINITY;
            }
            far[x] = __builtin_bit_cast(uint32_t, w);
          }
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int b = 0; b < DB; ++b)
              o[b] = mul32<T>(read_column(buf, (2 * n + x) * DB + b),
                              u32x4{far[4 * x], far[4 * x + 1], far[4 * x + 2], far[4 * x + 3]},
                              o[b]);
        }
#pragma unroll
        for (int b = 0; b < DB; ++b) {
          o[b] *= __builtin_ldexpf(1.0f, -kChunkFar);
          pin(o[b]);
        }
      }
    };
    auto only = [&](auto buf) {   // values in place, since only this step reads them
      for (int x = (int)threadIdx.x * 4; x < S::VBYTES; x += 256 * kWaves) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&vt(buf)[x]);
        const uint32_t was = *w, is = only_kind<T>(was, kind);
        taken |= kind == Kind::finite && is != was;
        *w = is;
      }
      __syncthreads();
    };
    constexpr int SCORES = KC * NB, SUMS = HALF ? KEYS / 16 * DB : 0;

    __syncthreads();   // the last pass has ended
    top = -INFINITY, l = 0.0f;
#pragma unroll
    for (int b = 0; b < DB; ++b) o[b] = f32x16{};
    if (block0 >= block1) return;
    if (wave < 2) write_down(block0 + wave, look_up(block0 + wave));
    __syncthreads();
    load(block0, even);
    if constexpr (HALF) store_values(even);

    auto step = [&](int block, auto buf, auto other) {
      __builtin_amdgcn_s_waitcnt(0x0F70);
      __syncthreads();
      const bool mine = (block & (kWaves - 1)) == wave && block + 2 < block1;
      const int page = look_up(block + 2);   // (by all: it is not waited for here)
      if (block + 1 < block1) load(block + 1, other);
#pragma unroll
      for (int b = 0; b < DB; ++b) pin(o[b]);
      if (pass > 0) only(buf);
      if (block * KEYS < some_see) {
        // the first block's maximum while the second's scores are formed
        read_ahead<SCORES>([&](int n) { return read_key(buf, n); },
                           [&](int n, u32x4 kf) { score(n, kf); },
                           [&](int n) {
                             if (NB == 2 && n == KC) look_at(0);
                           });
        settle(block);
        if constexpr (kShort<T>)
          if (!counts && __any(__builtin_fmaf(low, scale2, base) < (float)kChunkFaint))
            add_faint(buf);
        if constexpr (HALF) {
          // the probabilities of 16 keys while those of the 16 before are multiplied
          make_pairs(0, 4);
          read_ahead<SUMS>([&](int n) { return read_column(buf, n); },
                           [&](int n, u32x4 v) { add(n, v); },
                           [&](int n) {
                             const int step = n / DB + 1, b = n % DB;
                             if (step < KEYS / 16)
                               make_pairs(4 * step + 4 * b / DB, 4 * step + 4 * (b + 1) / DB);
                           });
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int row = result_row(i, h);
            const float p = power(i);
            l += p;
#pragma unroll
            for (int b = 0; b < DB; ++b) {
              const float v = *reinterpret_cast<const float*>(
                  &vt(buf)[row * ROW + 16 * ((8 * b + c / 4) ^ (row & S::TURN)) + 4 * (c % 4)]);
              o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, p, o[b], 0, 0, 0);
            }
          }
        }
      }
      if constexpr (HALF)
        if (block + 1 < block1) store_values(other);
      if (mine) write_down(block + 2, page);
    };
    for (int block = block0; block < block1; block += 2) {
      step(block, even, odd);
      if (block + 1 < block1) step(block + 1, odd, even);
    }
  };
  // writes the sums, or adds what values of `kind` make of them
  const int64_t rows = a.tokens * a.heads;
  auto write = [&](Kind kind) {
    const int y = wave * 32 + c;
    // no softmax, unless other splits have one
    if (met && top == -INFINITY && l == 0.0f) l = -1.0f;
    float sum = l + __shfl_xor(l, 32);
    if (y >= t.rows) return;
    if (sum < 0.0f && used == 1) sum = __builtin_nanf("");
    const int r = t.row0 + y, tok = r / a.group, head = hk * a.group + r % a.group;
    const int64_t at = (t.first + tok) * a.heads + head;
    T* out = static_cast<T*>(a.out) + (t.first + tok) * a.os.outer + head * a.os.head;
    float* part = a.part + (split * rows + at) * dim;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int d = 32 * b + result_row(i, h);
        if (d >= dim) continue;
        f32x4 v{o[b][i], o[b][i + 1], o[b][i + 2], o[b][i + 3]};
        if (kind != Kind::finite) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (v[e] == 0.0f) continue;
            if (used == 1)
              out[d + e] = (T)((float)out[d + e] + wild_value(kind));
            else
              part[d + e] += wild_value(kind);
          }
        } else if (used == 1) {
          Loose<T, 4> w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w.v[e] = (T)(sum == 0.0f ? 0.0f : v[e] * inv);
          *reinterpret_cast<Loose<T, 4>*>(out + d) = w;
        } else {
          *reinterpret_cast<f32x4*>(part + d) = v;
        }
      }
    if (kind == Kind::finite && h == 0) {
      if (used > 1)
        a.part_ml[split * rows + at] = float2{top * scale2 - lift, sum};
      else if (a.lse)
        a.lse[at] = sum == 0.0f ? INFINITY
                                : top * scale2 - lift + __builtin_amdgcn_logf(sum);
    }
  };

  // A value that is not finite makes its product with any probability so, zeros of rows
  // that do not see it among them. Then the keys are gone over again without such
  // values, and once more for each kind of them if there were any (there are none where
  // sums of finite ones came near their end).
#pragma unroll 1
  for (int pass = 0; pass < 6; ++pass) {
    sweep(pass);
    if (pass == 0) {
      int wild = 0;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) wild |= !(fabsf(o[b][i]) < kSafeSum);
      if (__syncthreads_or(wild)) continue;
    }
    write(pass == 0 ? Kind::finite : (Kind)(pass - 1));
    if (pass == 0 || (pass == 1 && !__syncthreads_or(taken))) break;
  }
}

// weight_out = weight + the probabilities that the rows give to 64 keys, which stay in
// registers: every wave takes every fourth 32 rows, forms the scores anew and sums
// p = 2^(score - lse) per key; the waves' sums are joined in order. Measured: f16, 6 x
// 700 rows x 14 heads over 3001 keys, 64 wide: 49 us (13.5 GFLOP); bound by reading the
// rows from L2, once for every 64 keys (32 keys: 70 us; rows not read ahead: 68).
template <typename T, int D>
__global__ void __launch_bounds__(256) k_weights_chunk(AttentionArgs a) {
  using S = Chunk<T, D>;
  constexpr int VE = S::VE, KC = S::KC, NB = kWeightBlocks;
  __shared__ float sums[kWaves][32 * NB];
  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int s = blockIdx.z, hk = blockIdx.y, chunks = (int)a.c.dim / VE;
  Tile t{};
  t.s = s;
  t.length = cache_length(a.c, s);
  sequence_rows(a, s, &t.first, &t.n);
  const int j0 = blockIdx.x * 32 * NB, rows = t.n * a.group;
  if (j0 >= t.length) return;

  u32x4 kf[NB][KC];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int j = j0 + 32 * b + c;
    int slot = 0;
    const int page = j < t.length ? cache_page(a.c, s, j, &slot) : -1;
    const T* k = static_cast<const T*>(a.c.k) + max(page, 0) * a.c.k_stride[0] +
                 hk * a.c.k_stride[1] + slot * a.c.k_stride[2];
#pragma unroll
    for (int i = 0; i < KC; ++i)
      kf[b][i] = page >= 0 && 2 * i + h < chunks
                     ? *reinterpret_cast<const u32x4*>(k + (2 * i + h) * VE)
                     : u32x4{};
  }
  float sum[NB][16];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[b][i] = 0.0f;

  // rows before the first that sees key j0 give nothing
  int row = wave * 32;
  if (a.causal) {
    const int first = max(0, j0 - (t.length - t.n)) * a.group / 32 * 32;
    row += first;
  }
  // a step's rows are read while the one before it is worked on
  u32x4 qf[KC], qn[KC];
  float lse, lse_n;
  int lim, lim_n;
  auto read = [&](int from) {
    const int r = min(from + c, rows - 1), tok = r / a.group, head = hk * a.group + r % a.group;
    lim_n = from + c < rows ? seen_keys(a, t, r) : 0;
    lse_n = a.lse[(t.first + tok) * a.heads + head];
    const T* q = static_cast<const T*>(a.q) + (t.first + tok) * a.qs.outer + head * a.qs.head;
#pragma unroll
    for (int i = 0; i < KC; ++i) {   // (keys are zero behind the width)
      const int at = min(2 * i + h, chunks - 1);
      qn[i] = load_loose(q + at * VE);
    }
  };
  if (rows > 0) read(row);
  for (; row < rows; row += 32 * kWaves) {
#pragma unroll
    for (int i = 0; i < KC; ++i) qf[i] = qn[i];
    lse = lse_n, lim = lim_n;
    read(row + 32 * kWaves);
    const bool masked = j0 + 32 * NB > seen_keys(a, t, row) || row + 32 > rows;
    const int left = lim - j0 - 4 * h;   // keys of this lane that its row sees
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      f32x16 z{};
#pragma unroll
      for (int i = 0; i < KC; ++i) z = mul32<T>(kf[b][i], qf[i], z);
      if (masked) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * b + result_row(i, 0) < left)
            sum[b][i] += __builtin_amdgcn_exp2f(z[i] * a.scale2 - lse);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[b][i] += __builtin_amdgcn_exp2f(z[i] * a.scale2 - lse);
      }
    }
  }
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float x = sum[b][i];
      for (int d = 16; d; d >>= 1) x += __shfl_xor(x, d);
      if (c == 0) sums[wave][32 * b + result_row(i, h)] = x;
    }
  __syncthreads();
  const int j = j0 + (int)threadIdx.x;
  if (threadIdx.x >= 32 * NB || j >= t.length) return;
  int slot;
  const int page = cache_page(a.c, s, j, &slot);
  if (page < 0) return;
  float gain = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) gain += sums[w][threadIdx.x];
  const float old = a.c.weight[page * a.c.weight_stride[0] + hk * a.c.weight_stride[1] + slot];
  a.weight_out[page * a.ws.outer + hk * a.ws.head + slot] = old + gain;
}

template <typename T, int D>
hipError_t launch_width(const AttentionArgs& a, hipStream_t stream) {
  k_attention_chunk<T, D><<<dim3((unsigned)work_groups(a)), 64 * kWaves, 0, stream>>>(a);
  return hipGetLastError();
}
template <typename T, int D>
hipError_t weights_width(const AttentionArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.c.columns * a.c.page + 32 * kWeightBlocks - 1) / (32 * kWeightBlocks)), (unsigned)a.c.heads,
                  (unsigned)a.c.sequences);
  k_weights_chunk<T, D><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const AttentionArgs& a, bool weights, hipStream_t stream) {
  if (a.c.dim <= 64)
    return weights ? weights_width<T, 64>(a, stream) : launch_width<T, 64>(a, stream);
  if (a.c.dim <= 96)
    return weights ? weights_width<T, 96>(a, stream) : launch_width<T, 96>(a, stream);
  if (a.c.dim <= 128)
    return weights ? weights_width<T, 128>(a, stream) : launch_width<T, 128>(a, stream);
  return weights ? weights_width<T, 256>(a, stream) : launch_width<T, 256>(a, stream);
}

hipError_t launch_dtype(const AttentionArgs& a, bool weights, hipStream_t stream) {
  if (a.c.dtype == LSSVM_BF16) return launch_type<bf16_t>(a, weights, stream);
  if (a.c.dtype == LSSVM_F16) return launch_type<f16_t>(a, weights, stream);
  return launch_type<float>(a, weights, stream);
}

}  // namespace

hipError_t launch_attention_chunk(const AttentionArgs& a, hipStream_t stream) {
  return launch_dtype(a, false, stream);
}

hipError_t launch_weights_chunk(const AttentionArgs& a, hipStream_t stream) {
  return launch_dtype(a, true, stream);
}

}  // namespace lssvm
