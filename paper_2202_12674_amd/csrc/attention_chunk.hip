// Attention of chunks of new tokens over a paged cache (include/lssvm_cache.h), and the
// weights that its rows give to the keys.
#include "attention.h"

namespace lssvm {
namespace {

constexpr int kWaves = 4;

typedef __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* l16x4_t;

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

// Kinds of values, and the values of a word that are of one: finite ones as they are,
// others as 1.
enum class Kind { finite, plus, minus, nan };
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
    if (k != kind)
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
};

// Where a chunk of a row stands in LDS. Reads of keys go down 32 rows at one chunk,
// and 8 rows in a row are spread over the banks. Reads of values take 32 bytes of four
// rows at a time, which are kept on different banks.
LSSVM_DEV int key_place(int row, int chunk) { return chunk ^ (row & 7); }
LSSVM_DEV int value_place(int row, int chunk) { return chunk ^ (2 * (row & 3)); }

// One tile of 128 RB rows against one split of its keys. A step's keys and values go
// from memory into LDS past the registers, one step ahead, and every wave takes 32 RB
// rows over them: scores S^T = K Q^T, so that a row's scores are a lane's (and the
// lane's 32 away); the running maximum and sum; and O^T += V^T P^T, whose operand P^T
// the scores already are, register for register, if V^T's keys are taken in the same
// order. V^T comes out of LDS by transposing reads, in fp32 by plain ones.
// 16-bit types: p is rounded to the stored type for the product, half a step of it,
// as the values themselves were; its sum is taken before that.
template <typename T, int D, int RB>
__global__ void __launch_bounds__(64 * kWaves, D * RB > 128 ? 1 : 2)
    k_attention_chunk(AttentionArgs a) {
  using S = Chunk<T, D>;
  constexpr int VE = S::VE, KEYS = S::KEYS, NB = S::NB, ROW = S::ROW, CH = S::CH, KC = S::KC,
                DB = S::DB, LOADS = S::LOADS;
  constexpr bool HALF = sizeof(T) == 2;
  __shared__ __attribute__((aligned(16))) char kt[2][KEYS * ROW];
  __shared__ __attribute__((aligned(16))) char vt[2][KEYS * ROW];
  __shared__ int64_t key_at[4][KEYS], value_at[4][KEYS];   // rows of a step, -1: none
  __shared__ uint64_t there[4];

  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // workgroups of one XCD take neighbouring tiles, which read the same keys
  const int64_t count = a.plan.tiles * a.plan.splits * a.c.heads, each = (count + 7) / 8;
  const int64_t work = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  if (work >= count) return;
  const int64_t pair = work / a.plan.tiles;
  const int hk = (int)(pair / a.plan.splits), split = (int)(pair % a.plan.splits);
  Tile t;
  if (!find_tile(a, work % a.plan.tiles, 32 * kWaves * RB, &t)) return;
  const int per = split_blocks(t.keys, KEYS, a.plan.splits, kChunkLeast);
  const int blocks = (t.keys + KEYS - 1) / KEYS;
  const int used = max(1, (blocks + per - 1) / per);
  if (split >= used) return;
  const int block0 = split * per, block1 = min(blocks, block0 + per);
  const int dim = (int)a.c.dim, chunks = dim / VE;

  // this lane's rows
  u32x4 qf[RB][KC];
  int lim[RB];
  int all_see = t.length, some_see = 0;   // keys that every (any) row of the wave sees
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int y = wave * 32 * RB + 32 * rb + c, r = t.row0 + min(y, t.rows - 1);
    lim[rb] = y < t.rows ? seen_keys(a, t, r) : 0;
    const int tok = r / a.group, head = hk * a.group + r % a.group;
    const T* q = static_cast<const T*>(a.q) + (t.first + tok) * a.qs.outer + head * a.qs.head;
#pragma unroll
    for (int k = 0; k < KC; ++k)
      qf[rb][k] = 2 * k + h < chunks ? load_loose(q + (2 * k + h) * VE) : u32x4{};
  }
  {
    const int y = wave * 32 * RB;
    if (y < t.rows) {
      all_see = seen_keys(a, t, t.row0 + y);
      some_see = seen_keys(a, t, t.row0 + min(y + 32 * RB, t.rows) - 1);
    }
  }

  const T* kbase = static_cast<const T*>(a.c.k) + hk * a.c.k_stride[1];
  const T* vbase = static_cast<const T*>(a.c.v) + hk * a.c.v_stride[1];

  // a lane's key of a step: looked up and, later, written down for all waves
  auto look_up = [&](int block, int* slot) {
    const int j = block * KEYS + (lane & (KEYS - 1));
    return j < t.length ? cache_page(a.c, t.s, j, slot) : -1;
  };
  auto write_down = [&](int block, int page, int slot) {
    const int at = (block - block0) & 3;
    if (lane < KEYS) {
      key_at[at][lane] = page < 0 ? -1 : page * a.c.k_stride[0] + slot * a.c.k_stride[2];
      value_at[at][lane] = page < 0 ? -1 : page * a.c.v_stride[0] + slot * a.c.v_stride[2];
    }
    const uint64_t ok = __ballot(page >= 0);
    if (lane == 0) there[at] = ok;
  };
  auto load = [&](int block) {
    const int at = (block - block0) & 3, buf = (block - block0) & 1;
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int first = (u * kWaves + wave) * 64;   // wave-uniform
      const int row = (first + lane) / CH, place = (first + lane) % CH;
      const int64_t ka = key_at[at][row], va = value_at[at][row];
      const int kc = key_place(row, place), vc = value_place(row, place);
      if (ka >= 0 && kc < chunks)
        __builtin_amdgcn_global_load_lds((gptr_t)(kbase + ka + kc * VE),
                                         (lptr_t)(&kt[buf][first * 16]), 16, 0, 0);
      else
        *reinterpret_cast<u32x4*>(&kt[buf][(first + lane) * 16]) = u32x4{};
      if (va >= 0 && vc < chunks)
        __builtin_amdgcn_global_load_lds((gptr_t)(vbase + va + vc * VE),
                                         (lptr_t)(&vt[buf][first * 16]), 16, 0, 0);
      else
        *reinterpret_cast<u32x4*>(&vt[buf][(first + lane) * 16]) = u32x4{};
    }
  };

  f32x16 o[RB][DB];
  float top[RB], l[RB];

  // WILD: of the values only those of `kind` count, and those that are not finite as 1,
  // times whether a row sees the key.
  auto sweep = [&](auto with_wild, Kind kind) {
    constexpr bool WILD = decltype(with_wild)::value;
    const bool counts = WILD && kind != Kind::finite;
    __syncthreads();   // the last sweep has ended
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      top[rb] = -INFINITY, l[rb] = 0.0f;
#pragma unroll
      for (int b = 0; b < DB; ++b) o[rb][b] = f32x16{};
    }
    if (wave < 2) {
      int slot = 0;
      const int page = look_up(block0 + wave, &slot);
      write_down(block0 + wave, page, slot);
    }
    __syncthreads();
    if (block0 < block1) load(block0);
    for (int block = block0; block < block1; ++block) {
      const int buf = (block - block0) & 1, j0 = block * KEYS;
      __builtin_amdgcn_s_waitcnt(0x0F70);   // this wave's loads have landed
      __syncthreads();                      // ... and everyone's; the other buffers are free
      const bool mine = (block & (kWaves - 1)) == wave && block + 2 < block1;
      int page = -1, slot = 0;
      if (mine) page = look_up(block + 2, &slot);
      if (block + 1 < block1) load(block + 1);
      if (j0 < some_see) {
        f32x16 s[RB][NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) s[rb][b] = f32x16{};
#pragma unroll
          for (int k = 0; k < KC; ++k) {
            const u32x4 kf = *reinterpret_cast<const u32x4*>(
                &kt[buf][(32 * b + c) * ROW + 16 * key_place(c, 2 * k + h)]);
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) s[rb][b] = mul32<T>(kf, qf[rb][k], s[rb][b]);
          }
        }
        const uint64_t ok = there[(block - block0) & 3];
        constexpr uint64_t every = KEYS == 64 ? ~(uint64_t)0 : (uint64_t(1) << KEYS) - 1;
        const bool masked = (ok & every) != every || j0 + KEYS > all_see;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          if (masked) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int k = 32 * b + result_row(i, h);
                if (j0 + k >= lim[rb] || !(ok >> k & 1)) s[rb][b][i] = -INFINITY;
                else s[rb][b][i] *= a.scale2;
              }
          } else {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
              for (int i = 0; i < 16; ++i) s[rb][b][i] *= a.scale2;
          }
          float high = s[rb][0][0];
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) high = fmaxf(high, s[rb][b][i]);
          high = max_across_32(high);
          if (__any(high > top[rb])) {
            const float grown = fmaxf(top[rb], high);
            const float old =
                __builtin_amdgcn_exp2f(top[rb] - (grown == -INFINITY ? 0.0f : grown));
            top[rb] = grown;
            l[rb] *= old;
#pragma unroll
            for (int b = 0; b < DB; ++b)
              if (!counts) o[rb][b] *= old;
          }
          const float base = top[rb] == -INFINITY ? 0.0f : top[rb];
          float sum = 0.0f;
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              // (a row that sees the key has a finite score or makes NaN here)
              s[rb][b][i] = __builtin_amdgcn_exp2f(s[rb][b][i] - base);
              sum += s[rb][b][i];
            }
          l[rb] += sum;
        }
        if constexpr (HALF) {
          typedef T t8 __attribute__((ext_vector_type(8)));
          const int i = lane & 15, part = lane >> 4 & 1;
#pragma unroll
          for (int step = 0; step < KEYS / 16; ++step) {
            u32x4 p[RB];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
              t8 x;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const int k = 32 * (step / 2) + result_row(8 * (step % 2) + e, h);
                x[e] = (T)s[rb][step / 2][8 * (step % 2) + e];
                if (counts) x[e] = (T)(j0 + k < lim[rb] && (ok >> k & 1) ? 1.0f : 0.0f);
              }
              p[rb] = __builtin_bit_cast(u32x4, x);
            }
#pragma unroll
            for (int b = 0; b < DB; ++b) {
              u32x4 v;
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const int row = 16 * step + 8 * y + 4 * h + i / 4;
                const int at = value_place(i / 4, 4 * b + 2 * part + i % 4 / 2);
                const s16x4 w = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (l16x4_t)(&vt[buf][row * ROW + 16 * at + 8 * (i % 2)]));
                const u32x2 w2 = __builtin_bit_cast(u32x2, w);
                v[2 * y] = w2[0], v[2 * y + 1] = w2[1];
              }
              if constexpr (WILD) {
#pragma unroll
                for (int u = 0; u < 4; ++u) v[u] = only_kind<T>(v[u], kind);
              }
#pragma unroll
              for (int rb = 0; rb < RB; ++rb) o[rb][b] = mul32<T>(v, p[rb], o[rb][b]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int row = result_row(i, h);
            if (counts) {
#pragma unroll
              for (int rb = 0; rb < RB; ++rb)
                s[rb][0][i] = j0 + row < lim[rb] && (ok >> row & 1) ? 1.0f : 0.0f;
            }
#pragma unroll
            for (int b = 0; b < DB; ++b) {
              uint32_t v = *reinterpret_cast<const uint32_t*>(
                  &vt[buf][row * ROW + 16 * value_place(row, 8 * b + c / 4) + 4 * (c % 4)]);
              if constexpr (WILD) v = only_kind<T>(v, kind);
#pragma unroll
              for (int rb = 0; rb < RB; ++rb)
                o[rb][b] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(v), s[rb][0][i],
                                                                o[rb][b], 0, 0, 0);
            }
          }
        }
      }
      if (mine) write_down(block + 2, page, slot);
    }
  };
  // writes the sums, or adds what values of `kind` make of them
  const int64_t rows = a.tokens * a.heads;
  auto write = [&](Kind kind) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int y = wave * 32 * RB + 32 * rb + c;
      const float sum = l[rb] + __shfl_xor(l[rb], 32);
      if (y >= t.rows) continue;
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
          f32x4 v{o[rb][b][i], o[rb][b][i + 1], o[rb][b][i + 2], o[rb][b][i + 3]};
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
          a.part_ml[split * rows + at] = float2{top[rb], sum};
        else if (a.lse)
          a.lse[at] = sum == 0.0f ? INFINITY : top[rb] + __builtin_amdgcn_logf(sum);
      }
    }
  };

  // A value that is not finite makes its product with any probability so, zeros of rows
  // that do not see it among them. Then the keys are gone over again without such
  // values, and once more for each kind of them.
  sweep(std::false_type{}, Kind::finite);
  int wild = 0;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) wild |= !__builtin_isfinite(o[rb][b][i]);
  if (!__syncthreads_or(wild)) {
    write(Kind::finite);
  } else {
#pragma unroll 1
    for (int kind = 0; kind < 4; ++kind) {
      sweep(std::true_type{}, (Kind)kind);
      write((Kind)kind);
    }
  }
}

// weight_out = weight + the probabilities that the rows give to 64 keys, which stay in
// registers: every wave takes every fourth 32 rows, forms the scores anew and sums
// p = 2^(score - lse) per key; the waves' sums are joined in order.
template <typename T, int D>
__global__ void __launch_bounds__(64 * kWaves) k_weights_chunk(AttentionArgs a) {
  using S = Chunk<T, D>;
  constexpr int VE = S::VE, KC = S::KC, NB = 2;
  __shared__ float sums[kWaves][64];
  const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int s = blockIdx.z, hk = blockIdx.y, chunks = (int)a.c.dim / VE;
  Tile t{};
  t.s = s;
  t.length = cache_length(a.c, s);
  sequence_rows(a, s, &t.first, &t.n);
  const int j0 = blockIdx.x * 64, rows = t.n * a.group;
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
  for (; row < rows; row += 32 * kWaves) {
    const int r = min(row + c, rows - 1), tok = r / a.group, head = hk * a.group + r % a.group;
    const int lim = row + c < rows ? seen_keys(a, t, r) : 0;
    const float lse = a.lse[(t.first + tok) * a.heads + head];
    const T* q = static_cast<const T*>(a.q) + (t.first + tok) * a.qs.outer + head * a.qs.head;
    u32x4 qf[KC];
#pragma unroll
    for (int i = 0; i < KC; ++i)
      qf[i] = 2 * i + h < chunks ? load_loose(q + (2 * i + h) * VE) : u32x4{};
    const bool masked = j0 + 64 > seen_keys(a, t, row) || row + 32 > rows;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      f32x16 z{};
#pragma unroll
      for (int i = 0; i < KC; ++i) z = mul32<T>(kf[b][i], qf[i], z);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = __builtin_amdgcn_exp2f(z[i] * a.scale2 - lse);
        sum[b][i] += masked && j0 + 32 * b + result_row(i, h) >= lim ? 0.0f : p;
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
  if (threadIdx.x >= 64 || j >= t.length) return;
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
  const int64_t count = a.plan.tiles * a.plan.splits * a.c.heads;
  const dim3 grid((unsigned)((count + 7) / 8 * 8));
  k_attention_chunk<T, D, kChunkRB><<<grid, 64 * kWaves, 0, stream>>>(a);
  return hipGetLastError();
}
template <typename T, int D>
hipError_t weights_width(const AttentionArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.c.columns * a.c.page + 63) / 64), (unsigned)a.c.heads,
                  (unsigned)a.c.sequences);
  k_weights_chunk<T, D><<<grid, 64 * kWaves, 0, stream>>>(a);
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
