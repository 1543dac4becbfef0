// Attention of new tokens over a paged cache (include/lssvm_cache.h): how a call is
// laid out, the joining of splits and the weights of few rows.
#include "attention.h"

namespace lssvm {

hipError_t launch_attention_few(const AttentionArgs& a, hipStream_t stream);
hipError_t launch_attention_chunk(const AttentionArgs& a, hipStream_t stream);
hipError_t launch_weights_chunk(const AttentionArgs& a, hipStream_t stream);

namespace {

constexpr int64_t kCUs = 256;
constexpr int kMostSplits = 64;
constexpr int64_t kL2Bytes = 4 << 20;      // of an XCD
constexpr int64_t kMostGroups = 1 << 23;   // workgroups of 256 that a grid is kept to
constexpr int64_t kWideKeys = 768;
constexpr int64_t round_up(int64_t v, int64_t m) { return (v + m - 1) / m * m; }

AttentionPlan make_plan(const lssvm_cache& c, int64_t tokens, int heads, bool accumulate) {
  AttentionPlan p{};
  const int64_t group = heads / c.heads, most = c.columns * c.page;
  // Tiles of 16 rows or of 128, by the rows that a sequence has on average: the latter
  // read every key once for all of them, through LDS; the former waste less on few rows.
  // 16-bit types, us of tiles of 16 and of 128: heads of 64 (8 sequences of 2000 keys) 64
  // rows 24, 24, 256 rows 32, 35, 512 rows 46, 40; of 128 (30 of 600) 16 rows 14, 26, 64
  // rows 30, 30, (8 of 4000) 8 rows 31, 27; of 256 (4 of 9000) 4 rows 38, 54, 16 rows 70,
  // 61. In fp32, where the matrix cores take eight times as long, tiles of 16 are better
  // (8 of 2000 x 128: 64 rows 48, 84, 1024 rows 241, 304; 2 of 6000 x 256, 8000 rows 915,
  // 976) until a head's keys and values outgrow an XCD's L2, from which every tile reads
  // them (16000 x 96, 4096 rows: 734, 474; 8192 x 128, 8192 rows: 2262, 2110).
  // (Tiles of 16 of the largest calls would be more than a grid holds: partly empty ones
  // add 2^22 at most to those here.)
  const int64_t rows = tokens * group / c.sequences;
  if (c.dtype == LSSVM_F32)
    p.few = rows <= 256 || c.dim > 128 || most * c.dim * 8 <= kL2Bytes;
  else
    p.few = rows <= (c.dim <= 64 ? 64 : c.dim <= 128 ? 16 : 8);
  p.few &= tokens * heads / 16 < kMostGroups;
  p.rows = p.few ? 16 : 128;
  // every sequence's last tile may be partly empty
  p.tiles = tokens * group / p.rows + std::min(c.sequences, tokens);
  // Splits: so many workgroups per CU, which also evens out sequences of different
  // lengths, but none of fewer than 128 keys (joining costs a launch and what the parts
  // take). Few rows: four, of wide heads, which fill the registers, two (64 x 16384
  // keys x 128, 2, 4 and 8 per CU: 559, 566, 557 us; 16 x 4000 keys 43, 43, 49; 20 x
  // 10000 keys x 256 103, 133, 179). Chunks: two, as many as a CU holds (1 x 512 rows
  // over 8192 keys, 1, 2 and 4: 187, 116, 136 us; 2 x 2048 over 2048 98, 98, 114); in
  // fp32 one, which the matrix cores are busy with (3 x 300 over 2500, 1 and 2: 91, 97).
  const int per_cu = p.few ? (c.dim <= 128 ? 4 : 2) : c.dtype == LSSVM_F32 ? 1 : 2;
  const int64_t whole = std::max<int64_t>(1, std::max(tokens * group / p.rows,
                                                      std::min(c.sequences, tokens)) * c.heads);
  const int64_t want = std::max<int64_t>(1, per_cu * kCUs / whole);
  p.splits = (int)std::max<int64_t>(
      1, std::min<int64_t>({want, (most + 127) / 128, p.few ? kMostSplits : 16}));
  // Short caches of few tiles: eight waves in place of four go over them whole, and
  // nothing is to be joined (1 x 500 keys 11 us against 14, 1000 15 against 14).
  if (p.few && c.dim <= 128 && whole <= kCUs && most <= kWideKeys) {
    p.wide = true;
    p.splits = 1;
  }
  // Weights of up to 32 rows come from their scores, which then take 4 bytes per row and
  // key; of more, the scores are formed again.
  p.pitch = accumulate && p.few && rows <= 32 ? round_up(most, 32) : 0;
  return p;
}

struct Carver {
  char* base;
  size_t off = 0;
  template <typename U>
  U* take(int64_t count) {
    U* p = base ? reinterpret_cast<U*>(base + off) : nullptr;
    off = (off + (size_t)count * sizeof(U) + 255) / 256 * 256;
    return p;
  }
};

size_t carve(AttentionArgs& a, void* workspace) {
  Carver c{static_cast<char*>(workspace)};
  const int64_t rows = a.tokens * a.heads;
  a.lse = c.take<float>(a.accumulate ? rows : 0);
  a.part = c.take<float>(a.plan.splits > 1 ? a.plan.splits * rows * a.c.dim : 0);
  a.part_ml = c.take<float2>(a.plan.splits > 1 ? a.plan.splits * rows : 0);
  a.scores = c.take<float>(a.plan.pitch * rows);
  if (!a.accumulate) a.lse = nullptr;
  return std::max<size_t>(c.off, 256);
}

// Joins the splits of 16 rows of a tile: out = sum_i 2^(m_i - m) part_i / sum_i 2^(m_i - m) l_i.
// Four values of a row per thread, eight splits on their way at once. It waits for its own
// chain of loads: 5 us for 32 rows of 12 splits, 6 us for 4200 rows of 2.
template <typename T>
__global__ void __launch_bounds__(256) k_attention_join(AttentionArgs a, int block, int least) {
  Tile t;
  if (!find_tile(a, blockIdx.x, a.plan.rows, &t)) return;
  const int per = split_blocks(t.keys, block, a.plan.splits, least);
  const int used = ((t.keys + block - 1) / block + per - 1) / per;
  if (used <= 1) return;
  const int hk = blockIdx.y, dim = (int)a.c.dim, quads = dim / 4, y0 = 16 * blockIdx.z;
  const int here = min(16, t.rows - y0);
  const int64_t rows = a.tokens * a.heads;
  auto row = [&](int y) {
    const int r = t.row0 + y0 + y;
    return (t.first + r / a.group) * a.heads + hk * a.group + r % a.group;
  };
  // every split's factor 2^(m_i - m) and the sum of all, once per row
  __shared__ float2 ml[16][kMostSplits];
  __shared__ float2 whole[16];
  for (int x = threadIdx.x; x < here * used; x += 256)
    ml[x / used][x % used] = a.part_ml[x % used * rows + row(x / used)];
  __syncthreads();
  if (threadIdx.x < here) {
    const int y = threadIdx.x;
    float m = -INFINITY, l = 0.0f;
    for (int i = 0; i < used; ++i) m = fmaxf(m, ml[y][i].x);
    const float base = m == -INFINITY ? 0.0f : m;
    bool sees = false;
    for (int i = 0; i < used; ++i) {
      const float f = __builtin_amdgcn_exp2f(ml[y][i].x - base);
      l += ml[y][i].y * f;
      sees |= ml[y][i].y < 0.0f;
      ml[y][i].x = f;
    }
    whole[y] = float2{m, l == 0.0f && sees ? __builtin_nanf("") : l};
  }
  __syncthreads();
  for (int x = threadIdx.x; x < here * quads; x += 256) {
    const int y = x / quads, d = x % quads * 4;
    const int r = t.row0 + y0 + y, tok = r / a.group, h = hk * a.group + r % a.group;
    const int64_t at = row(y);
    f32x4 v{};
#pragma unroll 8
    for (int i = 0; i < used; ++i)
      v += *reinterpret_cast<const f32x4*>(a.part + (i * rows + at) * dim + d) * ml[y][i].x;
    const float m = whole[y].x, l = whole[y].y;
    const float inv = 1.0f / l;
    Loose<T, 4> w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w.v[i] = (T)(l == 0.0f ? 0.0f : v[i] * inv);
    *reinterpret_cast<Loose<T, 4>*>(static_cast<T*>(a.out) + (t.first + tok) * a.os.outer +
                                    h * a.os.head + d) = w;
    if (a.lse && d == 0) a.lse[at] = l == 0.0f ? INFINITY : m + __builtin_amdgcn_logf(l);
  }
}

// weight_out = weight + the probabilities of few rows, from their stored scores. A
// thread has four keys: their rows are summed in order. Bound by memory: 64 x 4 rows of
// 12288 keys x 8 heads, 150 MB, in 40 us (3.7 TB/s; with a key per thread 69 us).
constexpr int kWeightKeys = 1024;   // per block
__global__ void __launch_bounds__(kWeightKeys / 4) k_weights_few(AttentionArgs a) {
  const int s = blockIdx.z, hk = blockIdx.y;
  const int L = cache_length(a.c, s);
  const int j = blockIdx.x * kWeightKeys + 4 * (int)threadIdx.x;
  if (j >= L) return;
  int64_t first;
  int n;
  sequence_rows(a, s, &first, &n);
  float gain[4] = {};
  for (int i = 0; i < n; ++i) {
    const int seen = a.causal ? L - n + i + 1 - j : L - j;   // of these keys and on
    if (seen <= 0) continue;
    const int64_t row = (first + i) * a.heads + hk * a.group;
#pragma unroll 4
    for (int h = 0; h < a.group; ++h) {
      const float lse = a.lse[row + h];
      const f32x4 z = *reinterpret_cast<const f32x4*>(a.scores + (row + h) * a.plan.pitch + j);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        gain[k] += k < seen ? __builtin_amdgcn_exp2f(z[k] - lse) : 0.0f;
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (j + k >= L) break;
    int slot;
    const int page = cache_page(a.c, s, j + k, &slot);
    if (page < 0) continue;
    const float old = a.c.weight[page * a.c.weight_stride[0] + hk * a.c.weight_stride[1] + slot];
    a.weight_out[page * a.ws.outer + hk * a.ws.head + slot] = old + gain[k];
  }
}

}  // namespace

size_t attention_workspace(const lssvm_cache& c, int64_t tokens, int heads, bool accumulate) {
  AttentionArgs a{};
  a.c = c;
  a.tokens = tokens;
  a.heads = heads;
  a.accumulate = accumulate;
  a.plan = make_plan(c, tokens, heads, accumulate);
  return carve(a, nullptr);
}

template <typename T>
hipError_t join(const AttentionArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.plan.tiles, (unsigned)a.c.heads, (unsigned)a.plan.rows / 16);
  const int block = a.plan.few ? few_keys<T> : chunk_keys<T>;
  k_attention_join<T><<<grid, 256, 0, stream>>>(a, block, a.plan.few ? kFewLeast : kChunkLeast);
  return hipGetLastError();
}

hipError_t launch_attention(AttentionArgs a, void* workspace, hipStream_t stream) {
  a.plan = make_plan(a.c, a.tokens, a.heads, a.accumulate);
  carve(a, workspace);
  hipError_t e = hipSuccess;
  if (a.tokens > 0) {
    e = a.plan.few ? launch_attention_few(a, stream) : launch_attention_chunk(a, stream);
    if (e == hipSuccess && a.plan.splits > 1)
      e = a.c.dtype == LSSVM_BF16  ? join<bf16_t>(a, stream)
          : a.c.dtype == LSSVM_F16 ? join<f16_t>(a, stream)
                                   : join<float>(a, stream);
  }
  if (e != hipSuccess || !a.accumulate) return e;
  if (a.plan.pitch == 0) return launch_weights_chunk(a, stream);
  k_weights_few<<<dim3((unsigned)((a.c.columns * a.c.page + kWeightKeys - 1) / kWeightKeys),
                       (unsigned)a.c.heads, (unsigned)a.c.sequences),
                  kWeightKeys / 4, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace lssvm
