// fcp_cache_attn: attention of the last tokens of every sequence over a paged 8-bit cache, and the sums of the weights that every cached token gets.
//
// O = softmax(scale Q K^T) V, rows of one KV head's whole group together (row r = token r / G, query head r % G of the group), keys in tiles of 64.
// For single tokens the cache's bytes bound it: every code is read once, and everything else has to hide behind that.
//   * S^T = K Q^T with the 16 x 16 x 32 bf16 instructions: the keys are the matrix rows, a query row is a column, so its maximum and sum stay in the lane.
//     Matrix row m of key tile t (of four) is key 16 (m / 4) + 4 t + m % 4 of the 64: then lane (column n, group g) ends with the scores of the 16
//     neighbouring keys 16 g .. 16 g + 15, in order, which is the operand that the product with V needs, without any exchange.
//   * O^T += V^T P^T: the cache holds values in groups of 16 tokens, a channel's 16 codes together, so a lane's 16 bytes are its channel's codes of its keys.
//   * Codes go from memory to registers in 16-byte loads and become bf16 there (exact); the keys' scale multiplies the scores, the values' scale (a power
//     of two) the probabilities.  The wave needs no LDS and no barrier in its loop.
// All (sequence, KV head, block of rows, key tile) form one line, cut into equal pieces for the blocks: a long sequence is split over many blocks and short ones
// share one, however ragged the lengths, which only the device knows.  The pieces of an item that does not lie in one block meet in a second launch.
#include "fcp_cache.h"

namespace fcp {
namespace {

constexpr int kTile = 64;              // keys of a tile
constexpr int kWaves = 4;              // of a block
constexpr int kLeastTiles = 4;         // of a block, where there are few
constexpr float kLow = -1e30f;         // running maximum before the first key: finite, so that exp2(-inf - it) is 0

struct AttnArgs {
  CacheView c;
  SeqView s;
  const __bf16* q;
  int64_t q_row;
  int32_t hq, group;
  float scale;                         // softmax_scale * log2(e)
  __bf16* o;
  float* lse;
  float* part;                         // two slots per block: rows x (D + 2) floats
  float* scores;                       // weigh: [tile][16 rows][64 keys], scaled by log2(e); or NULL
  int32_t blocks;                      // that share the line
};

// An item's sequence, and the line's length.
struct Line {
  int64_t total;                       // tiles of all items
  int64_t before;                      // tiles of the sequences before `seq`
  int32_t seq;
};

__device__ inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
__device__ inline int32_t tiles_of(int len) { return max((len + kTile - 1) / kTile, 1); }
// tiles on the line of a sequence: every block of `rows` rows of every KV head walks all of them (a sequence without cached tokens: one empty tile, which writes O = 0)
__device__ inline int64_t cost_of(const SeqSizes& z, int hkv, int group, int rows) {
  return z.n == 0 ? 0 : (int64_t)hkv * div_up((int64_t)z.n * group, rows) * tiles_of(z.len);
}

// The sequence that holds place `x` of the line (x < 0: sequence `want` is given and its `before` asked for).  Every thread of the block calls; 256 threads.
__device__ inline Line find_on_line(const SeqView& s, const CacheView& c, int group, int rows, int blocks, int block, int want) {
  __shared__ int64_t sums[kWaves];
  __shared__ int64_t found[2];
  const int per = (s.n_seqs + 255) / 256, a = min((int)threadIdx.x * per, s.n_seqs), b = min(a + per, s.n_seqs);
  int64_t mine = 0;
  for (int i = a; i < b; ++i) mine += cost_of(seq_sizes(s, i, c.page), c.hkv, group, rows);
  int64_t upto = mine;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t v = __shfl_up(upto, d);
    if (lane >= d) upto += v;
  }
  __syncthreads();                     // (of an earlier call, everybody has what it found)
  if (lane == 63) sums[threadIdx.x >> 6] = upto;
  if (threadIdx.x == 0) found[0] = -1;
  __syncthreads();
  int64_t total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < (int)(threadIdx.x >> 6)) upto += sums[w];
    total += sums[w];
  }
  int64_t at = upto - mine;            // of the thread's first sequence
  const int64_t x = want >= 0 ? 0 : (int64_t)block * total / blocks;
  if (want >= 0 ? (want >= a && want < b) : (x >= at && x < upto)) {
    for (int i = a; i < b; ++i) {
      const int64_t n = cost_of(seq_sizes(s, i, c.page), c.hkv, group, rows);
      if (want >= 0 ? i == want : x < at + n) {
        found[0] = i;
        found[1] = at;
        break;
      }
      at += n;
    }
  }
  __syncthreads();
  return {total, found[1], (int32_t)found[0]};
}

// Blocks that get a share of the line: those of the grid, fewer where there are few tiles.
__device__ inline int32_t sharing(int64_t total, int32_t blocks) { return (int32_t)min((int64_t)blocks, div_up(total, kLeastTiles)); }
__device__ inline int64_t share_begin(int64_t total, int32_t sharers, int32_t i) { return total * i / sharers; }
__device__ inline int32_t sharer_of(int64_t total, int32_t sharers, int64_t x) { return (int32_t)(((x + 1) * sharers - 1) / total); }

template <int D>
struct PartSlot { static constexpr int floats(int rows) { return rows * (D + 2); } };   // [rows][D] sums, [rows] maxima, [rows] sums of exponentials

// What a wave keeps of 16 * NB rows.
template <int D, int NB>
struct RowState {
  f32x4 o[NB][D / 16];
  float m[NB], l[NB];
};

// One wave's codes of a tile: keys, values, and the scales of the lane's 16 keys.
template <int D>
struct TileCodes {
  u32x4 k[4][D / 64], v[D / 16];
  float ks, vs;
  bool there;                          // the page of the lane's 16 keys exists and holds cached tokens
};

template <int D>
__device__ inline void load_tile(const AttnArgs& a, int seq, int head, int len, int tile, TileCodes<D>& t) {
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int key0 = tile * kTile;
  // keys: the lane's matrix row n holds, in key tile i, key 16 (n / 4) + 4 i + n % 4
  const int kk = key0 + 16 * (n >> 2);
  const int32_t kp = kk < len ? page_at(a.s, a.c, seq, kk >> a.c.log_page) : -1;
  const uint8_t* kb = a.c.k + (block_of(a.c, max(kp, 0), head) * a.c.page + ((kk + (n & 3)) & (a.c.page - 1))) * D + 16 * g;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < D / 64; ++j) t.k[i][j] = *reinterpret_cast<const u32x4*>(kb + 4 * i * D + 64 * j);
  const int vk = key0 + 16 * g;
  const int32_t vp = vk < len ? page_at(a.s, a.c, seq, vk >> a.c.log_page) : -1;
  const int64_t block = block_of(a.c, max(vp, 0), head);
  const uint8_t* vb = a.c.v + (block * a.c.page + (vk & (a.c.page - 1))) * D + 16 * n;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) t.v[i] = *reinterpret_cast<const u32x4*>(vb + 256 * i);
  t.there = vp >= 0;
  t.ks = t.there ? a.c.k_scale[block] : 0.f;
  t.vs = t.there ? a.c.v_scale[block] : 0.f;
}

__device__ inline float max_over_groups(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float sum_over_groups(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Which of the lane's 16 values are NaN codes, as values codes of 1 (and 0): for the columns that a mask hides them from.
__device__ inline uint32_t nan_bytes(uint32_t w) {         // 0x38 (1.0) where a byte is 0x7f or 0xff
  const uint32_t x = (w & 0x7f7f7f7fu) + 0x01010101u;      // 0x80 exactly for 0x7f
  return ((x & 0x80808080u) >> 7) * 0x38u;
}

// Scores, softmax and product of one tile for 16 rows (query fragments q, state of row block b).
template <int D, int Fmt, int NB>
__device__ inline void work_tile(const AttnArgs& a, TileCodes<D>& t, const bf16x8 (&q)[NB][D / 32], RowState<D, NB>& r, int tile, const int (&last)[NB], int len,
                                 bool full, float* scores) {
  const int lane = threadIdx.x & 63, g = lane >> 4;
  const int key0 = tile * kTile + 16 * g;                  // the lane's keys
  f32x4 s[NB][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b][i] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < D / 64; ++j) {
      const bf16x8 k0 = decode8<Fmt>(t.k[i][j][0], t.k[i][j][1]), k1 = decode8<Fmt>(t.k[i][j][2], t.k[i][j][3]);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        s[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[b][2 * j], s[b][i], 0, 0, 0);
        s[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[b][2 * j + 1], s[b][i], 0, 0, 0);
      }
    }
  }
  const float c = a.scale * t.ks;
  bf16x8 p[NB][2];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float x = s[b][i / 4][i % 4] * c;
      if (!full) x = t.there && key0 + i <= last[b] ? x : -INFINITY;
      s[b][i / 4][i % 4] = x;
      top = fmaxf(top, x);
    }
    if (scores)
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4*>(scores + (16 * b + (lane & 15)) * kTile + 16 * g + 4 * i) = s[b][i];
    // the maximum only grows in steps of more than 2^8: probabilities stay below 256, and most tiles leave the sums alone
    if (__ballot(top > r.m[b] + 8.f)) {
      const float m = fmaxf(r.m[b], max_over_groups(top));
      const float f = __builtin_amdgcn_exp2f(r.m[b] - m);
      r.m[b] = m;
      r.l[b] *= f;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) r.o[b][d] *= f;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float e = __builtin_amdgcn_exp2f(s[b][i / 4][i % 4] - r.m[b]);
      r.l[b] += e;
      p[b][i / 8][i % 8] = (__bf16)(e * t.vs);
    }
  }
  uint32_t odd = 0;
  if (!full) {
    // codes past the last token are whatever the page holds, and 0 * NaN is NaN: clear them
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int live = t.there ? min(max(len - key0 - 4 * w, 0), 4) : 0;
        t.v[i][w] = live == 4 ? t.v[i][w] : t.v[i][w] & ((1u << (8 * live)) - 1);
        if (Fmt == kE4m3) odd |= nan_bytes(t.v[i][w]);
      }
  }
  if (Fmt == kE4m3 && !full && __ballot(odd)) {
    // Rare: a cached value is NaN in a tile that some row sees in part.  Its rows get NaN, and only they: the NaN codes leave the product, and their
    // number among the keys that a row sees is counted by a product with 1.
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      u32x4 bad;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        bad[w] = nan_bytes(t.v[i][w]);
        t.v[i][w] &= ~(((bad[w] >> 3) & 0x01010101u) * 0xffu);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        f32x4 count = {0, 0, 0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16x8 seen;
#pragma unroll
          for (int j = 0; j < 8; ++j) seen[j] = (__bf16)(t.there && key0 + 8 * h + j <= last[b] ? 1.f : 0.f);
          count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8<Fmt>(bad[2 * h], bad[2 * h + 1]), seen, count, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) r.o[b][i][j] = count[j] > 0.f ? NAN : r.o[b][i][j];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bf16x8 v = decode8<Fmt>(t.v[i][2 * h], t.v[i][2 * h + 1]);
#pragma unroll
      for (int b = 0; b < NB; ++b) r.o[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[b][h], r.o[b][i], 0, 0, 0);
    }
}

// Final row, or its part: o channels 16 i + 4 g + 0..3 of the lane's row.
template <int D>
__device__ inline void write_row(const AttnArgs& a, int row, int head, const f32x4 (&o)[D / 16], float m, float l, int g) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
  __bf16* y = a.o + ((int64_t)row * a.hq + head) * D + 4 * g;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    bf16x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (__bf16)(o[i][j] * inv);
    *reinterpret_cast<bf16x4*>(y + 16 * i) = w;
  }
  if (g == 0) a.lse[(int64_t)head * a.s.n_rows + row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Waves of a block divide the tiles of a piece (Keys) or take rows of their own.
template <int D, int Fmt, int NB, bool Keys>
__global__ __launch_bounds__(256) void attn_kernel(AttnArgs a) {
  constexpr int kRows = 16 * NB * (Keys ? 1 : kWaves);     // of a block
  constexpr int kStride = D + 4;                           // floats of a staged row: rows on different banks
  __shared__ float stage[Keys ? kWaves * 16 * NB * kStride : 1];
  __shared__ float stage_m[kWaves * 16 * NB], stage_l[kWaves * 16 * NB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  // total first: how many blocks share the line depends on it
  Line line = find_on_line(a.s, a.c, a.group, kRows, 1, 0, -1);
  if (line.total == 0) return;
  const int32_t sharers = sharing(line.total, a.blocks), me = blockIdx.x;
  if (me >= sharers) return;
  int64_t at = share_begin(line.total, sharers, me);
  const int64_t end = share_begin(line.total, sharers, me + 1);
  line = find_on_line(a.s, a.c, a.group, kRows, sharers, me, -1);
  int seq = line.seq;
  int64_t base = line.before;
  SeqSizes z = seq_sizes(a.s, seq, a.c.page);
  while (at < end) {
    while (at >= base + cost_of(z, a.c.hkv, a.group, kRows)) {      // the next sequence with rows
      base += cost_of(z, a.c.hkv, a.group, kRows);
      z = seq_sizes(a.s, ++seq, a.c.page);
    }
    const int tiles = tiles_of(z.len), all_rows = z.n * a.group, row_blocks = (all_rows + kRows - 1) / kRows;
    const int item = (int)((at - base) / tiles), t0 = (int)((at - base) % tiles);
    const int t1 = (int)min((int64_t)tiles, t0 + end - at);
    const int head = item / row_blocks, rb = item % row_blocks;
    const int64_t at0 = at;
    at += t1 - t0;

    bf16x8 q[NB][D / 32];
    RowState<D, NB> r;
    int last[NB];                                          // last token that the lane's row sees
    int first_seen = INT32_MAX;                            // least of them in the wave
    bool any = false;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int row = rb * kRows + (Keys ? 0 : wave * 16 * NB) + 16 * b + n;
      const bool live = row < all_rows;
      const int tok = live ? row / a.group : 0;
      last[b] = live ? z.len - z.n + tok : -1;
      any = any || live;
      first_seen = min(first_seen, live ? last[b] : INT32_MAX);
      const __bf16* x = a.q + (int64_t)(z.row0 + tok) * a.q_row + (head * a.group + (live ? row % a.group : 0)) * D + 16 * g;
#pragma unroll
      for (int j = 0; j < D / 64; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bf16x8 w = *reinterpret_cast<const bf16x8*>(x + 64 * j + 8 * h);
          bf16x8 zero = {};
          q[b][2 * j + h] = live ? w : zero;
        }
      r.m[b] = kLow;
      r.l[b] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) r.o[b][i] = f32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) first_seen = min(first_seen, __shfl_xor(first_seen, d));
    // the last tile that any row of the block sees
    const int last_row = min(rb * kRows + kRows, all_rows) - 1, seen = z.len - z.n + last_row / a.group;
    const int t_end = min(t1, seen < 0 ? 0 : seen / kTile + 1);
    if (Keys || __ballot(any)) {
      TileCodes<D> t;
      for (int i = t0 + (Keys ? wave : 0); i < t_end; i += Keys ? kWaves : 1) {
        load_tile<D>(a, seq, head, z.len, i, t);
        const bool full = i * kTile + kTile - 1 <= first_seen && __ballot(!t.there) == 0;
        work_tile<D, Fmt, NB>(a, t, q, r, i, last, z.len, full, a.scores ? a.scores + (at0 - t0 + i) * (16 * kTile) : nullptr);
      }
      if (Keys && a.scores)                                // tiles of the piece that nobody sees
        for (int i = max(t_end, t0) + wave; i < t1; i += kWaves)
          for (int j = lane; j < 16 * kTile; j += 64) a.scores[(at0 - t0 + i) * (16 * kTile) + j] = -INFINITY;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) r.l[b] = sum_over_groups(r.l[b]);

    const bool whole = t0 == 0 && t1 == tiles;
    float* const slot = a.part + (int64_t)(2 * me + (t0 == 0 ? 1 : 0)) * PartSlot<D>::floats(kRows);
    if constexpr (Keys) {
      // the four waves' sums in the block's LDS, then each wave finishes a quarter of the channels
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int row = wave * 16 * NB + 16 * b + n;
        if (g == 0) { stage_m[row] = r.m[b]; stage_l[row] = r.l[b]; }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(&stage[row * kStride + 16 * i + 4 * g]) = r.o[b][i];
      }
      __syncthreads();
      for (int j = threadIdx.x; j < 16 * NB * (D / 4); j += 256) {
        const int lr = j / (D / 4), ch = 4 * (j % (D / 4)), row = rb * kRows + lr;
        if (row >= all_rows) continue;
        float m = kLow, l = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = fmaxf(m, stage_m[w * 16 * NB + lr]);
        f32x4 o = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = __builtin_amdgcn_exp2f(stage_m[w * 16 * NB + lr] - m);
          l += f * stage_l[w * 16 * NB + lr];
          o += f * *reinterpret_cast<const f32x4*>(&stage[(w * 16 * NB + lr) * kStride + ch]);
        }
        if (whole) {
          const int tok = z.row0 + row / a.group, h = head * a.group + row % a.group;
          const float inv = l == 0.f ? 0.f : 1.f / l;
          bf16x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = (__bf16)(o[i] * inv);
          *reinterpret_cast<bf16x4*>(a.o + ((int64_t)tok * a.hq + h) * D + ch) = w;
          if (ch == 0) a.lse[(int64_t)h * a.s.n_rows + tok] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
        } else {
          *reinterpret_cast<f32x4*>(slot + lr * D + ch) = o;
          if (ch == 0) { slot[kRows * D + lr] = m; slot[kRows * (D + 1) + lr] = l; }
        }
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int lr = wave * 16 * NB + 16 * b + n, row = rb * kRows + lr;
        if (row >= all_rows) continue;
        if (whole) {
          write_row<D>(a, z.row0 + row / a.group, head * a.group + row % a.group, r.o[b], r.m[b], r.l[b], g);
        } else {
#pragma unroll
          for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(slot + lr * D + 16 * i + 4 * g) = r.o[b][i];
          if (g == 0) { slot[kRows * D + lr] = r.m[b]; slot[kRows * (D + 1) + lr] = r.l[b]; }
        }
      }
    }
  }
}

// The items that several blocks worked: a block per (row, KV head), a wave per query head of the group, two or four channels a lane.
template <int D>
__global__ __launch_bounds__(256) void attn_merge_kernel(AttnArgs a, int rows_of_block) {
  const int tok = blockIdx.x / a.c.hkv, head = blockIdx.x % a.c.hkv, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // the row's sequence: the last one that begins at or before it and has rows
  int lo = 0, n = a.s.n_seqs;
  while (n > 1) {
    const int step = (n + 63) / 64, at = lo + lane * step;
    const int k = __popcll(__ballot(at < lo + n && a.s.cu[at] <= tok)) - 1, next = lo + max(k, 0) * step;
    n = min(step, lo + n - next);
    lo = next;
  }
  const int seq = lo;
  const SeqSizes z = seq_sizes(a.s, seq, a.c.page);
  if (tok < z.row0 || tok >= z.row0 + z.n) return;         // (uniform over the block)
  const Line line = find_on_line(a.s, a.c, a.group, rows_of_block, 1, 0, seq);
  const int32_t sharers = sharing(line.total, a.blocks);
  const int tiles = tiles_of(z.len), row_blocks = (z.n * a.group + rows_of_block - 1) / rows_of_block;
  for (int h = wave; h < a.group; h += kWaves) {
    const int row = (tok - z.row0) * a.group + h, rb = row / rows_of_block, lr = row % rows_of_block;
    const int64_t x = line.before + ((int64_t)head * row_blocks + rb) * tiles;
    const int32_t w0 = sharer_of(line.total, sharers, x), w1 = sharer_of(line.total, sharers, x + tiles - 1);
    if (w0 == w1) continue;
    const int floats = PartSlot<D>::floats(rows_of_block);
    auto slot = [&](int w) { return a.part + (int64_t)(2 * w + (w == w0 ? 1 : 0)) * floats; };
    float m = kLow;
    for (int w = w0 + lane; w <= w1; w += 64) m = fmaxf(m, slot(w)[rows_of_block * D + lr]);
    m = wave_maxf(m);
    float l = 0.f;
    constexpr int kCh = D / 64;
    float o[kCh] = {};
#pragma unroll 4
    for (int w = w0; w <= w1; ++w) {
      const float* s = slot(w);
      const float f = __builtin_amdgcn_exp2f(s[rows_of_block * D + lr] - m);
      l += f * s[rows_of_block * (D + 1) + lr];
#pragma unroll
      for (int i = 0; i < kCh; ++i) o[i] += f * s[lr * D + kCh * lane + i];
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    __bf16* y = a.o + ((int64_t)tok * a.hq + head * a.group + h) * D + kCh * lane;
#pragma unroll
    for (int i = 0; i < kCh; ++i) y[i] = (__bf16)(o[i] * inv);
    if (lane == 0) a.lse[(int64_t)(head * a.group + h) * a.s.n_rows + tok] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

// ---- weights ------------------------------------------------------------------------------------

// Adds exp(score - LSE), summed over the rows of the group, to the tokens' weights.  A block takes one (sequence, KV head, tile) at a time, the longest-seen
// first; its waves divide the rows.  The 16 sums of a lane (its keys) over its column's rows are added over the 16 columns, then over the waves.
struct WeighArgs {
  CacheView c;
  SeqView s;
  const __bf16* q;
  int64_t q_row;
  int32_t hq, group;
  float scale;
  const float* lse;
  int64_t lse_head;                    // floats between heads
};

template <int D, int Fmt>
__global__ __launch_bounds__(256) void weigh_kernel(WeighArgs a) {
  __shared__ float sum[kWaves][kTile];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  // the line with one block of rows per KV head
  const int kAll = INT32_MAX;
  const Line line = find_on_line(a.s, a.c, 1, kAll, 1, 0, -1);
  int seq = 0;
  int64_t base = 0;
  SeqSizes z = seq_sizes(a.s, 0, a.c.page);
  for (int64_t u = blockIdx.x; u < line.total; u += gridDim.x) {
    __syncthreads();                   // (everybody has read the sums of the tile before)
    while (u >= base + cost_of(z, a.c.hkv, 1, kAll)) {
      base += cost_of(z, a.c.hkv, 1, kAll);
      z = seq_sizes(a.s, ++seq, a.c.page);
    }
    const int tile = (int)((u - base) / a.c.hkv), head = (int)((u - base) % a.c.hkv);
    TileCodes<D> t;
    const int key0 = tile * kTile;
    {
      const int kk = key0 + 16 * (n >> 2);
      const int32_t kp = kk < z.len ? page_at(a.s, a.c, seq, kk >> a.c.log_page) : -1;
      const uint8_t* kb = a.c.k + (block_of(a.c, max(kp, 0), head) * a.c.page + ((kk + (n & 3)) & (a.c.page - 1))) * D + 16 * g;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < D / 64; ++j) t.k[i][j] = *reinterpret_cast<const u32x4*>(kb + 4 * i * D + 64 * j);
      const int vk = key0 + 16 * g;
      const int32_t vp = vk < z.len ? page_at(a.s, a.c, seq, vk >> a.c.log_page) : -1;
      t.there = vp >= 0;
      t.ks = t.there ? a.c.k_scale[block_of(a.c, vp, head)] : 0.f;
    }
    bf16x8 k[4][D / 32];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < D / 64; ++j) {
        k[i][2 * j] = decode8<Fmt>(t.k[i][j][0], t.k[i][j][1]);
        k[i][2 * j + 1] = decode8<Fmt>(t.k[i][j][2], t.k[i][j][3]);
      }
    const float c = a.scale * t.ks;
    float got[16] = {};
    const int all_rows = z.n * a.group;
    // the first token that sees the tile's first key
    const int tok0 = max(key0 - (z.len - z.n), 0), rb0 = (int)((int64_t)tok0 * a.group / 16);
    for (int rb = rb0 + wave; rb * 16 < all_rows; rb += kWaves) {
      const int row = rb * 16 + n;
      const bool live = row < all_rows;
      const int tok = live ? row / a.group : 0, h = head * a.group + (live ? row % a.group : 0);
      const int last = live ? z.len - z.n + tok : -1;
      const float lse2 = live ? a.lse[h * a.lse_head + z.row0 + tok] * kLog2e : -INFINITY;
      const __bf16* x = a.q + (int64_t)(z.row0 + tok) * a.q_row + h * D + 16 * g;
      f32x4 s[4] = {};
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        const bf16x8 q = *reinterpret_cast<const bf16x8*>(x + 64 * (j / 2) + 8 * (j % 2));
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[i][j], q, s[i], 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = __builtin_amdgcn_exp2f(s[i / 4][i % 4] * c - lse2);
        got[i] += t.there && key0 + 16 * g + i <= last && lse2 != -INFINITY ? p : 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int d = 8; d > 0; d >>= 1) got[i] += __shfl_xor(got[i], d);
    if (n == 0)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[wave][16 * g + i] = got[i];
    __syncthreads();
    if (threadIdx.x < kTile && key0 + (int)threadIdx.x < z.len) {
      const int key = key0 + threadIdx.x;
      const int32_t p = page_at(a.s, a.c, seq, key >> a.c.log_page);
      if (p >= 0) {
        float* w = a.c.weight + block_of(a.c, p, head) * a.c.page + (key & (a.c.page - 1));
        *w += (sum[0][threadIdx.x] + sum[1][threadIdx.x]) + (sum[2][threadIdx.x] + sum[3][threadIdx.x]);
      }
    }
  }
}

// The same from the scores that the attention kernel left (few rows): a wave per (sequence, KV head, tile), a key per lane.
__global__ __launch_bounds__(256) void weigh_scores_kernel(AttnArgs a, int rows_of_block) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Line line = find_on_line(a.s, a.c, a.group, rows_of_block, 1, 0, -1);
  if (line.total == 0) return;
  const int32_t sharers = sharing(line.total, a.blocks * kWaves), me = blockIdx.x;   // (a share has a few tiles of its own)
  if (me >= sharers) return;
  int64_t at = share_begin(line.total, sharers, me);
  const int64_t end = share_begin(line.total, sharers, me + 1);
  line = find_on_line(a.s, a.c, a.group, rows_of_block, sharers, me, -1);
  int seq = line.seq;
  int64_t base = line.before;
  SeqSizes z = seq_sizes(a.s, seq, a.c.page);
  while (at < end) {
    while (at >= base + cost_of(z, a.c.hkv, a.group, rows_of_block)) {
      base += cost_of(z, a.c.hkv, a.group, rows_of_block);
      z = seq_sizes(a.s, ++seq, a.c.page);
    }
    const int tiles = tiles_of(z.len), all_rows = z.n * a.group, row_blocks = (all_rows + rows_of_block - 1) / rows_of_block;
    const int item = (int)((at - base) / tiles), t0 = (int)((at - base) % tiles), t1 = (int)min((int64_t)tiles, t0 + end - at);
    const int head = item / row_blocks, rb = item % row_blocks;
    // the rows of all blocks of a head add to the same weights: those of the first block's share do it, so that no two do
    if (rb == 0)
      for (int i = t0 + wave; i < t1; i += kWaves) {
        const int key = i * kTile + lane;
        float got = 0.f;
        for (int row = 0; row < all_rows; ++row) {
          const float lse = a.lse[(int64_t)(head * a.group + row % a.group) * a.s.n_rows + z.row0 + row / a.group];
          if (lse == -INFINITY) continue;
          const float* s = a.scores + (base + ((int64_t)head * row_blocks + row / rows_of_block) * tiles + i) * (16 * kTile);
          got += __builtin_amdgcn_exp2f(s[(row % rows_of_block) * kTile + lane] - lse * kLog2e);
        }
        const int32_t p = key < z.len ? page_at(a.s, a.c, seq, key >> a.c.log_page) : -1;
        if (p >= 0) a.c.weight[block_of(a.c, p, head) * a.c.page + (key & (a.c.page - 1))] += got;
      }
    at += t1 - t0;
  }
}

// ---- host ---------------------------------------------------------------------------------------

constexpr int kBlocks = 512;           // that share the line: two per CU

// How a call is worked.  Up to 16 rows per sequence and KV head on average: a block of 16 rows whose waves divide the keys; more: 128 rows, a wave 32.
struct AttnPlan { int rows; bool keys; bool stored; int64_t part_floats, score_floats; };
AttnPlan plan_attn(const CacheView& c, int head_dim, int32_t n_seqs, int32_t max_pages, int32_t tq, int32_t hq, bool weigh) {
  const int group = hq / c.hkv;
  AttnPlan p;
  p.keys = (int64_t)tq * group <= (int64_t)16 * n_seqs;
  p.rows = p.keys ? 16 : 128;
  p.stored = weigh && p.keys;
  p.part_floats = (int64_t)2 * kBlocks * p.rows * (head_dim + 2);
  const int64_t tiles = max(((int64_t)max_pages * c.page + kTile - 1) / kTile, (int64_t)1);
  p.score_floats = p.stored ? tiles * c.hkv * (n_seqs + (int64_t)tq * group / 16) * 16 * kTile : 0;
  return p;
}

template <int D, int Fmt>
int launch_attn(const AttnArgs& a, const AttnPlan& p, bool weigh, hipStream_t st) {
  if (p.keys) attn_kernel<D, Fmt, 1, true><<<dim3(kBlocks), dim3(256), 0, st>>>(a);
  else attn_kernel<D, Fmt, 2, false><<<dim3(kBlocks), dim3(256), 0, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  attn_merge_kernel<D><<<dim3((unsigned)a.s.n_rows * a.c.hkv), dim3(256), 0, st>>>(a, p.rows);
  FCP_HIP_CHECK(hipGetLastError());
  if (p.stored) {
    weigh_scores_kernel<<<dim3(kBlocks * kWaves), dim3(256), 0, st>>>(a, p.rows);
    FCP_HIP_CHECK(hipGetLastError());
  }
  return FCP_OK;
}

int launch_weigh(const WeighArgs& a, int head_dim, int format, hipStream_t st) {
  auto kernel = head_dim == 128 ? (format == kE4m3 ? weigh_kernel<128, kE4m3> : weigh_kernel<128, kInt8>)
                                : (format == kE4m3 ? weigh_kernel<64, kE4m3> : weigh_kernel<64, kInt8>);
  kernel<<<dim3(4 * kBlocks), dim3(256), 0, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  return FCP_OK;
}

int check_heads(const char* who, const CacheView& c, int32_t hq) {
  if (hq < 1 || hq % c.hkv) return fail(FCP_ERR_UNSUPPORTED, "%s: %d query heads on %d KV heads", who, hq, c.hkv);
  return FCP_OK;
}
int check_rows(const char* who, const fcp_cache* cache, const void* q, int64_t q_row, int32_t tq, int32_t hq) {
  if (!q || q_row < (int64_t)hq * cache->head_dim || q_row % 8 || (uintptr_t)q % 16)
    return fail(FCP_ERR_INVALID_ARG, "%s: query rows must be at least hq * head_dim elements apart, a multiple of 8, and 16-byte aligned", who);
  if ((int64_t)tq * cache->hkv > INT32_MAX || (int64_t)tq * (hq / cache->hkv) > INT32_MAX - 256)
    return fail(FCP_ERR_UNSUPPORTED, "%s: more than 2^31 rows of all heads", who);
  return FCP_OK;
}

}  // namespace

size_t evict_scratch_bytes(const CacheView& c, int32_t n_seqs, int32_t max_pages);

}  // namespace fcp

extern "C" size_t fcp_cache_scratch_bytes(int which, const fcp_cache* cache, int32_t n_seqs, int32_t max_pages, int32_t tq, int32_t hq) {
  using namespace fcp;
  clear_error();
  const char* who = "fcp_cache_scratch_bytes";
  CacheView c;
  if (check_cache(who, cache, which != FCP_SCRATCH_CACHE_ATTN, &c)) return 0;
  if (n_seqs < 0 || max_pages < 0 || tq < 0) { fail(FCP_ERR_INVALID_ARG, "%s: negative size", who); return 0; }
  if (which == FCP_SCRATCH_CACHE_EVICT) return evict_scratch_bytes(c, n_seqs, max_pages);
  if (which != FCP_SCRATCH_CACHE_ATTN && which != FCP_SCRATCH_CACHE_WEIGH) { fail(FCP_ERR_INVALID_ARG, "%s: which = %d is not known", who, which); return 0; }
  if (check_heads(who, c, hq)) return 0;
  const bool weigh = which == FCP_SCRATCH_CACHE_WEIGH;
  const AttnPlan p = plan_attn(c, cache->head_dim, n_seqs, max_pages, tq, hq, weigh);
  return pad_to((size_t)p.part_floats * 4, 256) + pad_to((size_t)p.score_floats * 4, 256);
}

extern "C" int fcp_cache_attn(const fcp_cache* cache, const void* q, int64_t q_row, int32_t tq, int32_t hq, const int32_t* cu_seqlens,
                              const int32_t* kv_len, const int32_t* pages, int32_t n_seqs, int32_t max_pages, float softmax_scale, int32_t weigh, void* o,
                              float* lse, void* scratch, size_t scratch_bytes, void* stream) {
  using namespace fcp;
  clear_error();
  const char* who = "fcp_cache_attn";
  AttnArgs a = {};
  if (weigh != 0 && weigh != 1) return fail(FCP_ERR_INVALID_ARG, "%s: weigh must be 0 or 1", who);
  if (int rc = check_cache(who, cache, weigh, &a.c)) return rc;
  if (int rc = check_heads(who, a.c, hq)) return rc;
  if (int rc = check_seqs(who, cu_seqlens, true, kv_len, pages, n_seqs, max_pages, tq)) return rc;
  if (!(softmax_scale > 0.f) || !__builtin_isfinite(softmax_scale)) return fail(FCP_ERR_INVALID_ARG, "%s: softmax_scale must be above 0", who);
  if (tq == 0 || n_seqs == 0) return FCP_OK;
  if (int rc = check_rows(who, cache, q, q_row, tq, hq)) return rc;
  if (!o || !lse || (uintptr_t)o % 16 || (uintptr_t)lse % 4) return fail(FCP_ERR_INVALID_ARG, "%s: o and lse are required and must be aligned", who);
  if (!scratch || (uintptr_t)scratch % 256) return fail(FCP_ERR_INVALID_ARG, "%s: scratch must be 256-byte aligned", who);
  const AttnPlan p = plan_attn(a.c, cache->head_dim, n_seqs, max_pages, tq, hq, weigh);
  const size_t need = pad_to((size_t)p.part_floats * 4, 256) + pad_to((size_t)p.score_floats * 4, 256);
  if (scratch_bytes < need) return fail(FCP_ERR_CAPACITY, "%s: scratch has %zu bytes, %zu are needed", who, scratch_bytes, need);
  a.s = {cu_seqlens, kv_len, pages, n_seqs, max_pages, tq};
  a.q = static_cast<const __bf16*>(q);
  a.q_row = q_row;
  a.hq = hq;
  a.group = hq / a.c.hkv;
  a.scale = softmax_scale * kLog2e;
  a.o = static_cast<__bf16*>(o);
  a.lse = lse;
  a.part = static_cast<float*>(scratch);
  a.scores = p.stored ? reinterpret_cast<float*>(static_cast<char*>(scratch) + pad_to((size_t)p.part_floats * 4, 256)) : nullptr;
  a.blocks = kBlocks;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool e4m3 = cache->format == FCP_CACHE_E4M3;
  const int rc = cache->head_dim == 128 ? (e4m3 ? launch_attn<128, kE4m3>(a, p, weigh, st) : launch_attn<128, kInt8>(a, p, weigh, st))
                                        : (e4m3 ? launch_attn<64, kE4m3>(a, p, weigh, st) : launch_attn<64, kInt8>(a, p, weigh, st));
  if (rc || !weigh || p.stored) return rc;
  const WeighArgs w = {a.c, a.s, a.q, q_row, hq, a.group, a.scale, lse, tq};
  return launch_weigh(w, cache->head_dim, cache->format, st);
}

extern "C" int fcp_cache_weigh(const fcp_cache* cache, const void* q, int64_t q_row, int32_t tq, int32_t hq, const float* lse,
                               const int32_t* cu_seqlens, const int32_t* kv_len, const int32_t* pages, int32_t n_seqs, int32_t max_pages,
                               float softmax_scale, void* stream) {
  using namespace fcp;
  clear_error();
  const char* who = "fcp_cache_weigh";
  WeighArgs a = {};
  if (int rc = check_cache(who, cache, true, &a.c)) return rc;
  if (int rc = check_heads(who, a.c, hq)) return rc;
  if (int rc = check_seqs(who, cu_seqlens, true, kv_len, pages, n_seqs, max_pages, tq)) return rc;
  if (!(softmax_scale > 0.f) || !__builtin_isfinite(softmax_scale)) return fail(FCP_ERR_INVALID_ARG, "%s: softmax_scale must be above 0", who);
  if (tq == 0 || n_seqs == 0) return FCP_OK;
  if (int rc = check_rows(who, cache, q, q_row, tq, hq)) return rc;
  if (!lse || (uintptr_t)lse % 4) return fail(FCP_ERR_INVALID_ARG, "%s: lse is required", who);
  a.s = {cu_seqlens, kv_len, pages, n_seqs, max_pages, tq};
  a.q = static_cast<const __bf16*>(q);
  a.q_row = q_row;
  a.hq = hq;
  a.group = hq / a.c.hkv;
  a.scale = softmax_scale * kLog2e;
  a.lse = lse;
  a.lse_head = tq;
  return launch_weigh(a, cache->head_dim, cache->format, static_cast<hipStream_t>(stream));
}
