// Attention over the cache for few rows: what a wave does with the tiles of a piece (csrc/fcp_cache_attn.hip says how the work is laid out and why).
#pragma once
#include <type_traits>

#include "fcp_cache_attn.h"

namespace fcp {

// What a wave keeps of 16 rows.
template <int D>
struct RowState {
  f32x4 o[D / 16];
  float m, l;
};

// Pages of a tile for a lane: of the keys that its matrix row holds in the four key tiles, 16 (n / 4) + 4 i + n % 4, and of its 16 neighbouring keys 16 g ..; -1: not
// there, or no cached token in it.
struct TilePages { int32_t k, v; };
// The table's entries, of a sequence with cached tokens (past the last token the last one's: a load under a condition is waited for at once, and everything before it too) ..
__device__ inline TilePages ask_pages(const CacheView& c, const int32_t* table, int lane, int len, int tile) {
  const int kk = tile * kTile + 16 * ((lane & 15) >> 2), vk = tile * kTile + 16 * (lane >> 4);
  return {table[min(kk, len - 1) >> c.log_page], table[min(vk, len - 1) >> c.log_page]};
}
// .. and what they say.
__device__ inline TilePages pages_of(const CacheView& c, int lane, const TilePages& entries, int len, int tile) {
  const int kk = tile * kTile + 16 * ((lane & 15) >> 2), vk = tile * kTile + 16 * (lane >> 4);
  const uint32_t n = c.n_pages;
  return {kk < len && (uint32_t)entries.k < n ? entries.k : -1, vk < len && (uint32_t)entries.v < n ? entries.v : -1};
}
template <int D>
__device__ inline void load_keys(const CacheView& c, int lane, int head, int tile, int32_t page, u32x4 (&k)[4][D / 64]) {
  const int n = lane & 15, g = lane >> 4, kk = tile * kTile + 16 * (n >> 2) + (n & 3);
  const uint8_t* p = c.k + (block_of(c, max(page, 0), head) * c.page + (kk & (c.page - 1))) * D + 16 * g;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < D / 64; ++j) k[i][j] = *reinterpret_cast<const u32x4*>(p + 4 * i * D + 64 * j);
}
template <int D>
__device__ inline void load_values(const CacheView& c, int lane, int head, int tile, int32_t page, u32x4 (&v)[D / 16]) {
  const int vk = tile * kTile + 16 * (lane >> 4);
  const uint8_t* p = c.v + (block_of(c, max(page, 0), head) * c.page + (vk & (c.page - 1))) * D + 16 * (lane & 15);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) v[i] = *reinterpret_cast<const u32x4*>(p + 256 * i);
}
// scales of the lane's 16 neighbouring keys (1 where the page is not there: its scores are masked)
struct TileScales { float k, v; };
__device__ inline TileScales scales_of(const CacheView& c, int head, int32_t page) {
  const int64_t block = block_of(c, max(page, 0), head);
  const float k = c.k_scale[block], v = c.v_scale[block];
  return {page >= 0 ? k : 1.f, page >= 0 ? v : 1.f};
}

// S^T of one tile.
template <int D, int Fmt, int NB>
__device__ inline void scores_of(const u32x4 (&k)[4][D / 64], const bf16x8 (&q)[NB][D / 32], f32x4 (&s)[NB][4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b][i] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < D / 32; ++j) {
      const bf16x8 x = decode8<Fmt>(k[i][j / 2][2 * (j % 2)], k[i][j / 2][2 * (j % 2) + 1]);
#pragma unroll
      for (int b = 0; b < NB; ++b) s[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[b][j], s[b][i], 0, 0, 0);
    }
    if (Fmt == kInt8 || NB > 1) __builtin_amdgcn_sched_barrier(0);       // (left alone the compiler converts a tile's codes all at once, which takes 60 registers more and no less time)
  }
}

// A tile that some row of the wave sees in part, values: codes past the last token are whatever the page holds, and 0 * NaN is NaN, so they are cleared.  live: cached tokens among the
// lane's 16, from key0 on.  Rare: one that some rows do not see is NaN.  It leaves the product, and the first such token of each channel is noted in first_nan (of the wave, prepared at
// its first use; noted: there are some): the rows that see it get their NaN when the wave's tiles are done.
template <int D, int Fmt>
__device__ inline void clear_hidden(u32x4 (&v)[D / 16], int live, int key0, int32_t* first_nan, bool& noted) {
  uint32_t odd = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int n = min(max(live - 4 * w, 0), 4);
    const uint32_t keep = n == 4 ? 0xffffffffu : (1u << (8 * n)) - 1;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      v[i][w] &= keep;
      if (Fmt == kE4m3) odd |= ((v[i][w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    }
  }
  if (Fmt != kE4m3 || !__ballot(odd)) return;
  const int lane = lane_id();                              // (formed here: the compiler would keep addresses that follow from it in registers, and spill)
  if (!noted)
#pragma unroll
    for (int c = 0; c < D; c += 64) first_nan[c + lane] = INT32_MAX;
  noted = true;
  wave_exchange();
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    int at = INT32_MAX;
#pragma unroll
    for (int w = 3; w >= 0; --w) {
      const uint32_t nan = ((v[i][w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;        // 0x80 exactly for 0x7f
      if (nan) at = key0 + 4 * w + (__builtin_ctz(nan) >> 3);
      v[i][w] &= ~((nan >> 7) * 0xffu);
    }
    if (at != INT32_MAX) atomicMin(first_nan + 16 * i + (lane & 15), at);
  }
}

// Scores kept of a tile of an item: [rows / 4][4 key tiles][4 groups][4 rows][4 keys], tiles next to each other in the item's part of the line (which has room for 16 rows each).
// 16 neighbouring lanes of a store hold one group, so 4 rows of them are 64 bytes at one place; with rows outside groups they were four places, and that bounded the kernel.
__device__ inline int score_floats(int rows) { return (rows + 3) / 4 * (4 * kTile); }
constexpr int kRing = 16 * 4 * kTile;  // floats of a wave's ring: 16 tiles of four rows, 4 of 16
__device__ inline int score_at(int row) { return row / 4 * (4 * kTile) + row % 4 * 4; }

// Tiles first, first + step, ... below end for NB blocks of 16 rows of one KV head.  last_tok: last tokens that the lane's rows see; all_see: all rows see
// the tokens up to it.  A tile's keys are asked for when the keys before them have become scores, its values when the values before them are in the sums: a wave always has 8 to 16 KB
// on their way.  Page numbers are asked for a tile earlier, right behind keys: loads come back in order, so those behind values would be waited for with the values.
// Scored: the scores are kept (score_rows rows), in `ring` until it is full: stores between the loads hold these up, and that costs less in few long bursts.  64 sequences of 4700 tokens,
// int8, 32 heads on 8, 128 channels, with weights: 150 us, stored tile by tile 161; lengths from 819 to 16384: 180 and 186.
template <int D, int Fmt, bool Scored, int NB>
__device__ inline void walk(const CacheView& cache, float scale, const int32_t* table, int head, int len, int first, int end, int step, const bf16x8 (&q)[NB][D / 32], const int (&last_tok)[NB], int all_see,
                            RowState<D> (&r)[NB], float* scores, int score_rows, float* ring, int32_t* first_nan) {
  if (first >= end) return;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  u32x4 k[4][D / 64], v[D / 16];
  TilePages at = pages_of(cache, lane, ask_pages(cache, table, lane, len, first), len, first), next = ask_pages(cache, table, lane, len, first + step);
  load_keys<D>(cache, lane, head, first, at.k, k);
  TileScales sc = scales_of(cache, head, at.v);
  load_values<D>(cache, lane, head, first, at.v, v);
  asm volatile("");                                        // (these loads and the loop's own must not become one at its head: the compiler then copies all that it carries, and spills)
  // With 32 rows and e4m3 the registers are full: what follows from the lane is formed at every tile (64 sequences of up to 16384 tokens, 5 new: 177 us, else 181; int8 157 without, 162 with).
  // With 128 channels some 24 to 29 registers lie in memory all the same: the second part of the probabilities took their place.
  auto form_lane = [&] { return NB > 1 && Fmt == kE4m3 ? lane_id() : lane; };
  bool noted = false;
  int kept = 0;                                            // tiles in the ring, the last of them at hand
  auto flush = [&](int last) {
    const int lots = score_floats(score_rows) / 256;       // of 1 KB a tile
    wave_exchange();
    for (int t = 0; t < kept; ++t) {
      float* const to = scores + (int64_t)(last - (kept - 1 - t) * step) * (256 * lots) + 4 * lane;
      for (int x = 0; x < lots; ++x) *reinterpret_cast<f32x4*>(to + 256 * x) = *reinterpret_cast<const f32x4*>(ring + 256 * (t * lots + x) + 4 * lane);
    }
    wave_exchange();
  };
  // (The last tile apart: loads under a condition would all be waited for where it ends.)
  auto tile = [&](int i, auto more) {
    f32x4 s[NB][4];
    scores_of<D, Fmt>(k, q, s);
    TileScales sc_next = sc;
    TilePages at_next = at;
    if constexpr (more) {
      const int lane = form_lane();
      at_next = pages_of(cache, lane, next, len, i + step);
      load_keys<D>(cache, lane, head, i + step, at_next.k, k);
      sc_next = scales_of(cache, head, at_next.v);
      next = ask_pages(cache, table, lane, len, i + 2 * step);
    }
    const float c = scale * sc.k;
    const bool full = i * kTile + kTile - 1 <= all_see && !__ballot(at.v < 0);
    if (!full) {
      const int key0 = i * kTile + 16 * g;
#pragma unroll
      for (int b = 0; b < NB; ++b) mask_scores(s[b], at.v < 0 ? -1 : last_tok[b] - key0);
      clear_hidden<D, Fmt>(v, at.v < 0 ? 0 : len - key0, key0, first_nan, noted);
    }
    if constexpr (Scored) {
      if (n < score_rows) {
        float* const to = ring + kept * score_floats(score_rows) + score_at(n) + 16 * g;
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4*>(to + 64 * j) = s[0][j] * c;
      }
      ++kept;
    }
    // Probabilities go to the product in two parts, bf16 and what that leaves of them: the memory bounds this, and the matrix units have the time.  512 tokens, 4 heads: O is off by 0.0016 to
    // 0.0018 of its norm, its own rounding; with the first part alone by 0.0018 to 0.0025.  It takes 1 % more time over long tables, 3 to 7 % with up to 1000 tokens.
    bf16x8 p[NB][2], rest[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      raise_maximum<D>(s[b], c, r[b].o, r[b].m, r[b].l);
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][j / 4][j % 4], c, -r[b].m)), x = e * sc.v;
        r[b].l += e;
        p[b][j / 8][j % 8] = (__bf16)x;
        rest[b][j / 8][j % 8] = (__bf16)(x - (float)p[b][j / 8][j % 8]);
      }
    }
#pragma unroll
    for (int d = 0; d < D / 16; ++d) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bf16x8 x = decode8<Fmt>(v[d][2 * h], v[d][2 * h + 1]);
#pragma unroll
        for (int b = 0; b < NB; ++b) r[b].o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, rest[b][h], r[b].o[d], 0, 0, 0);
#pragma unroll
        for (int b = 0; b < NB; ++b) r[b].o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, p[b][h], r[b].o[d], 0, 0, 0);
      }
      if (Fmt == kInt8 || NB > 1) __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (more) {
      load_values<D>(cache, form_lane(), head, i + step, at_next.v, v);
      at = at_next;
      sc = sc_next;
    }
    if constexpr (Scored)
      if (!more || (kept + 1) * score_floats(score_rows) > kRing) {
        flush(i);
        kept = 0;
      }
  };
  int i = first;
  for (; i + step < end; i += step) tile(i, std::true_type{});
  tile(i, std::false_type{});
  if (Fmt == kE4m3 && noted) {
    wave_exchange();
#pragma unroll
    for (int d = 0; d < D / 16; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int first_bad = first_nan[16 * d + 4 * g + j];
#pragma unroll
        for (int b = 0; b < NB; ++b) r[b].o[d][j] = first_bad <= last_tok[b] ? NAN : r[b].o[d][j];
      }
    wave_exchange();
  }
}

}  // namespace fcp
