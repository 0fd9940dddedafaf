// Attention over the cache for many rows: what a block does with the tiles of a piece (csrc/fcp_cache_attn_rows.hip says how the work is laid out and why).
#pragma once
#include "fcp_cache_attn.h"

namespace fcp {

// LDS of a stage: keys as rows of D channels, values as rows (channels) of 64 keys, in chunks of 8 bf16 whose places in a row are permuted so that what is read or written at once
// lies on different banks.  That is 16 lanes, but not neighbours: 0 to 3 and 12 to 15 of one group of 16 with 4 to 11 of the next, so both groups' chunks count.  Values: chunk g + 4 u
// holds keys 16 g + 8 u and on (in the order of the keys two lanes met on every bank).
template <int D>
struct Stage {
  static constexpr int kKeyRow = 2 * D, kValueRow = 2 * kTile, kKeys = kTile * kKeyRow, kBytes = kKeys + D * kValueRow;
  static constexpr int kGroupBit = D == 128 ? 6 : 5;       // key_mix's part that comes from the group of 16 keys, in bytes
  // an operand's rows are 16 a + 4 i + b, a and b from 0 to 3: with 128 channels a row is a whole bank cycle, with 64 two rows are
  static __device__ int key_mix(int row) { return D == 128 ? ((row >> 4) & 3) * 4 + (row & 3) : ((row >> 4) & 3) * 2 + ((row >> 1) & 1); }
  static __device__ int value_mix(int ch) { return (ch >> 1) & 7; }
  static __device__ int key_at(int row, int chunk) { return row * kKeyRow + ((chunk ^ key_mix(row)) << 4); }
  static __device__ int value_at(int ch, int chunk) { return kKeys + ch * kValueRow + ((chunk ^ value_mix(ch)) << 4); }
};

// Four codes as bf16, times their scale, a power of two, or not: exact.
template <int Fmt, bool Scaled>
__device__ inline void decode4(uint32_t w, float scale, bf16x8& to, int at) {
  bf16x2 lo, hi;
  if constexpr (Fmt == kE4m3) {
    lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, Scaled ? scale : 1.f, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, Scaled ? scale : 1.f, true);
  } else {
    f32x2 f = decode_half<Fmt, false>(w), g = decode_half<Fmt, true>(w);
    if (Scaled) f = f32x2{f[0] * scale, f[1] * scale}, g = f32x2{g[0] * scale, g[1] * scale};
    lo = bf16x2{(__bf16)f[0], (__bf16)f[1]};
    hi = bf16x2{(__bf16)g[0], (__bf16)g[1]};
  }
  to[at] = lo[0];
  to[at + 1] = lo[1];
  to[at + 2] = hi[0];
  to[at + 3] = hi[1];
}

// A wave's share of a tile, D / 64 times: 64 D / 256 bytes of one group of 16 keys and as many of the group's values, which lie in one run each, 16 a lane.  Page, scales and
// sizes are the same for the whole wave, so they travel in scalar registers.
typedef const int32_t __attribute__((address_space(4)))* scalar_int;
typedef const float __attribute__((address_space(4)))* scalar_float;
__device__ inline scalar_int as_scalar(const int32_t* p) { return (scalar_int)(uintptr_t)p; }
__device__ inline scalar_float as_scalar(const float* p) { return (scalar_float)(uintptr_t)p; }

template <int D>
struct Share {
  u32x4 w[D / 64];
  float scale[D / 64];
  int live[D / 64];                    // of the 16 keys, those that are cached tokens (0: the page is not there)
};
// group of 16 keys, and the wave's place in it (in lots of 64 times 16 bytes)
template <int D> __device__ inline int group_of(int wave, int i) { return D == 128 ? wave / 2 + 2 * i : wave; }
template <int D> __device__ inline int lot_of(int wave) { return D == 128 ? wave & 1 : 0; }

// Pages that hold the wave's share of a tile, -1 where there is none; asked for a step before the share is, so that nobody waits for the one to ask for the other.
template <int D>
struct Pages { int32_t of[D / 64]; };
template <int D>
__device__ inline void load_pages(const CacheView& c, const int32_t* table, int len, int tile, int wave, Pages<D>& pages) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const int key = tile * kTile + kGroup * group_of<D>(wave, i);
    const int32_t page = as_scalar(table)[min(key, len - 1) >> c.log_page];        // (len is at most what the table holds)
    pages.of[i] = key < len && (uint32_t)page < (uint32_t)c.n_pages ? page : -1;
  }
}
// codes, scales: of the cache's keys, or of its values (a group of 16 tokens is one run of 16 D bytes in both).  Where there is no page the pool's first is read.
template <int D>
__device__ inline void load_share(const CacheView& c, const uint8_t* codes, const float* scales, const Pages<D>& pages, int head, int len, int tile, int wave, Share<D>& s) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const int key = tile * kTile + kGroup * group_of<D>(wave, i);
    const int64_t block = block_of(c, max(pages.of[i], 0), head), at = (block * c.page + (key & (c.page - 1))) * D + 1024 * lot_of<D>(wave);
    s.live[i] = pages.of[i] < 0 ? 0 : min(len - key, kGroup);
    s.scale[i] = as_scalar(scales)[block];
    s.w[i] = *reinterpret_cast<const u32x4*>(codes + at + 16 * (int)(threadIdx.x & 63));
  }
}

// The scale of a page that is not there is whatever the pool's first page holds, and 0 * NaN is NaN: 1 takes its place.  (Where the share is used: done where it is asked for this would wait
// for the load.  64 sequences of up to 16384 tokens, 16 new each, int8: 216 us, 228 there.)
template <int D>
__device__ inline void settle_scales(Share<D>& s) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i) s.scale[i] = s.live[i] ? s.scale[i] : 1.f;
}

// partly: some row of the block does not see the whole tile.  Its product with a NaN value would be NaN too, so zero takes that place, and the first such token of each channel is
// noted in first_nan: the rows that see it get their NaN at the item's end.
template <int D>
__device__ inline void without_nan(Share<D>& s, int wave, int32_t* first_nan, int first_key) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t nan = ((s.w[i][w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
      const int at = 4 * w + (__builtin_ctz(nan) >> 3);
      if (nan && at < s.live[i]) atomicMin(first_nan + 64 * lot_of<D>(wave) + (threadIdx.x & 63), first_key + kGroup * group_of<D>(wave, i) + at);
      s.w[i][w] &= ~((nan >> 7) * 0xffu);
    }
}
// Word i of a share, 0 to D / 16 - 1, on its way into LDS (half: what it shares a chunk with).
template <int D, int Fmt, bool Values>
__device__ inline void store_word(const Share<D>& s, int i, int wave, int place, unsigned char* stage, bf16x8& half) {
  typedef bf16x8 __attribute__((may_alias)) chunk;
  uint32_t w = s.w[i / 4][i % 4];
  if (Values) {                                            // codes past the last token are whatever the page holds, and 0 * NaN is NaN: they become zeros
    const int n = min(max(s.live[i / 4] - 4 * (i % 4), 0), 4);
    w &= (uint32_t)((1ull << (8 * n)) - 1);
  }
  decode4<Fmt, Values>(w, s.scale[i / 4], half, 4 * (i % 2));
  if (i % 2 == 0) return;
  const int g = group_of<D>(wave, i / 4), u = i / 2 % 2;
  place = fresh(place);                                    // (the compiler would keep the addresses that follow from it in registers, and spill them)
  const int at = Values ? place ^ (g << 4 | u << 6) : (place ^ (g << Stage<D>::kGroupBit | u << 4)) + kGroup * g * Stage<D>::kKeyRow;
  *reinterpret_cast<chunk*>(stage + at) = half;
}

// Products whose operands come from LDS, N operands: some are on their way while the products of those before run.  (Left alone the compiler asks for an operand when it is due, and waits.)
constexpr int kAhead = 4;
template <int N, typename Read, typename Multiply>
__device__ inline void stream_operands(Read read, Multiply multiply) {
  bf16x8 x[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) x[i] = read(i);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    multiply(i, x[i % kAhead]);
    if (i + kAhead < N) x[i % kAhead] = read(i + kAhead);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Where the lane's operands and codes lie in a stage.  The chunk's number only flips bits below a row's size, so what steps through chunks is an exclusive or with a constant.
struct RowsLane { int key_operand, value_operand, key_place, value_place; };
template <int D>
__device__ inline RowsLane rows_lane(int lane, int wave) {
  const int n = lane & 15, g = lane >> 4, mine = 64 * lot_of<D>(wave) + lane;
  return {Stage<D>::key_at(16 * (n >> 2) + (n & 3), g), Stage<D>::value_at(n, g), Stage<D>::key_at(mine / (D / 16), 2 * (mine % (D / 16))), Stage<D>::value_at(mine, 0)};
}

// In LDS beside the two stages: scales of the keys and cached tokens, [tile][group of 16 keys], and the first NaN of each channel, for this item and the next.
// Tiles t0 .. t_end - 1 (at least one) for kNB blocks of 16 rows of every wave.  last: last token that the lane's row sees; all of the block's rows see the tokens up to all_see.
// Rest: what the rounding of probabilities to bf16 leaves of them enters the product with V too (64 samples of a prompt of up to 16384 tokens, 256 rows: O is off by 0.0016 of its norm, its own
// rounding, in 59 us; without 0.0020 to 0.0021, 50).
template <int D, int Fmt, int kNB, bool Rest = false>
__device__ __forceinline__ void walk_rows(const CacheView& c, float scale, const int32_t* table, int head, int len, int t0, int t_end, const bf16x8 (&q)[kNB][D / 32], const int (&last)[kNB], int all_see,
                                 f32x4 (&o)[kNB][D / 16], float (&m)[kNB], float (&l)[kNB], int lane, int wave, const RowsLane at_lane, unsigned char* lds, float (&key_scale)[4][4],
                                 int32_t (&live)[4][4], int32_t (&first_nan)[2][D], int parity) {
  typedef bf16x8 __attribute__((may_alias)) chunk;
  const int g = lane >> 4;
  // Tile t's scores are formed a step ahead, so that its exponentials and the products for the next scores are one stream of instructions, and so are its product with the values
  // and the conversion of codes: no pipe waits for another.  Step t writes the keys of tile t + 2 and the values of tile t + 1 where those of tiles t and t - 1 lay.
  Share<D> keys, values;
  Pages<D> ahead = {}, at_hand;                            // of tiles t + 3 and t + 2 in step t
  auto ask_pages = [&](int t) {
    at_hand = ahead;
    load_pages<D>(c, table, len, t, wave, ahead);
  };
  auto ask_keys = [&](int t) { load_share<D>(c, c.k, c.k_scale, ahead, head, len, t, wave, keys); };
  auto ask_values = [&](int t) { load_share<D>(c, c.v, c.v_scale, at_hand, head, len, t, wave, values); };
  auto stage_of = [&](int t) { return lds + ((t - t0) & 1) * Stage<D>::kBytes; };
  auto tidy = [&](int t) {
    if (Fmt == kE4m3 && t * kTile + kTile - 1 > all_see) without_nan<D>(values, wave, first_nan[parity], t * kTile);
  };
  auto note_live = [&](int t) {
    settle_scales<D>(keys);
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
      if (lane == 0) live[t & 3][group_of<D>(wave, i)] = keys.live[i], key_scale[t & 3][group_of<D>(wave, i)] = keys.scale[i];
  };
  auto store_keys = [&](int t) {
    bf16x8 half;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) store_word<D, Fmt, false>(keys, i, wave, at_lane.key_place, stage_of(t), half);
    note_live(t);
  };
  ask_pages(t0);
  ask_keys(t0);
  ask_pages(t0 + 1);
  ask_values(t0);
  __syncthreads();                                     // (the stages of the item before have been read)
  if (Fmt == kE4m3 && threadIdx.x < D) first_nan[parity ^ 1][threadIdx.x] = INT32_MAX;
  store_keys(t0);
  ask_keys(t0 + 1);
  tidy(t0);
  settle_scales<D>(values);
  bf16x8 half;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) store_word<D, Fmt, true>(values, i, wave, at_lane.value_place, stage_of(t0), half);
  store_keys(t0 + 1);
  ask_pages(t0 + 2);
  ask_keys(t0 + 2);
  ask_values(t0 + 1);
  __syncthreads();
  // 16 keys after the other: their scores take the registers that the exponentials of as many leave
  auto scores = [&](int t, f32x4 (&s)[kNB][4], auto meanwhile) {
    const int k0 = fresh(at_lane.key_operand);
    constexpr int kSteps = D / 32;
    stream_operands<D / 8>([&](int i) { return *reinterpret_cast<const chunk*>(stage_of(t) + (k0 ^ (i % kSteps << 6)) + 4 * (i / kSteps) * Stage<D>::kKeyRow); },
                           [&](int i, bf16x8 k) {
#pragma unroll
                             for (int b = 0; b < kNB; ++b) {
                               const f32x4 zero = {0, 0, 0, 0};
                               s[b][i / kSteps] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[b][i % kSteps], i % kSteps == 0 ? zero : s[b][i / kSteps], 0, 0, 0);
                             }
                             meanwhile(i);
                           });
  };
  auto step = [&](int t, f32x4 (&s)[kNB][4], f32x4 (&s_next)[kNB][4]) {
    tidy(t + 1);
    ask_pages(t + 3);
    const int live_here = live[t & 3][g];
    const float to_exponent = scale * key_scale[t & 3][g];
    const bool full = t * kTile + kTile - 1 <= all_see && !__ballot(live_here < kGroup);
    int sees[kNB];
#pragma unroll
    for (int b = 0; b < kNB; ++b) sees[b] = min(last[b] - t * kTile - 16 * g, live_here - 1);
    if (!full)
#pragma unroll
      for (int b = 0; b < kNB; ++b) mask_scores(s[b], sees[b]);
#pragma unroll
    for (int b = 0; b < kNB; ++b) raise_maximum<D>(s[b], to_exponent, o[b], m[b], l[b]);
    __syncthreads();
    bf16x8 p[kNB][2], rest[kNB][2];
    scores(t + 1, s_next, [&](int i) {
#pragma unroll
      for (int j = 128 * kNB / D * i; j < 128 * kNB / D * (i + 1); ++j) {
        const int b = j / 16, x = j % 16;
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][x / 4][x % 4], to_exponent, -m[b]));
        l[b] += e;
        p[b][x / 8][x % 8] = (__bf16)e;
        if constexpr (Rest) rest[b][x / 8][x % 8] = (__bf16)(e - (float)p[b][x / 8][x % 8]);
      }
      // (left alone the compiler adds them up where the sum is due, and keeps them all until then)
#pragma unroll
      for (int b = 0; b < kNB; ++b) asm volatile("" : "+v"(l[b]));
    });
    __builtin_amdgcn_sched_barrier(0);
    settle_scales<D>(values);
    const int v0 = fresh(at_lane.value_operand);
    stream_operands<D / 8>([&](int i) { return *reinterpret_cast<const chunk*>(stage_of(t) + (v0 ^ (i / 4 % 2 << 6)) + 16 * (i / 8 * 4 + i % 4) * Stage<D>::kValueRow); },
                           [&](int i, bf16x8 v) {
                             auto add = [&](const bf16x8 (&x)[kNB][2]) {
#pragma unroll
                               for (int b = 0; b < kNB; ++b) {
                                 f32x4& sum = o[b][i / 8 * 4 + i % 4];
                                 sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, x[b][i / 4 % 2], sum, 0, 0, 0);
                               }
                             };
                             if constexpr (Rest) add(rest);
                             add(p);
                             if (i < D / 16) store_word<D, Fmt, false>(keys, i, wave, at_lane.key_place, stage_of(t), half);
                             else store_word<D, Fmt, true>(values, i - D / 16, wave, at_lane.value_place, stage_of(t + 1), half);
                           });
    note_live(t + 2);
    ask_keys(t + 3);
    ask_values(t + 2);
  };
  f32x4 s[2][kNB][4];
  scores(t0, s[0], [](int) {});
  for (int t = t0; t < t_end; t += 2) {
    step(t, s[0], s[1]);
    if (t + 1 < t_end) step(t + 1, s[1], s[0]);
  }
  if (Fmt == kE4m3)
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int first = first_nan[parity][16 * i + 4 * g + j];
#pragma unroll
        for (int b = 0; b < kNB; ++b) o[b][i][j] = first <= last[b] ? NAN : o[b][i][j];
      }
}

}  // namespace fcp
