// Attention over the paged 8-bit cache for many rows: pieces of prompts, or several new tokens of many query heads.
//
// A block takes 128 rows (or 64, where there are no more) of a KV head's group at a time, a wave 32 (16) of them, against tiles of 64 keys.  The products and the exponentials bound it (4 D flops a pair; an exponential
// takes as long as 64 flops of the matrix units per lane), so the codes must not become bf16 in every wave: a tile's codes come in whole lines, 32 a thread, become bf16 (exact) and
// go to LDS, from which the waves read the operands of the 16 x 16 x 32 instructions, each for all of its rows.  Operand rows straight from memory would be requests of 16 bytes
// a lane, a quarter of a line's rate, in every wave.  The keys' scale is taken with the scores, the values' with the codes.
// A step has two streams: the next tile's scores with this tile's exponentials, and this tile's product with the values with the conversion of codes for the tiles after; the matrix
// units and the others work at once, and operands from LDS are asked for four ahead.  One barrier a step.  Two blocks per CU: a wave has 256 registers, all in use.
// Pieces of 512 tokens over up to 16385, 2 sequences, 40 query heads on 8, 128 channels, 193 Gflop: 239 to 244 us with e4m3 (11 of them the merge), 270 with int8, whose codes take
// three times as many instructions; with score, exponentials and product one after the other, each operand asked for when it is due, 277 and 300 where this took 244 and 280 then.  Counted:
// the matrix units work 38 % of the CUs' time, 22 % of a wave's time are waits.  A large matrix product runs at 1213 Tflop/s here, this at 800.
// Probabilities enter the product with V as one bf16 (O is off by 0.0021 of its norm, by 0.0017 with fp32 throughout and one rounding).  In two parts, as with few rows, the products bound it still
// more: the pieces of 512 306 us instead of 240 with e4m3, 332 instead of 269 with int8; 64 rows, 64 sequences of up to 16384 tokens, 223 instead of 198, 243 instead of 215.
// Keys and rows are laid on the matrix as in the kernel for few rows: a lane ends with the scores of 16 neighbouring keys, which is the operand of the product with V.
#include "fcp_cache_attn.h"

namespace fcp {
namespace {

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
__device__ inline void load_pages(const AttnArgs& a, const int32_t* table, int len, int tile, int wave, Pages<D>& pages) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const int key = tile * kTile + kGroup * group_of<D>(wave, i);
    const int32_t page = as_scalar(table)[min(key, len - 1) >> a.c.log_page];        // (len is at most what the table holds)
    pages.of[i] = key < len && (uint32_t)page < (uint32_t)a.c.n_pages ? page : -1;
  }
}
// codes, scales: of the cache's keys, or of its values (a group of 16 tokens is one run of 16 D bytes in both).  Where there is no page the pool's first is read.
template <int D>
__device__ inline void load_share(const AttnArgs& a, const uint8_t* codes, const float* scales, const Pages<D>& pages, int head, int len, int tile, int wave, Share<D>& s) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const int key = tile * kTile + kGroup * group_of<D>(wave, i);
    const int64_t block = block_of(a.c, max(pages.of[i], 0), head), at = (block * a.c.page + (key & (a.c.page - 1))) * D + 1024 * lot_of<D>(wave);
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

// kNB: blocks of 16 rows of a wave.
template <int D, int Fmt, bool Short, int kNB>
__global__ __launch_bounds__(256, 2) void attn_rows_kernel(AttnArgs a) {
  constexpr int kRows = 64 * kNB;
  typedef bf16x8 __attribute__((may_alias)) chunk;
  extern __shared__ __align__(256) unsigned char lds[];    // two stages
  __shared__ float key_scale[4][4];                        // [tile][group of 16 keys]
  __shared__ int32_t live[4][4], first_nan[2][D];          // (the latter for this item and the next)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  // Where the lane's operands and codes lie in a stage.  The chunk's number only flips bits below a row's size, so what steps through chunks is an exclusive or with a constant.
  const int key_first = 16 * (n >> 2) + (n & 3), key_operand = Stage<D>::key_at(key_first, g), value_operand = Stage<D>::value_at(n, g);
  const int mine = 64 * lot_of<D>(wave) + lane, key_place = Stage<D>::key_at(mine / (D / 16), 2 * (mine % (D / 16))), value_place = Stage<D>::value_at(mine, 0);
  const int32_t me = blockIdx.x;
  constexpr int kLead = Short ? kWhole : kItemLead;
  const Line line = find_on_line<kLead>(a.s, a.c, a.group, kRows, a.blocks, me);
  Divided divided = {};
  int32_t at = 0, end = 0;
  if (line.seq >= 0) {
    at = line.begin(me);
    end = line.begin(me + 1);
  }
  int seq = line.seq;
  int32_t base = line.before;
  SeqSizes z = line.z;
  if (Fmt == kE4m3 && threadIdx.x < D) first_nan[1][threadIdx.x] = INT32_MAX;
  int parity = 1;                                          // of the items that see a tile
  while (at < end) {
    while (at >= base + cost_of<kLead>(z, a.c.hkv, a.group, kRows)) {  // the next sequence with rows
      base += cost_of<kLead>(z, a.c.hkv, a.group, kRows);
      z = seq_sizes(a.s, ++seq, a.c.page);
    }
    const int tiles = tiles_of(z.len), all_rows = z.n * a.group, row_blocks = (all_rows + kRows - 1) / kRows;
    const int places = places_of<kLead>(z.len), item = (at - base) / places, from = (at - base) % places;
    const Piece piece = piece_of<kLead>(tiles, from, end - at);
    const int head = item / row_blocks, rb = item % row_blocks, t0 = piece.first, t1 = piece.last;
    const int32_t item0 = at - from;
    at += piece.places;
    if (t0 == t1) continue;                                // (the item's lead alone)

    bf16x8 q[kNB][D / 32];
    f32x4 o[kNB][D / 16];
    float m[kNB], l[kNB];
    int last[kNB];                                         // last token that the lane's row sees
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
      const int row = rb * kRows + (wave * kNB + b) * 16 + n;
      const bool there = row < all_rows;
      const int tok = there ? row / a.group : 0;
      last[b] = there ? z.len - z.n + tok : -1;
      const __bf16* x = a.q + (int64_t)(z.row0 + tok) * a.q_row + (head * a.group + (there ? row % a.group : 0)) * D + 8 * g;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        const bf16x8 w = *reinterpret_cast<const bf16x8*>(x + 32 * j), zero = {};
        q[b][j] = there ? w : zero;
      }
      m[b] = kLow;
      l[b] = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) o[b][i] = f32x4{0, 0, 0, 0};
    }
    // all of the block's rows see the tokens up to all_see; tiles from t_end on nobody sees
    const int rows = min(all_rows - rb * kRows, kRows), all_see = z.len - z.n + rb * kRows / a.group;
    const int seen = z.len - z.n + (rb * kRows + rows - 1) / a.group;
    const int t_end = min(t1, seen < 0 ? 0 : seen / kTile + 1);
    if (t0 < t_end) {
      // Tile t's scores are formed a step ahead, so that its exponentials and the products for the next scores are one stream of instructions, and so are its product with the values
      // and the conversion of codes: no pipe waits for another.  Step t writes the keys of tile t + 2 and the values of tile t + 1 where those of tiles t and t - 1 lay.
      Share<D> keys, values;
      const int32_t* const table = a.s.pages + (int64_t)seq * a.s.max_pages;
      Pages<D> ahead = {}, at_hand;                            // of tiles t + 3 and t + 2 in step t
      auto ask_pages = [&](int t) {
        at_hand = ahead;
        load_pages<D>(a, table, z.len, t, wave, ahead);
      };
      auto ask_keys = [&](int t) { load_share<D>(a, a.c.k, a.c.k_scale, ahead, head, z.len, t, wave, keys); };
      auto ask_values = [&](int t) { load_share<D>(a, a.c.v, a.c.v_scale, at_hand, head, z.len, t, wave, values); };
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
        for (int i = 0; i < D / 16; ++i) store_word<D, Fmt, false>(keys, i, wave, key_place, stage_of(t), half);
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
      for (int i = 0; i < D / 16; ++i) store_word<D, Fmt, true>(values, i, wave, value_place, stage_of(t0), half);
      store_keys(t0 + 1);
      ask_pages(t0 + 2);
      ask_keys(t0 + 2);
      ask_values(t0 + 1);
      __syncthreads();
      // 16 keys after the other: their scores take the registers that the exponentials of as many leave
      auto scores = [&](int t, f32x4 (&s)[kNB][4], auto meanwhile) {
        const int k0 = fresh(key_operand);
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
        const float c = a.scale * key_scale[t & 3][g];
        const bool full = t * kTile + kTile - 1 <= all_see && !__ballot(live_here < kGroup);
        int sees[kNB];
#pragma unroll
        for (int b = 0; b < kNB; ++b) sees[b] = min(last[b] - t * kTile - 16 * g, live_here - 1);
        if (!full)
#pragma unroll
          for (int b = 0; b < kNB; ++b) mask_scores(s[b], sees[b]);
#pragma unroll
        for (int b = 0; b < kNB; ++b) raise_maximum<D>(s[b], c, o[b], m[b], l[b]);
        __syncthreads();
        bf16x8 p[kNB][2];
        scores(t + 1, s_next, [&](int i) {
#pragma unroll
          for (int j = 128 * kNB / D * i; j < 128 * kNB / D * (i + 1); ++j) {
            const int b = j / 16, x = j % 16;
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][x / 4][x % 4], c, -m[b]));
            l[b] += e;
            p[b][x / 8][x % 8] = (__bf16)e;
          }
          // (left alone the compiler adds them up where the sum is due, and keeps them all until then)
#pragma unroll
          for (int b = 0; b < kNB; ++b) asm volatile("" : "+v"(l[b]));
        });
        __builtin_amdgcn_sched_barrier(0);
        settle_scales<D>(values);
        const int v0 = fresh(value_operand);
        stream_operands<D / 8>([&](int i) { return *reinterpret_cast<const chunk*>(stage_of(t) + (v0 ^ (i / 4 % 2 << 6)) + 16 * (i / 8 * 4 + i % 4) * Stage<D>::kValueRow); },
                               [&](int i, bf16x8 v) {
#pragma unroll
                                 for (int b = 0; b < kNB; ++b) {
                                   f32x4& sum = o[b][i / 8 * 4 + i % 4];
                                   sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[b][i / 4 % 2], sum, 0, 0, 0);
                                 }
                                 if (i < D / 16) store_word<D, Fmt, false>(keys, i, wave, key_place, stage_of(t), half);
                                 else store_word<D, Fmt, true>(values, i - D / 16, wave, value_place, stage_of(t + 1), half);
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
      parity ^= 1;
    }
#pragma unroll
    for (int b = 0; b < kNB; ++b) l[b] = sum_over_groups(l[b]);

    const bool whole = t0 == 0 && t1 == tiles;
    if (t0 == 0 && !whole) divided = {line.owner(item0 + kItemLead + tiles - 1) - me + 1, z.row0, all_rows, head, rb, {}};
    float* const slot = a.part + (int64_t)(2 * me + (t0 == 0 ? 1 : 0)) * slot_floats(D, kRows);
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
      const int lr = (wave * kNB + b) * 16 + n, row = rb * kRows + lr;
      if (!whole) {                                        // sums as they lie in the registers: the merge divides them the same way
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(slot + (((wave * kNB + b) * (D / 16) + i) * 64 + lane) * 4) = o[b][i];
        if (g == 0) { slot[kRows * D + lr] = m[b]; slot[kRows * (D + 1) + lr] = l[b]; }
      } else if (row < all_rows) {
        const int tok = z.row0 + row / a.group, h = head * a.group + row % a.group;
        const float inv = l[b] == 0.f ? 0.f : 1.f / l[b];
        __bf16* const y = a.o + ((int64_t)tok * a.hq + h) * D + 4 * g;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          bf16x4 w;
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = (__bf16)(o[b][i][j] * inv);
          *reinterpret_cast<bf16x4*>(y + 16 * i) = w;
        }
        if (g == 0) a.lse[(int64_t)h * a.s.n_rows + tok] = l[b] == 0.f ? -INFINITY : (m[b] + __builtin_amdgcn_logf(l[b])) * kLn2;
      }
    }
  }
  if (!Short && threadIdx.x == 0) a.divided[me] = divided;
}

// Divided items: a block per (block in which one begins, 16 rows), four channels of a row a thread, in the order in which the sums lie.
template <int D, int kRows>
__global__ __launch_bounds__(256) void attn_rows_merge_kernel(AttnArgs a) {
  constexpr int kFloats = slot_floats(D, kRows);
  const int me = blockIdx.x, part = blockIdx.y, lane = threadIdx.x & 63;
  const Divided d = a.divided[me];
  const int lr = part * 16 + (lane & 15), row = d.row_block * kRows + lr;
  if (d.pieces == 0 || row >= d.all_rows) return;
  float m = kLow;
#pragma unroll 4
  for (int p = 0; p < d.pieces; ++p) m = fmaxf(m, piece_slot(a, me, p, kFloats)[kRows * D + lr]);
  f32x4 o[D / 64];
#pragma unroll
  for (int i = 0; i < D / 64; ++i) o[i] = f32x4{0, 0, 0, 0};
  float l = 0.f;
#pragma unroll 4
  for (int p = 0; p < d.pieces; ++p) {
    const float* s = piece_slot(a, me, p, kFloats);
    const float f = __builtin_amdgcn_exp2f(s[kRows * D + lr] - m);
    l += f * s[kRows * (D + 1) + lr];
#pragma unroll
    for (int i = 0; i < D / 64; ++i) o[i] += f * *reinterpret_cast<const f32x4*>(s + ((part * (D / 16) + 4 * i + (int)(threadIdx.x >> 6)) * 64 + lane) * 4);
  }
  const int tok = d.row0 + row / a.group, h = d.head * a.group + row % a.group;
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    bf16x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (__bf16)(o[i][j] * inv);
    *reinterpret_cast<bf16x4*>(a.o + ((int64_t)tok * a.hq + h) * D + 16 * (4 * i + (threadIdx.x >> 6)) + 4 * (lane >> 4)) = w;
  }
  if (threadIdx.x < 16) a.lse[(int64_t)h * a.s.n_rows + tok] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

template <int D, int Fmt>
int launch(const AttnArgs& a, int rows, bool whole, hipStream_t st) {
  constexpr int kLds = 2 * Stage<D>::kBytes;
  static std::atomic<uint64_t> raised[4];
  const bool half = rows == kManyRows / 2;
  auto kernel = half ? (whole ? attn_rows_kernel<D, Fmt, true, 1> : attn_rows_kernel<D, Fmt, false, 1>) : whole ? attn_rows_kernel<D, Fmt, true, 2> : attn_rows_kernel<D, Fmt, false, 2>;
  if (kLds > 64 * 1024 - 1024)
    if (int rc = raise_lds_limit(reinterpret_cast<const void*>(kernel), kLds, raised[2 * half + whole])) return rc;
  kernel<<<dim3(kBlocks), dim3(256), kLds, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  if (!whole) {
    auto merge = half ? attn_rows_merge_kernel<D, kManyRows / 2> : attn_rows_merge_kernel<D, kManyRows>;
    merge<<<dim3(kBlocks, (unsigned)(rows / 16)), dim3(256), 0, st>>>(a);
    FCP_HIP_CHECK(hipGetLastError());
  }
  return FCP_OK;
}

}  // namespace

int launch_attn_rows(const AttnArgs& a, int head_dim, int format, int rows, bool whole, hipStream_t st) {
  if (head_dim == 128) return format == kE4m3 ? launch<128, kE4m3>(a, rows, whole, st) : launch<128, kInt8>(a, rows, whole, st);
  return format == kE4m3 ? launch<64, kE4m3>(a, rows, whole, st) : launch<64, kInt8>(a, rows, whole, st);
}

}  // namespace fcp
