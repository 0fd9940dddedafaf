// What the kernels of attention over the cache share (csrc/fcp_cache_attn.hip: few rows; csrc/fcp_cache_attn_rows.hip: many): the line of tiles, the softmax of a tile, the
// slots of divided items.
#pragma once
#include "fcp_cache.h"

namespace fcp {

constexpr int kTile = 64;              // keys of a tile
constexpr int kWaves = 4;              // of a block
constexpr int kBlocks = 512;           // that share the line: two per CU
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
  struct Divided* divided;             // per block: the item that begins in it and goes on in the blocks after it
  float* scores;                       // weigh: 16 x 64 for every place on the line, scaled by log2(e), in the order in which waves hold them; or NULL
  int32_t blocks;                      // that share the line
};

// The line of the tiles of all items, and its division among blocks.  Sequence s has, for every KV head and every block of `rows` rows, all of its tiles (a sequence without
// cached tokens one empty tile, which writes O = 0).  Lead: places before an item's first tile, for what a block does for an item whatever its tiles; kWhole: an item is one place on the
// line, so that it lies in one block.
// Places are 32-bit numbers: the host sees to it that there are at most kMostPlaces.
struct Line {
  int32_t total;                       // places
  int32_t before;                      // those of the sequences before `seq`
  int32_t seq;
  SeqSizes z;                          // of `seq`
  int32_t sharers;                     // blocks that get a share
  // share i begins at i * size + min(i, larger): the first `larger` shares have size + 1 places
  __device__ int32_t size() const { return total / sharers; }
  __device__ int32_t larger() const { return total % sharers; }
  __device__ int32_t begin(int32_t i) const { return i * size() + min(i, larger()); }
  __device__ int32_t owner(int32_t x) const {
    const int32_t q = size(), r = larger(), first = r * (q + 1);
    return x < first ? x / (q + 1) : r + (x - first) / q;
  }
};

__device__ inline int32_t tiles_of(int len) { return max((len + kTile - 1) / kTile, 1); }
constexpr int kWhole = -1;
// Rows, first loads and the waves' meeting take a block about as long as four tiles.  Lead of 0 / 2 / 4 / 8, few rows, int8: 64 sequences of up to 16384 tokens with weights 186 / 181 / 180 / 181 us, of
// up to 4000 47.6 / 44.7 / 43.1 / 45.4, 16 of up to 8000 28.6 / 28.3 / 26.8 / 27.9, 5 of up to 2000 13.9 / 13.3 / 11.0 / 11.0; 64 of 4700 113 each.  0 / 2 / 4 / 6 / 10, many: 30 of up to 4000,
// 40 new tokens 96 / 84 / 85 / 89 / 96, 8 of up to 16000, 100 new 168 / 164 / 165 / 166 / 170; e4m3, 2 of up to 16385, 512 new 248 / 243 / 243 / 244 / 247.
constexpr int kItemLead = 4;
template <int Lead> __device__ inline int32_t places_of(int len) { return Lead == kWhole ? 1 : tiles_of(len) + Lead; }
template <int Lead>
__device__ inline int32_t cost_of(const SeqSizes& z, int hkv, int group, int rows) {
  return z.n == 0 ? 0 : hkv * ((z.n * group - 1) / rows + 1) * places_of<Lead>(z.len);
}

// The sequence that holds the beginning of share `block` (blocks = 0: place `block` itself); seq = -1 if there is none.  Every thread of the block (256, 512) calls; a thread
// looks at a run of sequences, all of which are asked for at once.  At most `blocks` shares, fewer where a share would have fewer than Least places.
// Where cu_seqlens falls, rows would belong to several sequences and there could be more places than the host counted: then there is no work at all.
template <int Lead, int Threads = 256, int Least = Lead == kWhole ? 1 : kLeastTiles>
static __device__ inline Line find_on_line(const SeqView& s, const CacheView& c, int group, int rows, int blocks, int block) {
  __shared__ int32_t sums[Threads / 64];
  __shared__ int32_t found[5];
  const int per = (s.n_seqs + Threads - 1) / Threads, a = min((int)threadIdx.x * per, s.n_seqs), b = min(a + per, s.n_seqs);
  int32_t mine = 0;
  bool falls = false;
  for (int i = a; i < b; ++i) {
    falls |= s.cu[i + 1] < s.cu[i];
    mine += cost_of<Lead>(seq_sizes(s, i, c.page), c.hkv, group, rows);
  }
  falls = __ballot(falls);
  int32_t upto = wave_prefix_sum(mine);
  if ((threadIdx.x & 63) == 63) sums[threadIdx.x >> 6] = falls ? -1 : upto;
  if (threadIdx.x == 0) found[0] = -1;
  __syncthreads();
  Line line = {};
  for (int w = 0; w < Threads / 64; ++w) {
    if (w < (int)(threadIdx.x >> 6)) upto += sums[w];
    line.total += sums[w];
    falls |= sums[w] < 0;
  }
  if (falls) line.total = 0;
  line.sharers = min(blocks, (line.total + Least - 1) / Least);
  int32_t at = upto - mine;            // of the thread's first sequence
  const int32_t x = falls ? -1 : blocks == 0 ? block : block >= line.sharers ? -1 : line.begin(block);
  if (x >= 0 && x >= at && x < upto) {
    for (int i = a; i < b; ++i) {
      const SeqSizes z = seq_sizes(s, i, c.page);
      const int32_t n = cost_of<Lead>(z, c.hkv, group, rows);
      if (x < at + n) {
        found[0] = i;
        found[1] = at;
        found[2] = z.row0;
        found[3] = z.n;
        found[4] = z.len;
        break;
      }
      at += n;
    }
  }
  __syncthreads();
  // (the same for all threads: scalar registers)
  line.seq = __builtin_amdgcn_readfirstlane(found[0]);
  line.before = __builtin_amdgcn_readfirstlane(found[1]);
  line.z = {__builtin_amdgcn_readfirstlane(found[2]), __builtin_amdgcn_readfirstlane(found[3]), __builtin_amdgcn_readfirstlane(found[4])};
  line.total = __builtin_amdgcn_readfirstlane(line.total);
  line.sharers = __builtin_amdgcn_readfirstlane(line.sharers);
  return line;
}

// A block's share of an item, from place `at` on (`from` places after the item's first) to place `end` at most: tiles first .. last - 1, and the places that they and the lead take.
struct Piece { int32_t first, last, places; };
template <int Lead>
__device__ inline Piece piece_of(int32_t tiles, int32_t from, int32_t room) {
  if (Lead == kWhole) return {0, tiles, 1};
  const int32_t n = min(tiles + Lead - from, room);
  return {max(from - Lead, 0), max(from + n - Lead, 0), n};
}

// An item that several blocks work: the block in which it begins says who it is and how many pieces it has; piece p lies in slot 2 (block + p), the first in slot
// 2 block + 1.  pieces = 0: none begins here.
struct Divided { int32_t pieces, row0, all_rows, head, row_block, pad[3]; };
static_assert(sizeof(Divided) == 32, "eight words");

// Floats of a slot: sums [rows][D] (in the kernel's own order), maxima [rows], sums of exponentials [rows].
__host__ __device__ constexpr int slot_floats(int head_dim, int rows) { return rows * (head_dim + 2); }
inline __device__ float* piece_slot(const AttnArgs& a, int block, int piece, int floats) { return a.part + (int64_t)(2 * (block + piece) + (piece == 0 ? 1 : 0)) * floats; }

// Places are 32-bit numbers, and so is the one that a block of the weights' kernel, one of up to 2 kBlocks, steps to past the last.
constexpr int64_t kMostPlaces = INT32_MAX - 2 * kBlocks;

constexpr int kManyRows = 128;         // rows of a block in the kernel for many, or half of them

size_t attn_scratch_bytes(const CacheView& c, int head_dim, int32_t n_seqs, int32_t max_pages, int32_t tq, int32_t hq);       // of fcp_cache_attn without weigh
int launch_attn_rows(const AttnArgs& a, int head_dim, int format, int rows, bool whole, hipStream_t st);

__device__ inline float max_over_groups(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float sum_over_groups(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Of the lane's 16 keys its row sees those up to `last`.
__device__ inline void mask_scores(f32x4 (&s)[4], int last) {
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i / 4][i % 4] = i <= last ? s[i / 4][i % 4] : -INFINITY;
}

// Softmax of one tile and 16 rows, its first part: the running maximum follows the raw scores s (c scales them), and what was summed up so far follows the maximum.  It only grows in steps of
// more than 2^8: probabilities stay below 256, and most tiles leave the sums alone.
template <int D>
__device__ inline void raise_maximum(const f32x4 (&s)[4], float c, f32x4 (&o)[D / 16], float& m, float& l) {
  float top = max3(s[0][0], s[0][1], s[0][2]);
#pragma unroll
  for (int i = 3; i < 15; i += 2) top = max3(top, s[i / 4][i % 4], s[(i + 1) / 4][(i + 1) % 4]);
  top = __builtin_elementwise_maximum(top, s[3][3]) * c;
  if (__ballot(top > m + 8.f)) {
    const float grown = fmaxf(m, max_over_groups(top)), f = __builtin_amdgcn_exp2f(m - grown);
    m = grown;
    l *= f;
#pragma unroll
    for (int d = 0; d < D / 16; ++d) o[d] *= f;
  }
}

}  // namespace fcp
