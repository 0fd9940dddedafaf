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
#include "fcp_cache_many.h"

namespace fcp {
namespace {

// kNB: blocks of 16 rows of a wave.
template <int D, int Fmt, bool Short, int kNB>
__global__ __launch_bounds__(256, 2) void attn_rows_kernel(AttnArgs a) {
  constexpr int kRows = 64 * kNB;
  extern __shared__ __align__(256) unsigned char lds[];    // two stages
  __shared__ float key_scale[4][4];
  __shared__ int32_t live[4][4], first_nan[2][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const RowsLane at_lane = rows_lane<D>(lane, wave);
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
      walk_rows<D, Fmt, kNB>(a.c, a.scale, a.s.pages + (int64_t)seq * a.s.max_pages, head, z.len, t0, t_end, q, last, all_see, o, m, l, lane, wave, at_lane, lds, key_scale, live, first_nan, parity);
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
