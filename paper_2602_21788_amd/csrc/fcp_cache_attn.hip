// fcp_cache_attn: attention of the last tokens of every sequence over a paged 8-bit cache, and the sums of the weights that every cached token gets.
//
// O = softmax(scale Q K^T) V, rows of one KV head's whole group together (row r = token r / G, query head r % G of the group), keys in tiles of 64.
// For single tokens the cache's bytes bound it: every code is read once, and everything else has to hide behind that.
//   * S^T = K Q^T with the 16 x 16 x 32 bf16 instructions: the keys are the matrix rows, a query row is a column, so its maximum and sum stay in the lane.
//     Matrix row m of key tile t (of four) is key 16 (m / 4) + 4 t + m % 4 of the 64: then lane (column n, group g) ends with the scores of the 16
//     neighbouring keys 16 g .. 16 g + 15, in order, which is the operand that the product with V needs, without any exchange.
//   * O^T += V^T P^T, P in two bf16 parts: the cache holds values in groups of 16 tokens, a channel's 16 codes together, so a lane's 16 bytes are its channel's codes of its keys.
//   * Codes go from memory to registers in 16-byte loads and become bf16 there (exact); the keys' scale multiplies the scores, the values' scale (a power
//     of two) the probabilities.  The wave needs no barrier in its loop, and LDS only for the scores that it keeps for the weights (a ring of its own).
// All (sequence, KV head, block of rows, key tile) form one line, cut into equal pieces for the blocks: a long sequence is split over many blocks and short ones
// share one, however ragged the lengths, which only the device knows.  The pieces of an item that does not lie in one block meet in a second launch.
// One token over 131072, 32 heads on 8, e4m3, 269 MB: 60 us, 4.5 TB/s, where a large copy reaches 4.9 (the join is 8 of them, mostly its launch); 64 of lengths 819 to 16384, int8: 132 us,
// 5.2 TB/s, with weights 180 (scores go out and come back).
#include "fcp_cache_few.h"

namespace fcp {
namespace {

// Few rows: a block takes 16 NB rows of a KV head at a time, its waves divide the tiles of a piece and join their sums in LDS.
// Short: items are whole.  Scored: scores are kept for the weights (items may be divided).
template <int D, int Fmt, bool Short, bool Scored, int NB>
__global__ __launch_bounds__(256, 2) void attn_kernel(AttnArgs a) {
  static_assert(!(Scored && (Short || NB > 1)), "scores are kept of items on the line of tiles, 16 rows of each");
  constexpr int kRows = 16 * NB;
  constexpr int kLead = Short ? kWhole : kItemLead;
  constexpr int kStride = D + 4;                           // floats of a staged row: rows on different banks
  // a wave's sums for the others, or, before it writes them, its ring of scores
  constexpr int kWaveFloats = Scored ? kRing : kRows * kStride;
  static_assert(kWaveFloats >= kRows * kStride, "the sums fit");
  __shared__ __align__(16) float stage[kWaves * kWaveFloats];
  __shared__ float stage_m[kWaves * kRows], stage_l[kWaves * kRows];
  __shared__ int32_t first_nan[kWaves][Fmt == kE4m3 ? D : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const int32_t me = blockIdx.x;
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
  while (at < end) {
    while (at >= base + cost_of<kLead>(z, a.c.hkv, a.group, kRows)) {      // the next sequence with rows
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

    int last[NB], first_seen = INT32_MAX;                  // last tokens that the lane's rows see; the first of those of all rows
    bf16x8 q[NB][D / 32];
    RowState<D> r[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int my_row = rb * kRows + 16 * b + n;
      const bool live = my_row < all_rows;
      const int my_tok = live ? my_row / a.group : 0;
      last[b] = live ? z.len - z.n + my_tok : -1;
      first_seen = min(first_seen, live ? last[b] : INT32_MAX);
      const __bf16* x = a.q + (int64_t)(z.row0 + my_tok) * a.q_row + (head * a.group + (live ? my_row % a.group : 0)) * D + 16 * g;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        const bf16x8 w = *reinterpret_cast<const bf16x8*>(x + 64 * (j / 2) + 8 * (j % 2)), zero = {};
        q[b][j] = live ? w : zero;
      }
      r[b].m = kLow;
      r[b].l = 0.f;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) r[b].o[i] = f32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) first_seen = min(first_seen, __shfl_xor(first_seen, d));
    // the last tile that any of the rows sees
    const int rows = min(all_rows - rb * kRows, kRows), seen = z.len - z.n + (rb * kRows + rows - 1) / a.group;
    const int t_end = min(t1, seen < 0 ? 0 : seen / kTile + 1);
    float* const scores = Scored ? a.scores + (int64_t)item0 * (16 * kTile) : nullptr;
    walk<D, Fmt, Scored>(a.c, a.scale, a.s.pages + (int64_t)seq * a.s.max_pages, head, z.len, t0 + wave, t_end, kWaves, q, last, first_seen, r, scores, rows, stage + wave * kWaveFloats, first_nan[wave]);
    if constexpr (Scored)                                  // tiles of the piece that nobody sees
      for (int i = max(t_end, t0) + wave; i < t1; i += kWaves)
        for (int j = lane; j < score_floats(rows); j += 64) scores[(int64_t)i * score_floats(rows) + j] = -INFINITY;

    const bool whole = t0 == 0 && t1 == tiles;
    if (t0 == 0 && !whole) divided = {line.owner(item0 + kItemLead + tiles - 1) - me + 1, z.row0, all_rows, head, rb, {}};
    float* const slot = a.part + (int64_t)(2 * me + (t0 == 0 ? 1 : 0)) * slot_floats(D, kRows);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int lr = 16 * b + n;
      r[b].l = sum_over_groups(r[b].l);
      if (g == 0) { stage_m[wave * kRows + lr] = r[b].m; stage_l[wave * kRows + lr] = r[b].l; }
#pragma unroll
      for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(&stage[wave * kWaveFloats + lr * kStride + 16 * i + 4 * g]) = r[b].o[i];
    }
    __syncthreads();
    for (int j = threadIdx.x; j < rows * (D / 4); j += 256) {
      const int lr = j / (D / 4), ch = 4 * (j % (D / 4)), row = rb * kRows + lr;
      float m = kLow, l = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, stage_m[w * kRows + lr]);
      f32x4 o = {0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(stage_m[w * kRows + lr] - m);
        l += f * stage_l[w * kRows + lr];
        o += f * *reinterpret_cast<const f32x4*>(&stage[w * kWaveFloats + lr * kStride + ch]);
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
  }
  if (!Short && threadIdx.x == 0) a.divided[me] = divided;
}

// Pieces p, p + kWaves, ... of a row joined by a wave, N asked for at a time; kCh channels a lane.  What was summed up so far follows the maximum.
template <int D, int kRows, int N>
__device__ inline void join_pieces(const AttnArgs& a, int me, int pieces, int p, int row, float& m, float& l, float (&o)[D / 64]) {
  constexpr int kCh = D / 64, kFloats = slot_floats(D, kRows);
  const int ch = kCh * (threadIdx.x & 63);
  for (; p < pieces; p += N * kWaves) {
    float pm[N], pl[N], po[N][kCh];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float* const s = piece_slot(a, me, min(p + i * kWaves, pieces - 1), kFloats);
      pm[i] = s[kRows * D + row];
      pl[i] = s[kRows * (D + 1) + row];
#pragma unroll
      for (int c = 0; c < kCh; ++c) po[i][c] = s[row * D + ch + c];
    }
    float top = m;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, pm[i]);   // (the last one again where there are no more)
    const float before = __builtin_amdgcn_exp2f(m - top);
    m = top;
    l *= before;
#pragma unroll
    for (int c = 0; c < kCh; ++c) o[c] *= before;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool there = p + i * kWaves < pieces;
      const float f = __builtin_amdgcn_exp2f(pm[i] - m);
      l += there ? f * pl[i] : 0.f;
#pragma unroll
      for (int c = 0; c < kCh; ++c) o[c] += there ? f * po[i][c] : 0.f;
    }
  }
}

// Divided items: blocks_of_item blocks for each block in which one may begin, a row at a time, whose waves divide the pieces.  Everything of eight pieces is asked for at once.
template <int D, int kRows>
__global__ __launch_bounds__(256) void attn_merge_kernel(AttnArgs a, int blocks_of_item) {
  constexpr int kCh = D / 64;
  __shared__ float sum_o[kWaves][D], sum_m[kWaves], sum_l[kWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), me = blockIdx.x / blocks_of_item;
  const Divided d = a.divided[me];
  const int rows = min(d.all_rows - d.row_block * kRows, kRows);
  if (d.pieces == 0) return;
  for (int lr = blockIdx.x % blocks_of_item; lr < rows; lr += blocks_of_item) {
    float m = kLow, l = 0.f, o[kCh] = {};
    if (d.pieces <= kWaves) join_pieces<D, kRows, 1>(a, me, d.pieces, wave, lr, m, l, o);
    else join_pieces<D, kRows, 8>(a, me, d.pieces, wave, lr, m, l, o);
#pragma unroll
    for (int i = 0; i < kCh; ++i) sum_o[wave][kCh * lane + i] = o[i];
    if (lane == 0) { sum_m[wave] = m; sum_l[wave] = l; }
    __syncthreads();
    float f[kWaves];
    m = fmaxf(fmaxf(sum_m[0], sum_m[1]), fmaxf(sum_m[2], sum_m[3]));
#pragma unroll
    for (int w = 0; w < kWaves; ++w) f[w] = __builtin_amdgcn_exp2f(sum_m[w] - m);
    l = (f[0] * sum_l[0] + f[1] * sum_l[1]) + (f[2] * sum_l[2] + f[3] * sum_l[3]);
    const int row = d.row_block * kRows + lr, tok = d.row0 + row / a.group, h = d.head * a.group + row % a.group, ch = threadIdx.x;
    if (ch < D) {
      const float sum = (f[0] * sum_o[0][ch] + f[1] * sum_o[1][ch]) + (f[2] * sum_o[2][ch] + f[3] * sum_o[3][ch]);
      a.o[((int64_t)tok * a.hq + h) * D + ch] = (__bf16)(l == 0.f ? 0.f : sum * (1.f / l));
    }
    if (ch == 0) a.lse[(int64_t)h * a.s.n_rows + tok] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
    __syncthreads();
  }
}

// ---- weights ------------------------------------------------------------------------------------

// Adds exp(score - LSE), summed over the rows of the group, to the tokens' weights: the products bound it, and the exponentials, which take longer than they do.  A block takes one
// (sequence, KV head, tile) at a time, those with the most rows first; its waves hold the tile's keys and divide the rows, 16 at a time, the next ones on their way.  The 16 sums of a
// lane (its keys) over its column's rows are added over the 16 columns, then over the waves.
// It is made for prompts: one of 4096 tokens, 8 heads on 8 of 128 channels, 31 us, 555 Tflop/s.  Of a head's few rows it has work for some of its waves only, each with the tile's keys: 64
// sequences of up to 16384 tokens, int8, 32 heads on 8, 5 new tokens each (20 rows) 758 us with weights, 157 without; 16 new (64 rows) 880 and 219.
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
// Sum over the 16 lanes of a row.
template <int Ctrl> __device__ inline float plus_dpp(float x) { return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), Ctrl, 0xf, 0xf, false)); }
__device__ inline float sum_of_16(float x) { return plus_dpp<0x121>(plus_dpp<0x122>(plus_dpp<0x124>(plus_dpp<0x128>(x)))); }   // turned by 8, 4, 2, 1 lanes

constexpr int kWeighThreads = 512, kWeighWaves = kWeighThreads / 64;

template <int D, int Fmt>
__global__ __launch_bounds__(kWeighThreads, 2) void weigh_kernel(WeighArgs a) {
  constexpr int kRowBytes = 16 * 2 * D;                    // of a wave's 16 rows
  __shared__ float sum[kWeighWaves][kTile];
  __shared__ __align__(256) unsigned char rows_lds[kWeighWaves * 2 * kRowBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  // the line with one block of rows per KV head
  const int kAll = INT32_MAX;
  const Line line = find_on_line<0, kWeighThreads>(a.s, a.c, 1, kAll, 0, blockIdx.x);
  if (line.seq < 0) return;
  int seq = line.seq;
  int32_t base = line.before;
  SeqSizes z = line.z;
  for (int32_t u = blockIdx.x; u < line.total; u += gridDim.x) {
    __syncthreads();                   // (everybody has read the sums of the tile before)
    while (u >= base + cost_of<0>(z, a.c.hkv, 1, kAll)) {
      base += cost_of<0>(z, a.c.hkv, 1, kAll);
      z = seq_sizes(a.s, ++seq, a.c.page);
    }
    const int tile = (u - base) / a.c.hkv, head = (u - base) % a.c.hkv;
    const int key0 = tile * kTile, all_rows = z.n * a.group;
    // the first token that sees the tile's first key
    const int tok0 = max(key0 - (z.len - z.n), 0), rb0 = (int)((int64_t)tok0 * a.group / 16);
    const TilePages at = pages_of(a.c, lane, z.len > 0 ? ask_pages(a.c, a.s.pages + (int64_t)seq * a.s.max_pages, lane, z.len, tile) : TilePages{-1, -1}, z.len, tile);
    const TileScales sc = scales_of(a.c, head, at.v);
    // What the wave asks for a block of 16 rows ahead: queries through LDS, four lanes a row, so that a request is 64 bytes (operand rows straight from memory are 16 bytes a
    // request, and the requests bounded the kernel: a prompt of 4096 tokens, 8 heads, 48 us instead of 36), and the LSE of the lane's row n.
    // Row lane / 4 (queries) and row n (LSE, mask) of the block: token and query head of the group, and where they lie, stepped without divisions.
    const int step = 16 * kWeighWaves, step_tok = step / a.group, step_h = step % a.group;
    auto start = [&](int row, int& tok, int& h) { tok = row / a.group; h = row % a.group; };
    const int first_row = 16 * (rb0 + wave);
    int q_tok, q_h, tok, h, q_row = first_row + lane / 4, row = first_row + n;
    start(q_row, q_tok, q_h);
    start(row, tok, h);
    const __bf16* const q0 = a.q + (int64_t)z.row0 * a.q_row + head * a.group * D + 8 * ((lane & 3) ^ (lane >> 4));
    const float* const lse0 = a.lse + head * a.group * a.lse_head + z.row0;
    int64_t q_at = (int64_t)q_tok * a.q_row + q_h * D, lse_at = h * a.lse_head + tok;
    const int64_t q_step = step_tok * a.q_row + step_h * D, q_wrap = a.q_row - a.group * D, lse_step = step_h * a.lse_head + step_tok, lse_wrap = 1 - a.group * a.lse_head;
    unsigned char* const buffers = rows_lds + wave * 2 * kRowBytes;
    auto ask = [&](int buffer, float& lse) {               // (rows that are not there: the first one's)
      const __bf16* x = q0 + (q_row < all_rows ? q_at : 0);
      // 64-byte piece j of all 16 rows goes to the buffer's j-th KB, lane after lane: row lane / 4, place lane % 4, which holds chunk (lane % 4) ^ (row / 4) of the piece
#pragma unroll
      for (int j = 0; j < D / 32; ++j) lds_load_b128(x + 32 * j, lds_offset(buffers) + buffer * kRowBytes + 1024 * j);
      lse = lse0[row < all_rows ? lse_at : 0];
    };
    float lse[2];
    ask(0, lse[0]);
    bf16x8 k[4][D / 32];
    {
      u32x4 raw[4][D / 64];
      load_keys<D>(a.c, lane, head, tile, at.k, raw);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
          k[i][2 * j] = decode8<Fmt>(raw[i][j][0], raw[i][j][1]);
          k[i][2 * j + 1] = decode8<Fmt>(raw[i][j][2], raw[i][j][3]);
        }
    }
    // (operand 2 j + e holds channels 64 j + 16 g + 8 e ..: chunk 2 (g % 2) + e of piece 2 j + g / 2)
    int q_from[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) q_from[e] = 1024 * (g >> 1) + 64 * n + 16 * ((2 * (g & 1) + e) ^ (n >> 2));
    const float c = a.scale * sc.k;
    const int there = at.v < 0 ? -1 : 15;                  // (keys of a page that is not there are not seen)
    float got[16] = {};
    auto add = [&](int buffer, const float& now, float& next) {
      __builtin_amdgcn_s_waitcnt(kWaitVm0);                // the buffer's rows are there
      const float mine = now;
      const float lse2 = mine * kLog2e;
      // of the lane's keys, those up to `last` are seen; none by rows that are not there, and by rows that saw nothing
      const int last = row < all_rows && mine != -INFINITY ? min(z.len - z.n + tok - key0 - 16 * g, there) : -1;
      auto move = [&](int& r, int& t, int& hh) {
        r += step;
        t += step_tok;
        hh += step_h;
        const bool wraps = hh >= a.group;
        hh -= wraps ? a.group : 0;
        t += wraps;
        return wraps;
      };
      q_at += q_step + (move(q_row, q_tok, q_h) ? q_wrap : 0);
      lse_at += lse_step + (move(row, tok, h) ? lse_wrap : 0);
      bf16x8 q[D / 32];
      typedef bf16x8 __attribute__((may_alias)) chunk;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) q[j] = *reinterpret_cast<const chunk*>(buffers + buffer * kRowBytes + 2048 * (j / 2) + q_from[j % 2]);
      ask(buffer ^ 1, next);
      f32x4 s[4] = {};
#pragma unroll
      for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[i][j], q[j], s[i], 0, 0, 0);
      if (__ballot(last < 15)) {
        if (!__ballot(last >= 0)) return;
        // (chosen behind the exponential: a score or an LSE that is NaN must not reach keys that the row does not see)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 4][i % 4], c, -lse2));
          got[i] += i <= last ? e : 0.f;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) got[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 4][i % 4], c, -lse2));
      }
    };
    for (int rb = rb0 + wave; rb * 16 < all_rows; rb += 2 * kWeighWaves) {
      add(0, lse[0], lse[1]);
      add(1, lse[1], lse[0]);
    }
    __builtin_amdgcn_s_waitcnt(kWaitVm0);                  // (the rows asked for in vain have landed before the buffers are used again)
#pragma unroll
    for (int i = 0; i < 16; ++i) got[i] = sum_of_16(got[i]);
    if (n == 0)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[wave][16 * g + i] = got[i];
    __syncthreads();
    if (threadIdx.x < kTile && key0 + (int)threadIdx.x < z.len) {
      const int key = key0 + threadIdx.x;
      const int32_t p = page_at(a.s, a.c, seq, key >> a.c.log_page);
      if (p >= 0) {
        float* w = a.c.weight + block_of(a.c, p, head) * a.c.page + (key & (a.c.page - 1));
        float all = 0.f;
#pragma unroll
        for (int i = 0; i < kWeighWaves; ++i) all += sum[i][threadIdx.x];
        *w += all;
      }
    }
  }
}

// The same from the scores that the attention kernel left (blocks of 16 rows): a wave takes four rows of a tile at a time, which are 1 KB at one place, four keys a lane, and four tiles.  The sums
// over a quad's four rows then go to the lanes in the order of the keys, so that weights are read and written 256 bytes at a time.
__device__ inline float sum_of_quad(float x) {             // neighbours (1 0 3 2), then pairs (2 3 0 1)
  x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xb1, 0xf, 0xf, false));
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4e, 0xf, 0xf, false));
}
constexpr int kScoreTiles = 4 * kWaves;   // that a block works at once
__global__ __launch_bounds__(256) void weigh_scores_kernel(AttnArgs a, int rows_of_block) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t me = blockIdx.x;
  const Line line = find_on_line<kItemLead, 256, kScoreTiles>(a.s, a.c, a.group, rows_of_block, gridDim.x, me);
  if (line.seq < 0) return;
  int32_t at = line.begin(me);
  const int32_t end = line.begin(me + 1);
  int seq = line.seq;
  int32_t base = line.before;
  SeqSizes z = line.z;
  while (at < end) {
    while (at >= base + cost_of<kItemLead>(z, a.c.hkv, a.group, rows_of_block)) {
      base += cost_of<kItemLead>(z, a.c.hkv, a.group, rows_of_block);
      z = seq_sizes(a.s, ++seq, a.c.page);
    }
    const int tiles = tiles_of(z.len), all_rows = z.n * a.group, row_blocks = (all_rows + rows_of_block - 1) / rows_of_block;
    const int places = places_of<kItemLead>(z.len), item = (at - base) / places, from = (at - base) % places;
    const Piece piece = piece_of<kItemLead>(tiles, from, end - at);
    const int head = item / row_blocks, rb = item % row_blocks, t0 = piece.first, t1 = piece.last;
    // the rows of all blocks of a head add to the same weights: those of the first block's share do it, so that no two do
    if (rb == 0 && z.len > 0) {
      const int32_t* const table = a.s.pages + (int64_t)seq * a.s.max_pages;
      constexpr int kUnroll = kScoreTiles / kWaves;
      // lane 16 i + 4 g + r holds row r of keys 16 g + 4 i ..; key 16 g + 4 i + k's sum is element k there
      const int sub = lane & 3, from = 16 * ((lane >> 2) & 3) + 4 * (lane >> 4) + sub;
      for (int i = t0 + wave; i < t1; i += kWaves * kUnroll) {
        // everything is asked for before anything is waited for: the first four rows' scores and LSE, the pages, then the weights so far
        f32x4 s[kUnroll], got[kUnroll] = {};
        float sum[kUnroll], lse = 0.f;
        auto rows_at = [&](int r0) {
          const int row = min(r0 + sub, all_rows - 1);
          lse = a.lse[(int64_t)(head * a.group + row % a.group) * a.s.n_rows + z.row0 + row / a.group];
          const int b = row / rows_of_block, floats = score_floats(min(all_rows - b * rows_of_block, rows_of_block));
          const float* const s0 = a.scores + ((int64_t)base + ((int64_t)head * row_blocks + b) * places) * (16 * kTile) + score_at(row % rows_of_block) + 16 * (lane >> 2);
#pragma unroll
          for (int j = 0; j < kUnroll; ++j) s[j] = *reinterpret_cast<const f32x4*>(s0 + (int64_t)min(i + kWaves * j, t1 - 1) * floats);
        };
        rows_at(0);
        int32_t page[kUnroll];
        float* to[kUnroll];
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) page[j] = table[min((i + kWaves * j) * kTile + lane, z.len - 1) >> a.c.log_page];
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) {
          const int key = (i + kWaves * j) * kTile + lane;
          const bool there = (uint32_t)page[j] < (uint32_t)a.c.n_pages;
          to[j] = a.c.weight + block_of(a.c, there ? page[j] : 0, head) * a.c.page + (key & (a.c.page - 1));
          sum[j] = *to[j];
          if (!there || i + kWaves * j >= t1 || key >= z.len) to[j] = nullptr;
        }
        for (int r0 = 0; r0 < all_rows; r0 += 4) {
          if (r0 > 0) rows_at(r0);
          const float lse2 = r0 + sub < all_rows && lse != -INFINITY ? lse * kLog2e : INFINITY;       // (else nothing is added)
          if (__ballot(lse2 != lse2)) {                    // rare: a row's NaN must not reach keys that it does not see, whose scores are -inf
#pragma unroll
            for (int j = 0; j < kUnroll; ++j)
#pragma unroll
              for (int k = 0; k < 4; ++k) got[j][k] += s[j][k] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s[j][k] - lse2);
            continue;
          }
#pragma unroll
          for (int j = 0; j < kUnroll; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k) got[j][k] += __builtin_amdgcn_exp2f(s[j][k] - lse2);
        }
#pragma unroll
        for (int j = 0; j < kUnroll; ++j) {
#pragma unroll
          for (int k = 0; k < 4; ++k) got[j][k] = sum_of_quad(got[j][k]);
          const float mine = sub < 2 ? (sub == 0 ? got[j][0] : got[j][1]) : (sub == 2 ? got[j][2] : got[j][3]);
          const float all = __shfl(mine, from);
          if (to[j]) *to[j] = sum[j] + all;
        }
      }
    }
    at += piece.places;
  }
}

// ---- host ---------------------------------------------------------------------------------------

// Tables of up to this many tiles: an item is not divided among blocks, which saves the second launch.  Few rows (not divided / divided; one token of each sequence, 32 heads on 8, 128
// channels, int8): one sequence of 500 tokens 8.6 / 10.4 us, of 1000 11.8 / 10.6, of 1500 15.3 / 11.0; 16 of up to 1000 12.3 / 13.1, of up to 1500 15.8 / 13.9.  Twice as many where there are
// items for all blocks, since shares would end inside items of a few tiles: 64 of up to 1000 17.5 / 20.3, of up to 1500 22.6 / 23.2, of up to 2000 27.7 / 26.9 (with 5 new tokens each 37.7 / 41.5).
// Many rows: a tile costs more, so fewer.  40 new tokens each (blocks of 128 rows): 8 of up to 250 15.9 / 21.3, of 380 20.1 / 22.2, of 500 23.6 / 22.8; 16 new (64 rows, 64 channels, e4m3): 8 of
// up to 500 12.5 / 13.4, 64 of up to 500 16.2 / 21.1.
int whole_tiles(int rows, int64_t items) { return rows == kManyRows ? 6 : rows == kManyRows / 2 ? 8 : items >= kBlocks ? 32 : 16; }

// How a call is worked.  Up to 16 or 32 rows per sequence and KV head on average: a block of as many rows, whose waves divide the keys; more: 64 or 128 rows, which its waves divide.
// 64 sequences of up to 16384 tokens, int8, 32 heads on 8: 5 new tokens each (20 rows), 32 rows a block 157 us, 128 rows 250; 16 new (64 rows), 64 rows a block 219 us, 128 rows 264.  Of up
// to 1000: 24 / 39, 36 / 42; 8 of up to 8000: 29 / 40, 39 / 44.
struct AttnPlan { int rows; bool stored; bool whole; int64_t part_floats, score_floats, places; };
AttnPlan plan_attn(const CacheView& c, int head_dim, int32_t n_seqs, int32_t max_pages, int32_t tq, int32_t hq, bool weigh) {
  const int group = hq / c.hkv;
  AttnPlan p;
  const int64_t all_rows = (int64_t)tq * group;
  p.rows = all_rows <= (int64_t)16 * n_seqs ? 16 : all_rows <= (int64_t)32 * n_seqs ? 32 : all_rows <= (int64_t)64 * n_seqs ? kManyRows / 2 : kManyRows;
  p.stored = weigh && p.rows == 16;
  p.part_floats = (int64_t)2 * kBlocks * slot_floats(head_dim, p.rows);
  const int64_t tiles = max(((int64_t)max_pages * c.page + kTile - 1) / kTile, (int64_t)1);
  p.whole = !p.stored && tiles <= whole_tiles(p.rows, (int64_t)n_seqs * c.hkv);
  p.places = (tiles + kItemLead) * c.hkv * (n_seqs + (int64_t)tq * group / p.rows);
  p.score_floats = p.stored ? p.places * 16 * kTile : 0;
  return p;
}

// slots, and who the divided items are
size_t part_bytes(const AttnPlan& p) { return pad_to((size_t)p.part_floats * 4, 256) + pad_to(kBlocks * sizeof(Divided), 256); }
// .. and kept scores
size_t attn_bytes(const AttnPlan& p) { return part_bytes(p) + pad_to((size_t)p.score_floats * 4, 256); }

template <int D, int Fmt>
int launch_attn(const AttnArgs& a, const AttnPlan& p, hipStream_t st) {
  const dim3 grid(kBlocks), block(256);
  if (p.rows > 32) return launch_attn_rows(a, D, Fmt, p.rows, p.whole, st);
  auto kernel = p.rows == 32 ? (p.whole ? attn_kernel<D, Fmt, true, false, 2> : attn_kernel<D, Fmt, false, false, 2>)
                             : p.whole ? attn_kernel<D, Fmt, true, false, 1> : p.stored ? attn_kernel<D, Fmt, false, true, 1> : attn_kernel<D, Fmt, false, false, 1>;
  kernel<<<grid, block, 0, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  if (!p.whole) {
    // A block for each row that an item has on average, but 4 at least.  4 / 8 / 16 / 32 blocks: 64 sequences of up to 4000 tokens, 4 rows 43.1 / 44.5 / 46.6 / 50.4 us; 16 of up to
    // 8000, 16 rows 16.3 / 14.1 / 13.3 / 13.8.
    const int64_t rows = ((int64_t)a.s.n_rows * a.group + a.s.n_seqs - 1) / a.s.n_seqs;
    const int of_item = rows <= 4 ? 4 : rows <= 8 ? 8 : rows <= 16 ? 16 : 32;
    auto merge = p.rows == 32 ? attn_merge_kernel<D, 32> : attn_merge_kernel<D, 16>;
    merge<<<dim3((unsigned)(kBlocks * of_item)), block, 0, st>>>(a, of_item);
    FCP_HIP_CHECK(hipGetLastError());
  }
  if (p.stored) {
    weigh_scores_kernel<<<dim3((unsigned)min((p.places + kScoreTiles - 1) / kScoreTiles, (int64_t)5 * kBlocks / 2)), block, 0, st>>>(a, p.rows);
    FCP_HIP_CHECK(hipGetLastError());
  }
  return FCP_OK;
}

int launch_weigh(const WeighArgs& a, int head_dim, int format, hipStream_t st) {
  const int64_t most = max(((int64_t)a.s.max_pages * a.c.page + kTile - 1) / kTile, (int64_t)1) * a.c.hkv * a.s.n_seqs;
  auto kernel = head_dim == 128 ? (format == kE4m3 ? weigh_kernel<128, kE4m3> : weigh_kernel<128, kInt8>)
                                : (format == kE4m3 ? weigh_kernel<64, kE4m3> : weigh_kernel<64, kInt8>);
  kernel<<<dim3((unsigned)min(most, (int64_t)2 * kBlocks)), dim3(kWeighThreads), 0, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  return FCP_OK;
}

int check_places(const char* who, const AttnPlan& p) {
  if (p.places > kMostPlaces) return fail(FCP_ERR_UNSUPPORTED, "%s: tables and rows that may make 2^31 tiles of work", who);
  return FCP_OK;
}

}  // namespace

int check_heads(const char* who, const CacheView& c, int32_t hq) {
  if (hq < 1 || hq % c.hkv) return fail(FCP_ERR_UNSUPPORTED, "%s: %d query heads on %d KV heads", who, hq, c.hkv);
  return FCP_OK;
}
// (times log2(e) and a scale of 2^-110 it must not become 0: a masked score, -inf, times 0 is NaN)
int check_scale(const char* who, float scale) {
  if (!(scale >= 0x1p-32f) || !__builtin_isfinite(scale)) return fail(FCP_ERR_INVALID_ARG, "%s: softmax_scale must be finite and at least 2^-32", who);
  return FCP_OK;
}
int check_row_count(const char* who, int32_t tq, int32_t hq) {
  if ((int64_t)tq * hq > INT32_MAX - 256) return fail(FCP_ERR_UNSUPPORTED, "%s: more than 2^31 rows of all heads", who);
  return FCP_OK;
}
int check_rows(const char* who, const fcp_cache* cache, const void* q, int64_t q_row, int32_t tq, int32_t hq) {
  if (!q || q_row < (int64_t)hq * cache->head_dim || q_row % 8 || (uintptr_t)q % 16)
    return fail(FCP_ERR_INVALID_ARG, "%s: query rows must be at least hq * head_dim elements apart, a multiple of 8, and 16-byte aligned", who);
  return check_row_count(who, tq, hq);
}

// 0: refused
size_t evict_scratch_bytes(const char* who, const CacheView& c, int32_t n_seqs, int32_t max_pages);
size_t page_scratch_bytes(const char* who, const CacheView& c, bool fork, int32_t n_seqs, int32_t max_pages);
size_t shared_scratch_bytes(const char* who, const CacheView& c, int head_dim, int32_t n_seqs, int32_t max_pages, int32_t tq, int32_t hq);

size_t attn_scratch_bytes(const CacheView& c, int head_dim, int32_t n_seqs, int32_t max_pages, int32_t tq, int32_t hq) {
  return attn_bytes(plan_attn(c, head_dim, n_seqs, max_pages, tq, hq, false));
}

}  // namespace fcp

extern "C" size_t fcp_cache_scratch_bytes(int which, const fcp_cache* cache, int32_t n_seqs, int32_t max_pages, int32_t tq, int32_t hq) {
  using namespace fcp;
  clear_error();
  const char* who = "fcp_cache_scratch_bytes";
  CacheView c;
  if (check_cache(who, cache, which == FCP_SCRATCH_CACHE_WEIGH || which == FCP_SCRATCH_CACHE_EVICT, &c)) return 0;
  if (check_sizes(who, c, n_seqs, max_pages, tq)) return 0;
  if (which == FCP_SCRATCH_CACHE_EVICT) return evict_scratch_bytes(who, c, n_seqs, max_pages);
  if (which == FCP_SCRATCH_CACHE_FORK || which == FCP_SCRATCH_CACHE_COMPACT) return page_scratch_bytes(who, c, which == FCP_SCRATCH_CACHE_FORK, n_seqs, max_pages);
  if (which == FCP_SCRATCH_CACHE_SHARED) return shared_scratch_bytes(who, c, cache->head_dim, n_seqs, max_pages, tq, hq);
  if (which != FCP_SCRATCH_CACHE_ATTN && which != FCP_SCRATCH_CACHE_WEIGH) { fail(FCP_ERR_INVALID_ARG, "%s: which = %d is not known", who, which); return 0; }
  if (check_heads(who, c, hq)) return 0;
  const bool weigh = which == FCP_SCRATCH_CACHE_WEIGH;
  const AttnPlan p = plan_attn(c, cache->head_dim, n_seqs, max_pages, tq, hq, weigh);
  if (n_seqs > 0 && tq > 0 && (check_row_count(who, tq, hq) || check_places(who, p))) return 0;
  return attn_bytes(p);
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
  if (int rc = check_seqs(who, a.c, cu_seqlens, true, kv_len, pages, n_seqs, max_pages, tq)) return rc;
  if (int rc = check_scale(who, softmax_scale)) return rc;
  if (tq == 0 || n_seqs == 0) return FCP_OK;
  if (int rc = check_rows(who, cache, q, q_row, tq, hq)) return rc;
  if (!o || !lse || (uintptr_t)o % 16 || (uintptr_t)lse % 4) return fail(FCP_ERR_INVALID_ARG, "%s: o and lse are required and must be aligned", who);
  if (!scratch || (uintptr_t)scratch % 256) return fail(FCP_ERR_INVALID_ARG, "%s: scratch must be 256-byte aligned", who);
  const AttnPlan p = plan_attn(a.c, cache->head_dim, n_seqs, max_pages, tq, hq, weigh);
  if (int rc = check_places(who, p)) return rc;
  const size_t need = attn_bytes(p);
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
  a.divided = reinterpret_cast<Divided*>(static_cast<char*>(scratch) + pad_to((size_t)p.part_floats * 4, 256));
  a.scores = p.stored ? reinterpret_cast<float*>(static_cast<char*>(scratch) + part_bytes(p)) : nullptr;
  a.blocks = kBlocks;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool e4m3 = cache->format == FCP_CACHE_E4M3;
  const int rc = cache->head_dim == 128 ? (e4m3 ? launch_attn<128, kE4m3>(a, p, st) : launch_attn<128, kInt8>(a, p, st))
                                        : (e4m3 ? launch_attn<64, kE4m3>(a, p, st) : launch_attn<64, kInt8>(a, p, st));
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
  if (int rc = check_seqs(who, a.c, cu_seqlens, true, kv_len, pages, n_seqs, max_pages, tq)) return rc;
  if (int rc = check_scale(who, softmax_scale)) return rc;
  if (tq == 0 || n_seqs == 0) return FCP_OK;
  if (int rc = check_rows(who, cache, q, q_row, tq, hq)) return rc;
  if (!lse || (uintptr_t)lse % 4) return fail(FCP_ERR_INVALID_ARG, "%s: lse is required", who);
  if (int rc = check_places(who, plan_attn(a.c, cache->head_dim, n_seqs, max_pages, tq, hq, false))) return rc;
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
