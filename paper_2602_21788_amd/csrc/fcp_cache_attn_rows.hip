// Attention over the paged 8-bit cache for many rows: pieces of prompts, or several new tokens of many query heads.
//
// A block takes 128 rows of a KV head's group at a time, a wave 32 of them, against tiles of 64 keys.  The products and the exponentials bound it (4 D flops a pair; an exponential
// takes as long as 64 flops of the matrix units per lane), so the codes must not become bf16 in every wave: a tile's codes come in whole lines, 32 a thread, become bf16 in
// the page's scale there (exact) and go to LDS, from which the waves read the operands of the 16 x 16 x 32 instructions, each for two blocks of 16 rows.  The next tile's codes
// are on their way meanwhile, in registers; one barrier a tile, two stages.  Two blocks per CU, in no lock step: the one's exponentials meet the other's products.
// Operand rows straight from memory would be requests of 16 bytes a lane, a quarter of a line's rate, in every wave.
// Keys and rows are laid on the matrix as in the kernel for few rows: a lane ends with the scores of 16 neighbouring keys, which is the operand of the product with V.
#include "fcp_cache_attn.h"

namespace fcp {
namespace {

constexpr int kNB = 2;                 // blocks of 16 rows of a wave

// LDS of a stage: keys as rows of D channels, values as rows (channels) of 64 keys, in chunks of 8 bf16 whose places in a row are permuted so that the 16 rows of
// an operand lie on different banks.
template <int D>
struct Stage {
  static constexpr int kKeyRow = 2 * D, kValueRow = 2 * kTile, kKeys = kTile * kKeyRow, kBytes = kKeys + D * kValueRow;
  // an operand's rows are 16 a + 4 i + b, a and b from 0 to 3: with 128 channels a row is a whole bank cycle, with 64 two rows are
  static __device__ int key_mix(int row) { return D == 128 ? ((row >> 4) & 3) * 4 + (row & 3) : ((row >> 4) & 3) * 2 + ((row >> 1) & 1); }
  static __device__ int value_mix(int ch) { return (ch >> 1) & 7; }
  static __device__ int key_at(int row, int chunk) { return row * kKeyRow + ((chunk ^ key_mix(row)) << 4); }
  static __device__ int value_at(int ch, int chunk) { return kKeys + ch * kValueRow + ((chunk ^ value_mix(ch)) << 4); }
};

// 16 codes as bf16 in their scale, a power of two: exact.
template <int Fmt>
__device__ inline void decode16(u32x4 w, float scale, bf16x8& a, bf16x8& b) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bf16x2 lo, hi;
    if constexpr (Fmt == kE4m3) {
      lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], scale, true);
    } else {
      const f32x2 f = decode_half<Fmt, false>(w[i]), g = decode_half<Fmt, true>(w[i]);
      lo = bf16x2{(__bf16)(f[0] * scale), (__bf16)(f[1] * scale)};
      hi = bf16x2{(__bf16)(g[0] * scale), (__bf16)(g[1] * scale)};
    }
    bf16x8& to = i < 2 ? a : b;
    to[4 * (i & 1)] = lo[0];
    to[4 * (i & 1) + 1] = lo[1];
    to[4 * (i & 1) + 2] = hi[0];
    to[4 * (i & 1) + 3] = hi[1];
  }
}

// A wave's share of a tile, D / 64 times: 64 D / 256 bytes of one group of 16 keys and as many of the group's values, which lie in one run each, 16 a lane.  Page, scales and
// sizes are the same for the whole wave, so they travel in scalar registers.
typedef const int32_t __attribute__((address_space(4)))* scalar_int;
typedef const float __attribute__((address_space(4)))* scalar_float;
__device__ inline scalar_int as_scalar(const int32_t* p) { return (scalar_int)(uintptr_t)p; }
__device__ inline scalar_float as_scalar(const float* p) { return (scalar_float)(uintptr_t)p; }

template <int D>
struct Share {
  u32x4 k[D / 64], v[D / 64];
  float ks[D / 64], vs[D / 64];
  int live[D / 64];                    // of the 16 keys, those that are cached tokens (0: the page is not there)
};
// group of 16 keys, and the wave's place in it (in lots of 64 times 16 bytes)
template <int D> __device__ inline int group_of(int wave, int i) { return D == 128 ? wave / 2 + 2 * i : wave; }
template <int D> __device__ inline int lot_of(int wave) { return D == 128 ? wave & 1 : 0; }

template <int D>
__device__ inline void load_share(const AttnArgs& a, const int32_t* table, int head, int len, int tile, int wave, Share<D>& s) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const int key = tile * kTile + kGroup * group_of<D>(wave, i), place = key >> a.c.log_page;
    int32_t page = -1;
    if (key < len) page = as_scalar(table)[place];         // (len is at most what the table holds)
    const bool there = (uint32_t)page < (uint32_t)a.c.n_pages;
    const int64_t block = block_of(a.c, there ? page : 0, head), at = (block * a.c.page + (key & (a.c.page - 1))) * D + 1024 * lot_of<D>(wave);
    s.live[i] = there ? min(len - key, kGroup) : 0;
    s.ks[i] = as_scalar(a.c.k_scale)[block];
    s.vs[i] = as_scalar(a.c.v_scale)[block];
    const int mine = 16 * (int)(threadIdx.x & 63);
    s.k[i] = *reinterpret_cast<const u32x4*>(a.c.k + at + mine);
    s.v[i] = *reinterpret_cast<const u32x4*>(a.c.v + at + mine);
  }
}
// live: per group of 16 keys; odd: a value is NaN.  partly: some row of the block does not see the whole tile.
template <int D, int Fmt>
__device__ inline void store_share(const Share<D>& s, int wave, unsigned char* stage, int32_t* live, int32_t* odd, bool partly) {
  typedef bf16x8 __attribute__((may_alias)) chunk;
  // (the thread's number is formed anew: the compiler would keep the addresses that follow from it in registers, and spill them)
  const int lane = fresh((int)threadIdx.x) & 63;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const int g = group_of<D>(wave, i), at = 64 * lot_of<D>(wave) + lane, key = kGroup * g + at / (D / 16), c = at % (D / 16), ch = at;
    bf16x8 x, y;
    decode16<Fmt>(s.k[i], s.ks[i], x, y);
    *reinterpret_cast<chunk*>(stage + Stage<D>::key_at(key, 2 * c)) = x;
    *reinterpret_cast<chunk*>(stage + Stage<D>::key_at(key, 2 * c + 1)) = y;
    u32x4 v = s.v[i];
    if (s.live[i] < kGroup) {                              // codes past the last token are whatever the page holds, and 0 * NaN is NaN
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int n = min(max(s.live[i] - 4 * w, 0), 4);
        v[w] &= n == 4 ? 0xffffffffu : (1u << (8 * n)) - 1;
      }
    }
    if (Fmt == kE4m3 && partly) {
      uint32_t o = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) o |= ((v[w] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
      if (o) *odd = 1;
    }
    decode16<Fmt>(v, s.vs[i], x, y);
    *reinterpret_cast<chunk*>(stage + Stage<D>::value_at(ch, 2 * g)) = x;
    *reinterpret_cast<chunk*>(stage + Stage<D>::value_at(ch, 2 * g + 1)) = y;
    if (lane == 0) live[g] = s.live[i];
  }
}

template <int D, int Fmt, bool Short>
__global__ __launch_bounds__(256, 2) void attn_rows_kernel(AttnArgs a) {
  typedef bf16x8 __attribute__((may_alias)) chunk;
  extern __shared__ __align__(256) unsigned char lds[];    // two stages
  __shared__ int32_t live[2][4], odd[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  // the lane's operand rows: neither permutation depends on the 4 i or 16 d that steps through them
  const int key_first = 16 * (n >> 2) + (n & 3), key_row = key_first * Stage<D>::kKeyRow, key_mix = Stage<D>::key_mix(key_first);
  const int value_row = Stage<D>::kKeys + n * Stage<D>::kValueRow, value_mix = Stage<D>::value_mix(n);
  const int32_t me = blockIdx.x;
  const Line line = find_on_line<Short>(a.s, a.c, a.group, kManyRows, a.blocks, me, -1);
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
    while (at >= base + cost_of<Short>(z, a.c.hkv, a.group, kManyRows)) {  // the next sequence with rows
      base += cost_of<Short>(z, a.c.hkv, a.group, kManyRows);
      z = seq_sizes(a.s, ++seq, a.c.page);
    }
    const int tiles = tiles_of(z.len), all_rows = z.n * a.group, row_blocks = (all_rows + kManyRows - 1) / kManyRows;
    const int item = Short ? at - base : (at - base) / tiles, t0 = Short ? 0 : (at - base) % tiles;
    const int t1 = Short ? tiles : min(tiles, t0 + end - at);
    const int head = item / row_blocks, rb = item % row_blocks;
    const int32_t at0 = at;
    at += Short ? 1 : t1 - t0;

    bf16x8 q[kNB][D / 32];
    f32x4 o[kNB][D / 16];
    float m[kNB], l[kNB];
    int last[kNB];                                         // last token that the lane's row sees
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
      const int row = rb * kManyRows + (wave * kNB + b) * 16 + n;
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
    const int rows = min(all_rows - rb * kManyRows, kManyRows), all_see = z.len - z.n + rb * kManyRows / a.group;
    const int seen = z.len - z.n + (rb * kManyRows + rows - 1) / a.group;
    const int t_end = min(t1, seen < 0 ? 0 : seen / kTile + 1);
    if (t0 < t_end) {
      Share<D> share;
      const int32_t* const table = a.s.pages + (int64_t)seq * a.s.max_pages;
      load_share<D>(a, table, head, z.len, t0, wave, share);
      if (threadIdx.x < 2) odd[threadIdx.x] = 0;
      __syncthreads();                                     // (the stages of the item before have been read)
      store_share<D, Fmt>(share, wave, lds, live[0], &odd[0], t0 * kTile + kTile - 1 > all_see);
      load_share<D>(a, table, head, z.len, t0 + 1, wave, share);     // (past the last tile: pages that are not there, the pool's first is read)
      for (int t = t0; t < t_end; ++t) {
        const int st = (t - t0) & 1;
        unsigned char* const stage = lds + st * Stage<D>::kBytes;
        __syncthreads();
        if (t + 1 < t_end) store_share<D, Fmt>(share, wave, lds + (st ^ 1) * Stage<D>::kBytes, live[st ^ 1], &odd[st ^ 1], (t + 1) * kTile + kTile - 1 > all_see);
        load_share<D>(a, table, head, z.len, t + 2, wave, share);
        __builtin_amdgcn_sched_barrier(0);                 // (the compiler would keep operands of all parts of the step in registers, and spill)

        f32x4 s[kNB][4];
        const unsigned char* const keys = stage + fresh(key_row);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
          for (int b = 0; b < kNB; ++b) s[b][i] = f32x4{0, 0, 0, 0};
#pragma unroll
          for (int j = 0; j < D / 32; ++j) {
            const bf16x8 k = *reinterpret_cast<const chunk*>(keys + 4 * i * Stage<D>::kKeyRow + (((4 * j + g) ^ key_mix) << 4));
#pragma unroll
            for (int b = 0; b < kNB; ++b) s[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[b][j], s[b][i], 0, 0, 0);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        bf16x8 p[kNB][2];
        const int live_here = live[st][g];
        const bool full = t * kTile + kTile - 1 <= all_see && !__ballot(live_here < kGroup);
        const unsigned char* const values = stage + fresh(value_row);
        auto value = [&](int d, int u) { return *reinterpret_cast<const chunk*>(values + 16 * d * Stage<D>::kValueRow + (((2 * g + u) ^ value_mix) << 4)); };
        int sees[kNB];
#pragma unroll
        for (int b = 0; b < kNB; ++b) sees[b] = min(last[b] - t * kTile - 16 * g, live_here - 1);
        if (!full)
#pragma unroll
          for (int b = 0; b < kNB; ++b) mask_scores(s[b], sees[b]);
#pragma unroll
        for (int b = 0; b < kNB; ++b) softmax_of<D>(s[b], a.scale, 1.f, o[b], m[b], l[b], p[b], nullptr);
        __builtin_amdgcn_sched_barrier(0);
        if (Fmt == kE4m3 && !full && odd[st]) {
          // Rare: a value that some rows do not see is NaN.  The rows that see it get NaN and the others do not: the product with the probabilities takes zeros in its place,
          // and its number among the keys that a row sees is counted by a product with 1.
#pragma unroll
          for (int b = 0; b < kNB; ++b)
#pragma unroll
            for (int d = 0; d < D / 16; ++d) {
              __builtin_amdgcn_sched_barrier(0);
              f32x4 count = {0, 0, 0, 0};
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                bf16x8 v = value(d, u), bad, one;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                  const bool nan = __builtin_isnan((float)v[j]);
                  bad[j] = (__bf16)(nan ? 1.f : 0.f);
                  one[j] = (__bf16)(8 * u + j <= fresh(sees[b]) ? 1.f : 0.f);
                  v[j] = nan ? (__bf16)0.f : v[j];
                }
                count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bad, one, count, 0, 0, 0);
                o[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[b][u], o[b][d], 0, 0, 0);
              }
#pragma unroll
              for (int j = 0; j < 4; ++j) o[b][d][j] = count[j] > 0.f ? NAN : o[b][d][j];
            }
          __builtin_amdgcn_sched_barrier(0);
        } else {
#pragma unroll
          for (int d = 0; d < D / 16; ++d)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const bf16x8 v = value(d, u);
#pragma unroll
              for (int b = 0; b < kNB; ++b) o[b][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[b][u], o[b][d], 0, 0, 0);
            }
        }
      }
    }
#pragma unroll
    for (int b = 0; b < kNB; ++b) l[b] = sum_over_groups(l[b]);

    const bool whole = t0 == 0 && t1 == tiles;
    if (t0 == 0 && !whole) divided = {line.owner(at0 + tiles - 1) - me + 1, z.row0, all_rows, head, rb, {}};
    float* const slot = a.part + (int64_t)(2 * me + (t0 == 0 ? 1 : 0)) * slot_floats(D, kManyRows);
#pragma unroll
    for (int b = 0; b < kNB; ++b) {
      const int lr = (wave * kNB + b) * 16 + n, row = rb * kManyRows + lr;
      if (!whole) {                                        // sums as they lie in the registers: the merge divides them the same way
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4*>(slot + (((wave * kNB + b) * (D / 16) + i) * 64 + lane) * 4) = o[b][i];
        if (g == 0) { slot[kManyRows * D + lr] = m[b]; slot[kManyRows * (D + 1) + lr] = l[b]; }
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
template <int D>
__global__ __launch_bounds__(256) void attn_rows_merge_kernel(AttnArgs a) {
  constexpr int kFloats = slot_floats(D, kManyRows);
  const int me = blockIdx.x, part = blockIdx.y, lane = threadIdx.x & 63;
  const Divided d = a.divided[me];
  const int lr = part * 16 + (lane & 15), row = d.row_block * kManyRows + lr;
  if (d.pieces == 0 || row >= d.all_rows) return;
  float m = kLow;
#pragma unroll 4
  for (int p = 0; p < d.pieces; ++p) m = fmaxf(m, piece_slot(a, me, p, kFloats)[kManyRows * D + lr]);
  f32x4 o[D / 64];
#pragma unroll
  for (int i = 0; i < D / 64; ++i) o[i] = f32x4{0, 0, 0, 0};
  float l = 0.f;
#pragma unroll 4
  for (int p = 0; p < d.pieces; ++p) {
    const float* s = piece_slot(a, me, p, kFloats);
    const float f = __builtin_amdgcn_exp2f(s[kManyRows * D + lr] - m);
    l += f * s[kManyRows * (D + 1) + lr];
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
int launch(const AttnArgs& a, bool whole, hipStream_t st) {
  constexpr int kLds = 2 * Stage<D>::kBytes;
  static std::atomic<uint64_t> raised[2];
  auto kernel = whole ? attn_rows_kernel<D, Fmt, true> : attn_rows_kernel<D, Fmt, false>;
  if (kLds > 64 * 1024 - 1024)
    if (int rc = raise_lds_limit(reinterpret_cast<const void*>(kernel), kLds, raised[whole])) return rc;
  kernel<<<dim3(kBlocks), dim3(256), kLds, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  if (!whole) {
    attn_rows_merge_kernel<D><<<dim3(kBlocks, kManyRows / 16), dim3(256), 0, st>>>(a);
    FCP_HIP_CHECK(hipGetLastError());
  }
  return FCP_OK;
}

}  // namespace

int launch_attn_rows(const AttnArgs& a, int head_dim, int format, bool whole, hipStream_t st) {
  if (head_dim == 128) return format == kE4m3 ? launch<128, kE4m3>(a, whole, st) : launch<128, kInt8>(a, whole, st);
  return format == kE4m3 ? launch<64, kE4m3>(a, whole, st) : launch<64, kInt8>(a, whole, st);
}

}  // namespace fcp
