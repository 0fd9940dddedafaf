// fcp_cache_evict: the cached tokens with the greatest attention weight kept, per KV head, and moved to new pages.
//
// First the k-th greatest weight among the tokens of a (sequence, KV head) that are neither among the first nor the most recent is found, by counting an ordered integer's
// upper 11 bits and then, among the tokens that share those of the k-th, the next 11 and the last 10; the kept tokens are listed in order.  A block does that alone for
// short tables.  One CU takes about 20 us to look at 131072 weights once, so long ones are cut into chunks: one launch counts, one lists each chunk's tokens with the k-th's
// upper bits, one finds the border among those (every block for itself) and writes the chunk's part of the list.
// The last launch moves the tokens: a wave per (new page, KV head, keys or values).
// 4 sequences of up to 131072 tokens, 8 heads: choosing 7.5 + 10 + 18 us, chains of loads and barriers; moving 95 (the kernel says why).  4 of up to 600, 4 heads of 64 channels: 7 and 4.
// Pages of 128 tokens and 128 channels take more than 256 registers for a page's codes, one wave a SIMD instead of three: the long sequences 205 us altogether, with pages of 64 131.
#include "fcp_cache.h"

namespace fcp {
namespace {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
constexpr int kBins = 2048;
constexpr int kListed = 16384;         // tokens of a table that a block chooses from alone: candidates in 64 KB of LDS, weights in 16 registers a thread
constexpr int kMaxChunks = 32;

struct EvictArgs {
  CacheView c;
  SeqView s;                           // (no rows)
  const int32_t* new_pages;
  int32_t max_new, places, budget, first, recent;          // entries of a row of new_pages, those of them that can get a token
  int32_t* kept;
  int32_t* new_len;
  // long tables: tokens of a chunk, chunks; per (sequence, KV head): counts of each chunk, candidates, of each chunk the tokens above their upper bits, border
  int32_t chunk, chunks;
  int32_t* counts;                     // [chunks][kBins]
  uint32_t* list;                      // [max_pages * page]
  int32_t* above;                      // [chunks]
  int32_t* border;                     // upper bits, places left, candidates, unused
};

// An integer that orders weights: greater weight, greater integer; -0 and 0 are equal, every NaN is greatest.
__device__ inline uint32_t order_of(float w) {
  if (__builtin_isnan(w)) return 0xffffffffu;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ inline int32_t cached(const EvictArgs& a, int seq) {
  const int64_t room = (int64_t)a.s.max_pages * a.c.page;
  const int32_t n = max(a.s.kv_len[seq], 0);
  return n < room ? n : (int32_t)room;
}
// Weights of tokens t .. t + 3 (t a multiple of 4) as ordered integers; where the page is missing, of 0.
struct Quad { uint32_t u[4]; };
__device__ inline Quad orders_of(const EvictArgs& a, int32_t page, int head, int t) {
  f32x4 w = {0, 0, 0, 0};
  if (page >= 0) w = *reinterpret_cast<const f32x4*>(a.c.weight + block_of(a.c, page, head) * a.c.page + (t & (a.c.page - 1)));
  return {{order_of(w[0]), order_of(w[1]), order_of(w[2]), order_of(w[3])}};
}
// A thread's tokens of a block's 4096 U from `from` on: in round u those from from + 4096 u + 4 thread on.  All page numbers are asked for at once, then all weights, and these
// stay in registers for every look that the block takes at them.
template <int U>
struct Held {
  Quad q[U];
  int first;
  __device__ int token(int u) const { return first + 4 * kSelectThreads * u; }
  __device__ void load(const EvictArgs& a, int seq, int head, int from, int to) {
    first = from + 4 * (int)threadIdx.x;
    int32_t page[U];
#pragma unroll
    for (int u = 0; u < U; ++u) page[u] = token(u) < to ? page_at(a.s, a.c, seq, token(u) >> a.c.log_page) : -1;
#pragma unroll
    for (int u = 0; u < U; ++u) q[u] = orders_of(a, page[u], head, token(u));
  }
  // f(order, whether the token lies in [lo, hi))
  template <class F>
  __device__ void each(int lo, int hi, F f) const {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 4; ++j) f(q[u].u[j], token(u) + j >= lo && token(u) + j < hi);
  }
};
// One more in a bin.  Weights are often equal, and additions to one address wait for each other: the lanes that share the first lane's bin add once.
__device__ inline void count_in(int32_t* bins, uint32_t bin, bool in) {
  const uint64_t all = __ballot(in);
  if (!all) return;
  const uint32_t first = __builtin_amdgcn_readlane(bin, __ffsll((unsigned long long)all) - 1);
  const uint64_t same = __ballot(in && bin == first);
  if (in && bin != first) atomicAdd(&bins[bin], 1);
  if ((int)(threadIdx.x & 63) == __ffsll((unsigned long long)same) - 1) atomicAdd(&bins[first], (int32_t)__popcll(same));
}

// The bin that holds the want-th greatest, how many of it are wanted, and how many it holds.  The block's threads take two bins each, from the greatest down.
struct Found { int32_t bin, want, held; };
__device__ inline Found find_bin(const int32_t* bins, int32_t want) {
  __shared__ int32_t sums[kSelectWaves];
  __shared__ Found found;
  const int tid = threadIdx.x, wave = tid >> 6, b = kBins - 1 - 2 * tid;
  const int32_t x = bins[b], y = bins[b - 1], upto_wave = wave_prefix_sum(x + y);
  if ((tid & 63) == 63) sums[wave] = upto_wave;
  __syncthreads();
  int32_t over = upto_wave - x - y;
  for (int w = 0; w < wave; ++w) over += sums[w];
  if (over < want && want <= over + x) found = {b, want - over, x};
  else if (over + x < want && want <= over + x + y) found = {b - 1, want - over - x, y};
  __syncthreads();
  return found;
}
static_assert(kBins == 2 * kSelectThreads, "two bins a thread");

// Writes the kept ones of the block's tokens below `to` to the list from `place` on: the protected ones, those above the border, and of those at it the first ones while `want`
// lasts; `equals` of them came before.  none: no other than the protected.  Both counts are moved on.
template <int U>
__device__ inline void emit(const Held<U>& x, int32_t* kept, int to, int lo, int hi, bool none, uint32_t border, int32_t want, int32_t& place, int32_t& equals) {
  __shared__ int32_t sums[U][kSelectWaves];                // of a wave's tokens in a round: surely kept, and at the border (upper half)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t sure[U], equal[U];                              // a bit per token
  int32_t upto[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    sure[u] = equal[u] = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = x.token(u) + j;
      const bool in = t < to, safe = t < lo || t >= hi;
      sure[u] |= (uint32_t)(in && (safe || (!none && x.q[u].u[j] > border))) << j;
      equal[u] |= (uint32_t)(in && !safe && !none && x.q[u].u[j] == border) << j;
    }
    upto[u] = wave_prefix_sum(__popc(sure[u]) | __popc(equal[u]) << 16);
    if (lane == 63) sums[u][wave] = upto[u];
  }
  __syncthreads();
  int32_t before = 0;                                      // the rounds and waves before
#pragma unroll
  for (int u = 0; u < U; ++u) {
    int32_t here = before;
#pragma unroll
    for (int w = 0; w < kSelectWaves; ++w) {
      here += w < wave ? sums[u][w] : 0;
      before += sums[u][w];
    }
    here += upto[u] - (__popc(sure[u]) | __popc(equal[u]) << 16);
    int32_t eq = equals + (here >> 16);                    // at the border, before the lane's
    int32_t at = place + (here & 0xffff) + min(eq, want) - min(equals, want);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool is_equal = equal[u] >> j & 1;
      if ((sure[u] >> j & 1) || (is_equal && eq < want)) kept[at++] = x.token(u) + j;
      eq += is_equal;
    }
  }
  place += (before & 0xffff) + min(equals + (before >> 16), want) - min(equals, want);
  equals += before >> 16;
}

// What all blocks of a (sequence, KV head) begin with; the first writes the new length and the list's ends.  done: every token is kept.
struct Select { int32_t n, lo, hi, want; int32_t* kept; bool done; };
__device__ inline Select open_select(const EvictArgs& a, int seq, int head, bool writes) {
  const int n = cached(a, seq), n_new = min(n, a.budget), tid = threadIdx.x;
  int32_t* const kept = a.kept + ((int64_t)seq * a.c.hkv + head) * a.budget;
  if (writes) {
    if (head == 0 && tid == 0) a.new_len[seq] = n_new;
    for (int64_t i = n_new + tid; i < a.budget; i += kSelectThreads) kept[i] = -1;     // (64 bits: a budget may be 2^31 - 1)
    if (n <= a.budget)
      for (int i = tid; i < n; i += kSelectThreads) kept[i] = i;
  }
  return {n, a.first, n - a.recent, a.budget - a.first - a.recent, kept, n <= a.budget};
}

// The last kept weight among the m candidates of a list, which share its upper 11 bits (border): bits 20 .. 10, then 9 .. 0.  On return `want` is how many of those at the border
// are kept.
template <class List>
__device__ inline void find_border(const List& list, int32_t m, int32_t* bins, uint32_t& border, int32_t& want) {
  const int tid = threadIdx.x, lane = tid & 63;
  for (int shift = 10; shift >= 0; shift -= 10) {
    bins[tid] = bins[tid + kSelectThreads] = 0;
    __syncthreads();
    for (int i = tid; i - lane < m; i += kSelectThreads) {
      const uint32_t u = i < m ? list[i] : 0;
      const bool in = i < m && (shift == 10 || (u >> 10) == (border >> 10));
      count_in(bins, shift == 10 ? (u >> 10) & 2047 : u & 1023, in);
    }
    __syncthreads();
    const Found f = find_bin(bins, want);
    border |= (uint32_t)f.bin << shift;
    want = f.want;
  }
}

// Short tables (of up to 4096 U tokens): a block per (sequence, KV head).
template <int U>
__global__ __launch_bounds__(kSelectThreads) void select_kernel(EvictArgs a) {
  __shared__ int32_t bins[kBins];
  __shared__ uint32_t list[4 * U * kSelectThreads];
  __shared__ int32_t s_listed;
  const int seq = blockIdx.x / a.c.hkv, head = blockIdx.x % a.c.hkv, tid = threadIdx.x;
  const Select z = open_select(a, seq, head, true);
  if (z.done) return;
  Held<U> x;
  x.load(a, seq, head, 0, z.n);
  int32_t want = z.want, place = 0, equals = 0;
  uint32_t border = 0;
  if (want > 0) {
    bins[tid] = bins[tid + kSelectThreads] = 0;
    if (tid == 0) s_listed = 0;
    __syncthreads();
    x.each(z.lo, z.hi, [&](uint32_t u, bool in) { count_in(bins, u >> 21, in); });
    __syncthreads();
    const Found f = find_bin(bins, want);
    x.each(z.lo, z.hi, [&](uint32_t u, bool in) {
      if (in && (int)(u >> 21) == f.bin) list[atomicAdd(&s_listed, 1)] = u;
    });
    border = (uint32_t)f.bin << 21;
    want = f.want;
    find_border(list, f.held, bins, border, want);
  }
  emit(x, z.kept, z.n, z.lo, z.hi, z.want == 0, border, want, place, equals);
}

// Long tables, a block per (sequence and KV head, chunk), 8192 tokens at a time.  First: the chunk's tokens by their upper 11 bits.
constexpr int kRounds = 2, kStep = 4 * kRounds * kSelectThreads;
__global__ __launch_bounds__(kSelectThreads) void count_kernel(EvictArgs a) {
  __shared__ int32_t bins[kBins];
  const int chunk = blockIdx.y, sh = blockIdx.x, seq = sh / a.c.hkv, head = sh % a.c.hkv, tid = threadIdx.x;
  const Select z = open_select(a, seq, head, chunk == 0);
  if (z.done || z.want == 0 || chunk * a.chunk >= z.n) return;
  bins[tid] = bins[tid + kSelectThreads] = 0;
  __syncthreads();
  for (int t = chunk * a.chunk; t < min((chunk + 1) * a.chunk, z.hi); t += kStep) {
    Held<kRounds> x;
    x.load(a, seq, head, t, z.hi);
    x.each(z.lo, z.hi, [&](uint32_t u, bool in) { count_in(bins, u >> 21, in); });
  }
  __syncthreads();
  int32_t* const to = a.counts + ((int64_t)sh * a.chunks + chunk) * kBins;
  to[tid] = bins[tid];
  to[tid + kSelectThreads] = bins[tid + kSelectThreads];
}

// Second: the chunk's tokens that share the k-th greatest's upper bits, listed behind those of the chunks before; and how many tokens of the chunk lie above them.
__global__ __launch_bounds__(kSelectThreads) void list_kernel(EvictArgs a) {
  __shared__ int32_t bins[kBins];
  __shared__ int32_t s_listed, s_above;
  const int chunk = blockIdx.y, sh = blockIdx.x, seq = sh / a.c.hkv, head = sh % a.c.hkv, tid = threadIdx.x;
  const Select z = open_select(a, seq, head, false);
  if (z.done || z.want == 0 || chunk * a.chunk >= z.n) return;
  const int used = (z.n + a.chunk - 1) / a.chunk;
  const int32_t* const counts = a.counts + (int64_t)sh * a.chunks * kBins;
  Held<kRounds> held;
  held.load(a, seq, head, chunk * a.chunk, z.hi);
  int32_t x = 0, y = 0;
#pragma unroll 8
  for (int c = 0; c < used; ++c) {
    x += counts[(int64_t)c * kBins + tid];
    y += counts[(int64_t)c * kBins + tid + kSelectThreads];
  }
  bins[tid] = x;
  bins[tid + kSelectThreads] = y;
  if (tid == 0) s_listed = s_above = 0;
  __syncthreads();
  const Found f = find_bin(bins, z.want);
  int32_t base = 0;
  for (int c = 0; c < chunk; ++c) base += counts[(int64_t)c * kBins + f.bin];
  const int32_t* const own = counts + (int64_t)chunk * kBins;
  const int32_t above = (tid > f.bin ? own[tid] : 0) + (tid + kSelectThreads > f.bin ? own[tid + kSelectThreads] : 0);
  if (above) atomicAdd(&s_above, above);
  uint32_t* const list = a.list + (int64_t)sh * a.s.max_pages * a.c.page + base;
  for (int t = chunk * a.chunk; t < min((chunk + 1) * a.chunk, z.hi); t += kStep) {
    if (t > chunk * a.chunk) held.load(a, seq, head, t, z.hi);
    held.each(z.lo, z.hi, [&](uint32_t u, bool in) {
      if (in && (int)(u >> 21) == f.bin) list[atomicAdd(&s_listed, 1)] = u;
    });
  }
  __syncthreads();
  if (tid == 0) {
    a.above[(int64_t)sh * a.chunks + chunk] = s_above;
    if (chunk == 0) {
      int32_t* const b = a.border + (int64_t)sh * 4;
      b[0] = f.bin;
      b[1] = f.want;
      b[2] = f.held;
    }
  }
}

// Third: the border among the candidates, and the chunk's part of the list.
__global__ __launch_bounds__(kSelectThreads) void emit_kernel(EvictArgs a) {
  __shared__ int32_t bins[kBins];
  __shared__ int32_t s_above, s_equal;
  const int chunk = blockIdx.y, sh = blockIdx.x, seq = sh / a.c.hkv, head = sh % a.c.hkv, tid = threadIdx.x, lane = tid & 63;
  const Select z = open_select(a, seq, head, false);
  const int c0 = chunk * a.chunk, c1 = min(c0 + a.chunk, z.n);
  if (z.done || c0 >= z.n) return;
  Held<kRounds> x;
  x.load(a, seq, head, c0, z.n);
  // the protected before the chunk
  int32_t place = min(c0, z.lo) + max(c0 - z.hi, 0), want = z.want, equals = 0;
  uint32_t border = 0;
  if (want > 0) {
    const int32_t* const b = a.border + (int64_t)sh * 4;
    const uint32_t* const list = a.list + (int64_t)sh * a.s.max_pages * a.c.page;
    border = (uint32_t)b[0] << 21;
    want = b[1];
    if (tid == 0) s_above = s_equal = 0;
    // candidates of the chunks before, and all of their tokens above the candidates
    const int32_t* const counts = a.counts + (int64_t)sh * a.chunks * kBins;
    int32_t before = lane < chunk ? counts[(int64_t)lane * kBins + b[0]] : 0, over = lane < chunk ? a.above[(int64_t)sh * a.chunks + lane] : 0;
    before = __builtin_amdgcn_readlane(wave_prefix_sum(before), 63);
    place += __builtin_amdgcn_readlane(wave_prefix_sum(over), 63);
    find_border(list, b[2], bins, border, want);
    int32_t above = 0, equal = 0;                          // of the candidates before, those that are kept
#pragma unroll 4
    for (int i = tid; i < before; i += kSelectThreads) {
      const uint32_t u = list[i];
      above += u > border;
      equal += u == border;
    }
    above = __builtin_amdgcn_readlane(wave_prefix_sum(above), 63);
    equal = __builtin_amdgcn_readlane(wave_prefix_sum(equal), 63);
    if (lane == 0 && above) atomicAdd(&s_above, above);
    if (lane == 0 && equal) atomicAdd(&s_equal, equal);
    __syncthreads();
    equals = s_equal;
    place += s_above + min(equals, want);
  }
  for (int t = c0; t < c1; t += kStep) {
    if (t > c0) {
      __syncthreads();                                     // (everybody has read the sums of the tokens before)
      x.load(a, seq, head, t, z.n);
    }
    emit(x, z.kept, min(t + kStep, c1), z.lo, z.hi, z.want == 0, border, want, place, equals);
  }
}
static_assert(kMaxChunks <= 64, "a chunk per lane");

// Lane `from`'s value.
__device__ inline float pick(float x, int from) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), from)); }

// Codes of a word (four tokens of a channel, or four channels of a token) in other units: the largest magnitude (in units 2^16 times as large, which no value leaves), and
// the codes.  A token's scale is multiplied in 2^-16 times.  NaN is no magnitude, and stays.
constexpr float kFar = 0x1p-16f;
// The factor from a token's units to the new page's.  A code other than 0 leaves the format with a factor above 2^18, so only zeros meet a greater one; it stays finite, since 0 times
// infinity is NaN.  (Below 2^-126 all codes become zeros.)
__device__ inline float unit_factor(float scale, float to_units) { return fminf(fmaxf(scale * to_units, 0x1p-126f), 0x1p126f); }
template <int Fmt>
__device__ inline float largest(uint32_t w, float s0, float s1, float s2, float s3, float top) {
  const f32x2 a = decode_half<Fmt, false>(w), b = decode_half<Fmt, true>(w);
  top = fmaxf(fmaxf(top, fabsf(a[0] * s0)), fabsf(a[1] * s1));
  return fmaxf(fmaxf(top, fabsf(b[0] * s2)), fabsf(b[1] * s3));
}
template <int Fmt>
__device__ inline uint32_t in_units(uint32_t w, float s0, float s1, float s2, float s3) {
  const f32x2 a = decode_half<Fmt, false>(w), b = decode_half<Fmt, true>(w);
  return encode_half<Fmt, true>(b[0] * s2, b[1] * s3, encode_half<Fmt, false>(a[0] * s0, a[1] * s1, 0));
}

// A wave per (new page, KV head, keys or values).  Lane j first finds where slot j's token lies and its scale, so that the tokens' codes can all be asked for at
// once; they stay in registers until the page's scale is known.  Keys move as 16 bytes of a row; of the values, which lie 16 tokens together, a lane takes its channels'
// 16 bytes and picks the token's.  Groups: of 16 slots in a page.
template <int D, int Fmt, int Groups>
__global__ __launch_bounds__(256) void move_kernel(EvictArgs a) {
  constexpr int P = Groups * kGroup, kPer = (P + 63) / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int job = blockIdx.y * 4 + wave;
  if (job >= 2 * a.c.hkv) return;
  const int head = job >> 1, seq = blockIdx.x / a.places, place = blockIdx.x % a.places;
  const bool value = job & 1;
  const int n_new = min(cached(a, seq), a.budget), count = min(P, n_new - place * P);
  if (count <= 0) return;
  const int32_t page = a.new_pages[(int64_t)seq * a.max_new + place];
  if ((uint32_t)page >= (uint32_t)a.c.n_pages) return;
  const int32_t* const kept = a.kept + ((int64_t)seq * a.c.hkv + head) * a.budget + place * P;
  const int64_t block = block_of(a.c, page, head);
  // slot lane + 64 i: token's page, slot there, scale; past the last token and where a page is missing: scale 0
  int32_t from_page[kPer], from_slot[kPer];
  float scale[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int j = lane + 64 * i;
    const int t = j < count ? kept[j] : 0;
    const int32_t p = j < count ? page_at(a.s, a.c, seq, t >> a.c.log_page) : -1;
    from_page[i] = max(p, 0);
    from_slot[i] = t & (P - 1);
    const int64_t b = block_of(a.c, from_page[i], head);
    const float s = (value ? a.c.v_scale : a.c.k_scale)[b];
    scale[i] = p < 0 ? 0.f : s;
    if (!value && j < P) a.c.weight[block * P + j] = p < 0 ? 0.f : a.c.weight[b * P + from_slot[i]];
  }
  uint8_t* const codes = (value ? a.c.v : a.c.k) + block * P * D;
  float top = 0.f;
  if (!value) {
    constexpr int LPR = D / 16, RPI = 64 / LPR, N = (P + RPI - 1) / RPI;       // lanes of a row, rows of a load, loads
    const int sub = lane / LPR, ch = 16 * (lane % LPR);
    u32x4 w[N];
    float s[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int slot = min(RPI * i + sub, P - 1);
      const int32_t fp = __shfl(from_page[RPI * i / 64], slot & 63), fs = __shfl(from_slot[RPI * i / 64], slot & 63);
      s[i] = __shfl(scale[RPI * i / 64], slot & 63);
      w[i] = *reinterpret_cast<const u32x4*>(a.c.k + (block_of(a.c, fp, head) * P + fs) * D + ch);
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w[i][j] = s[i] == 0.f ? 0u : w[i][j];
        const float f = s[i] * kFar;
        top = largest<Fmt>(w[i][j], f, f, f, f, top);
      }
    top = wave_maxf(top);
    const int e = exponent_for<Fmt>(top, 16);
    if (lane == 0) a.c.k_scale[block] = power2(e);
    const float to_units = power2(-e);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int slot = RPI * i + sub;
      const float f = unit_factor(s[i], to_units);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i][j] = in_units<Fmt>(w[i][j], f, f, f, f);
      if (slot < P) *reinterpret_cast<u32x4*>(codes + slot * D + ch) = w[i];
    }
  } else {
    // The word of four tokens that holds the token is asked for, for 32 tokens at once: a group's lines are fetched once, by whichever token comes first, and nearly every group of a
    // long sequence cut to an eighth has one.  4 sequences of up to 131072 tokens to 16384, 8 heads: 290 MB read and 124 written in 95 us, 4.4 TB/s, where a large copy reaches 4.9;
    // values alone 74 us, keys alone 30.  (Two waves a page and half the chain of loads: 91.  Single bytes of channels that lie 32 bytes apart are a request each: 131.)
    constexpr int NC = D / 64, kBatch = P < 32 ? P : 32;   // channels of a lane: lane, lane + 64; tokens on their way
    u32x4 w[Groups][NC];
#pragma unroll
    for (int b = 0; b < P / kBatch; ++b) {
      uint32_t x[kBatch][NC];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int slot = kBatch * b + j;
        const int32_t fp = __builtin_amdgcn_readlane(from_page[slot / 64], slot & 63), at = __builtin_amdgcn_readlane(from_slot[slot / 64], slot & 63);
        const uint8_t* v = a.c.v + (block_of(a.c, fp, head) * P + (at & ~(kGroup - 1))) * D + (at & 12);
#pragma unroll
        for (int c = 0; c < NC; ++c) x[j][c] = *reinterpret_cast<const uint32_t*>(v + 16 * lane + 1024 * c);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int slot = kBatch * b + j, g = slot / kGroup, q = slot % kGroup / 4, byte = slot % 4;
        const int32_t at = __builtin_amdgcn_readlane(from_slot[slot / 64], slot & 63);
        // byte `byte` of the result's word is byte at % 4 of the token's word; the others stay
        const uint32_t sel = (0x07060504u & ~(0xffu << (8 * byte))) | (uint32_t)(at & 3) << (8 * byte);
#pragma unroll
        for (int c = 0; c < NC; ++c) w[g][c][q] = __builtin_amdgcn_perm(byte == 0 ? 0u : w[g][c][q], x[j][c], sel);
      }
    }
#pragma unroll
    for (int g = 0; g < Groups; ++g)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float s[4];
        uint32_t gone = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int slot = g * kGroup + 4 * q + j;
          s[j] = pick(scale[slot / 64], slot & 63);
          gone |= s[j] == 0.f ? 0xffu << (8 * j) : 0u;
          s[j] *= kFar;
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          w[g][c][q] &= ~gone;
          top = largest<Fmt>(w[g][c][q], s[0], s[1], s[2], s[3], top);
        }
      }
    top = wave_maxf(top);
    const int e = exponent_for<Fmt>(top, 16);
    if (lane == 0) a.c.v_scale[block] = power2(e);
    const float to_units = power2(-e);
#pragma unroll
    for (int g = 0; g < Groups; ++g) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float s[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int slot = g * kGroup + 4 * q + j;
          s[j] = unit_factor(pick(scale[slot / 64], slot & 63), to_units);
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) w[g][c][q] = in_units<Fmt>(w[g][c][q], s[0], s[1], s[2], s[3]);
      }
#pragma unroll
      for (int c = 0; c < NC; ++c) *reinterpret_cast<u32x4*>(codes + (g * D + lane + 64 * c) * kGroup) = w[g][c];
    }
  }
}

template <int D, int Fmt>
void launch_move(const EvictArgs& a, dim3 grid, hipStream_t st) {
  auto kernel = a.c.page == 16 ? move_kernel<D, Fmt, 1> : a.c.page == 32 ? move_kernel<D, Fmt, 2> : a.c.page == 64 ? move_kernel<D, Fmt, 4> : move_kernel<D, Fmt, 8>;
  kernel<<<grid, dim3(256), 0, st>>>(a);
}

// Where the parts of scratch lie.  A table of up to kListed tokens needs none of them.
struct EvictPlan { int32_t chunk, chunks; size_t counts, list, above, border, bytes; };
EvictPlan plan_evict(const CacheView& c, int32_t n_seqs, int32_t max_pages) {
  EvictPlan p = {};
  const int64_t room = (int64_t)max_pages * c.page, lists = (int64_t)n_seqs * c.hkv;
  if (room <= kListed) { p.bytes = 256; return p; }
  p.chunk = (int32_t)(((room + kMaxChunks - 1) / kMaxChunks + kStep - 1) / kStep * kStep);
  p.chunks = (int32_t)((room + p.chunk - 1) / p.chunk);
  p.list = pad_to((size_t)lists * p.chunks * kBins * 4, 256);
  p.above = p.list + pad_to((size_t)lists * room * 4, 256);
  p.border = p.above + pad_to((size_t)lists * p.chunks * 4, 256);
  p.bytes = p.border + pad_to((size_t)lists * 16, 256);
  return p;
}

int check_lists(const char* who, const CacheView& c, int32_t n_seqs) {
  if (!fits_axis((int64_t)n_seqs * c.hkv, kSelectThreads)) return fail(FCP_ERR_UNSUPPORTED, "%s: 2^22 KV heads of all sequences or more", who);
  return FCP_OK;
}

}  // namespace

size_t evict_scratch_bytes(const char* who, const CacheView& c, int32_t n_seqs, int32_t max_pages) {
  return check_lists(who, c, n_seqs) ? 0 : plan_evict(c, n_seqs, max_pages).bytes;
}

}  // namespace fcp

extern "C" int fcp_cache_evict(const fcp_cache* cache, const int32_t* pages, const int32_t* kv_len, int32_t n_seqs, int32_t max_pages,
                               const int32_t* new_pages, int32_t max_new_pages, int32_t budget, int32_t n_first, int32_t n_recent, int32_t* kept,
                               int32_t* new_len, void* scratch, size_t scratch_bytes, void* stream) {
  using namespace fcp;
  clear_error();
  const char* who = "fcp_cache_evict";
  EvictArgs a = {};
  if (int rc = check_cache(who, cache, true, &a.c)) return rc;
  if (int rc = check_seqs(who, a.c, nullptr, false, kv_len, pages, n_seqs, max_pages, 0)) return rc;
  if (n_first < 0 || n_recent < 0 || budget < 1 || (int64_t)n_first + n_recent > budget)
    return fail(FCP_ERR_INVALID_ARG, "%s: budget must be at least 1 and n_first + n_recent, which must not be negative", who);
  if (max_new_pages < 0) return fail(FCP_ERR_INVALID_ARG, "%s: negative size", who);
  if (n_seqs == 0) return FCP_OK;
  if (!kept || !new_len || (max_new_pages > 0 && !new_pages)) return fail(FCP_ERR_INVALID_ARG, "%s: null argument", who);
  if (new_len == kv_len) return fail(FCP_ERR_INVALID_ARG, "%s: new_len must not be kv_len", who);
  const int64_t room = (int64_t)max_pages * a.c.page, most = room < budget ? room : budget;
  if ((int64_t)max_new_pages * a.c.page < most)
    return fail(FCP_ERR_CAPACITY, "%s: %d new pages of %d tokens for up to %lld", who, max_new_pages, a.c.page, (long long)most);
  if (!scratch || (uintptr_t)scratch % 256) return fail(FCP_ERR_INVALID_ARG, "%s: scratch must be 256-byte aligned", who);
  const EvictPlan p = plan_evict(a.c, n_seqs, max_pages);
  const size_t need = p.bytes;
  if (scratch_bytes < need) return fail(FCP_ERR_CAPACITY, "%s: scratch has %zu bytes, %zu are needed", who, scratch_bytes, need);
  const int64_t use = (most + a.c.page - 1) / a.c.page;      // (further entries of new_pages are not used)
  if (int rc = check_lists(who, a.c, n_seqs)) return rc;
  if (!fits_axis((int64_t)n_seqs * use, 256)) return fail(FCP_ERR_UNSUPPORTED, "%s: 2^24 new pages of all sequences or more", who);
  a.s = {nullptr, kv_len, pages, n_seqs, max_pages, 0};
  a.new_pages = new_pages;
  a.max_new = max_new_pages;
  a.places = (int32_t)use;
  a.budget = budget;
  a.first = n_first;
  a.recent = n_recent;
  a.kept = kept;
  a.new_len = new_len;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (p.chunks == 0) {
    auto kernel = room <= 4 * kSelectThreads ? select_kernel<1> : select_kernel<4>;
    kernel<<<dim3((unsigned)(n_seqs * a.c.hkv)), dim3(kSelectThreads), 0, st>>>(a);
  } else {
    char* const area = static_cast<char*>(scratch);
    a.chunk = p.chunk;
    a.chunks = p.chunks;
    a.counts = reinterpret_cast<int32_t*>(area + p.counts);
    a.list = reinterpret_cast<uint32_t*>(area + p.list);
    a.above = reinterpret_cast<int32_t*>(area + p.above);
    a.border = reinterpret_cast<int32_t*>(area + p.border);
    const dim3 grid((unsigned)(n_seqs * a.c.hkv), (unsigned)p.chunks);
    count_kernel<<<grid, dim3(kSelectThreads), 0, st>>>(a);
    FCP_HIP_CHECK(hipGetLastError());
    list_kernel<<<grid, dim3(kSelectThreads), 0, st>>>(a);
    FCP_HIP_CHECK(hipGetLastError());
    emit_kernel<<<grid, dim3(kSelectThreads), 0, st>>>(a);
  }
  FCP_HIP_CHECK(hipGetLastError());
  if (use == 0) return FCP_OK;
  const dim3 grid((unsigned)(n_seqs * use), (unsigned)((2 * a.c.hkv + 3) / 4));
  const bool e4m3 = cache->format == FCP_CACHE_E4M3;
  (cache->head_dim == 128 ? (e4m3 ? launch_move<128, kE4m3> : launch_move<128, kInt8>) : (e4m3 ? launch_move<64, kE4m3> : launch_move<64, kInt8>))(a, grid, st);
  FCP_HIP_CHECK(hipGetLastError());
  return FCP_OK;
}
