// fcp_cache_append: new key and value rows quantised into a paged 8-bit cache, and the checks that all calls of the cache share.
//
// A unit is one page that gets new tokens, for one KV head, keys or values: a wave works it alone, since all of the page's codes share one
// scale 2^e, e the least exponent that holds the largest magnitude.  Reads 2 bytes and writes 1 per element: the memory bounds long prompts, the chain
// table -> page -> scale -> codes single tokens.
// The page's new rows stay in registers while their scale is found.  Key rows are written as they come; of the values a lane holds a group of 16 tokens of two
// channels, which in the cache's order are 16 bytes for each, so the transposition costs nothing.
// 24 prompts of up to 4001 tokens, 8 heads of 128 channels, int8, 199 MB: 46 us, 4.3 TB/s, where a large copy reaches 4.9.  One token of each of 64 sequences: 6.6 us.
// Pages of 128 tokens take 221 to 245 registers for a page's rows, two waves a SIMD instead of three or four: the prompts 59 us.
#include "fcp_cache.h"

namespace fcp {
namespace {

struct AppendArgs {
  CacheView c;
  SeqView s;
  const __bf16* x[2];                              // new keys, values
  int64_t row[2];
  int32_t units;
};

// Which sequence holds unit u: units are numbered so that a sequence's begin at cu / page + 2 seq, which leaves every sequence room for all pages that its rows
// can touch, (n - 1) / page + 2 at most.  The numbers grow with the sequence: a search, 64 ways at a time.
__device__ inline int64_t first_unit(const SeqView& s, int log_page, int seq) { return (int64_t)(min(max(s.cu[seq], 0), s.n_rows) >> log_page) + 2 * (int64_t)seq; }
struct UnitSeq { int32_t seq; int64_t first_unit; SeqSizes z; };
__device__ inline UnitSeq seq_of_unit(const SeqView& s, int log_page, int u) {
  const int lane = threadIdx.x & 63;
  if (s.n_seqs <= 64) {
    // a sequence per lane, all of its numbers at once: with the search and then its sizes a single token's chain of loads is one longer
    const int i = min(lane, s.n_seqs - 1);
    const SeqSizes z = seq_sizes(s, i, 1 << log_page);
    const int64_t first = first_unit(s, log_page, i);
    const int k = max((int)__popcll(__ballot(lane < s.n_seqs && first <= u)) - 1, 0);
    return {k, (int64_t)__builtin_amdgcn_readlane((int32_t)first, k), {__builtin_amdgcn_readlane(z.row0, k), __builtin_amdgcn_readlane(z.n, k), __builtin_amdgcn_readlane(z.len, k)}};
  }
  int lo = 0, n = s.n_seqs;                        // the sequence is in lo .. lo + n - 1
  while (n > 1) {
    const int step = (n + 63) / 64, at = lo + lane * step;
    const bool below = at < lo + n && first_unit(s, log_page, at) <= u;
    const int k = __popcll(__ballot(below)) - 1;   // (true for a run of lanes from the first on; lane 0's always is)
    const int next = lo + max(k, 0) * step;
    n = min(step, lo + n - next);
    lo = next;
  }
  return {lo, first_unit(s, log_page, lo), seq_sizes(s, lo, 1 << log_page)};
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Largest of the finite magnitudes in a word of two bf16; these are ordered as integers.
__device__ inline uint32_t finite2(uint32_t w) {
  const uint32_t p = w & 0x7fffu, q = (w >> 16) & 0x7fffu;
  return max(p < 0x7f80u ? p : 0u, q < 0x7f80u ? q : 0u);
}
__device__ inline uint32_t wave_max16(uint32_t x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, d));
  return x;
}
// Two bf16 as codes in the lower 16 bits.  Odd: there are values that are not finite.
template <int Fmt, bool Odd>
__device__ inline uint32_t code2(uint32_t w, float to_units) {
  const float a = __uint_as_float(w << 16) * to_units, b = __uint_as_float(w & 0xffff0000u) * to_units;
  return Odd ? encode2<Fmt>(a, b) : encode_half<Fmt, false>(a, b, 0) & 0xffffu;
}

// The largest finite magnitude of a wave's words w[0 .. N - 1] of bf16 pairs as a float; odd: some are not finite.
template <int N>
__device__ inline float top_of(const uint32_t (&w)[N], bool& odd) {
  u16x2 t = {0, 0};
#pragma unroll
  for (int i = 0; i < N; ++i) t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
  uint32_t top = wave_max16(max((uint32_t)t[0], (uint32_t)t[1]));
  odd = top >= 0x7f80u;
  if (odd) {                                       // rare: once more without them
    top = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, finite2(w[i]));
    top = wave_max16(top);
  }
  return __uint_as_float(top << 16);
}

// Exponent of the page's scale after new values of magnitude `top`, and the earlier tokens' units in the new ones (1: they stay as they are).
template <int Fmt>
__device__ inline int grow(float top, bool earlier, float* scale, float& again) {
  int e = exponent_for<Fmt>(top);
  again = 1.f;
  if (earlier) {
    const int before = exponent_of(*scale);
    e = max(e, before);
    again = power2(before - e);
  }
  if ((threadIdx.x & 63) == 0) *scale = power2(e);
  return e;
}

template <int D, int Fmt, int Groups>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
  constexpr int P = Groups * kGroup;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int job = blockIdx.y * 4 + wave;           // (KV head, keys or values)
  if (job >= 2 * a.c.hkv) return;
  const int head = job >> 1, u = blockIdx.x;
  const bool value = job & 1;
  const UnitSeq of = seq_of_unit(a.s, a.c.log_page, u);
  const int seq = of.seq;
  const SeqSizes z = of.z;
  // tokens len - n .. len - 1; those before the first slot (a caller's error) are not written
  const int64_t first = (int64_t)z.len - z.n;
  if (z.n == 0 || z.len == 0) return;
  const int32_t place = (int32_t)((first > 0 ? first : 0) >> a.c.log_page) + (int32_t)(u - of.first_unit);
  const int64_t t0 = (int64_t)place * P;
  if (t0 >= z.len) return;
  const int32_t page = page_at(a.s, a.c, seq, place);
  if (page < 0) return;
  const int lo = __builtin_amdgcn_readfirstlane((int)max(first - t0, (int64_t)0)), hi = __builtin_amdgcn_readfirstlane((int)min((int64_t)P, z.len - t0));
  const int64_t row = a.row[value];
  // row of slot j: row0 + (t0 + j - first)
  const __bf16* const x = a.x[value] + ((int64_t)z.row0 + t0 - first) * row + head * D;
  const int64_t block = block_of(a.c, page, head);
  uint8_t* const codes = (value ? a.c.v : a.c.k) + block * P * D;
  bool odd;
  float again;
  if (!value) {
    // a lane: eight channels of a row, every RPI-th row.  Slots that get no new row repeat the nearest one that does, which changes no maximum.
    constexpr int LPR = D / 8, RPI = 64 / LPR, N = P / RPI;
    const int sub = lane / LPR, ch = 8 * (lane % LPR);
    uint32_t w[4 * N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      u32x4 r = {0, 0, 0, 0};
      if (RPI * i < hi && RPI * (i + 1) > lo) r = *reinterpret_cast<const u32x4*>(x + min(max(RPI * i + sub, lo), hi - 1) * row + ch);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[4 * i + j] = r[j];
    }
    const float top = top_of(w, odd);
    const int e = grow<Fmt>(top, lo > 0, a.c.k_scale + block, again);
    const float to_units = power2(-e);
    if (again != 1.f)
#pragma unroll 1
      for (int j = sub; j < lo; j += RPI) {
        uint32_t* const c = reinterpret_cast<uint32_t*>(codes + j * D + ch);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const f32x2 f = decode_half<Fmt, false>(c[q]), g = decode_half<Fmt, true>(c[q]);
          c[q] = encode2<Fmt>(f[0] * again, f[1] * again) | encode2<Fmt>(g[0] * again, g[1] * again) << 16;
        }
      }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int slot = RPI * i + sub;
      u32x2 c;
#pragma unroll
      for (int q = 0; q < 2; ++q)
        c[q] = odd ? code2<Fmt, true>(w[4 * i + 2 * q], to_units) | code2<Fmt, true>(w[4 * i + 2 * q + 1], to_units) << 16
                   : code2<Fmt, false>(w[4 * i + 2 * q], to_units) | code2<Fmt, false>(w[4 * i + 2 * q + 1], to_units) << 16;
      if (slot >= lo && slot < hi) *reinterpret_cast<u32x2*>(codes + slot * D + ch) = c;
    }
    if (a.c.weight)
      for (int j = lo + lane; j < hi; j += 64) a.c.weight[block * P + j] = 0.f;
  } else {
    // a lane: two neighbouring channels of all tokens (64 channels: of every second group), which the cache holds as 16 bytes a group each
    constexpr int LPR = D / 2, TPW = 64 / LPR, N = (Groups + TPW - 1) / TPW;
    const int sub = lane / LPR, ch = 2 * (lane % LPR);
    uint32_t w[N * kGroup];
    u32x4 old[N][2];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int g = min(sub + TPW * i, Groups - 1);
      const bool any = TPW * i * kGroup < hi && TPW * (i + 1) * kGroup > lo;
      if (any) {
#pragma unroll
        for (int j = 0; j < kGroup; ++j) w[kGroup * i + j] = *reinterpret_cast<const uint32_t*>(x + min(max(g * kGroup + j, lo), hi - 1) * row + ch);
      } else {
#pragma unroll
        for (int j = 0; j < kGroup; ++j) w[kGroup * i + j] = 0;
      }
      old[i][0] = old[i][1] = u32x4{0, 0, 0, 0};
      if (any && (TPW * i * kGroup < lo || TPW * (i + 1) * kGroup > hi)) {                // codes that stay
        const u32x4* const c = reinterpret_cast<const u32x4*>(codes + (g * D + ch) * kGroup);
        old[i][0] = c[0];
        old[i][1] = c[1];
      }
    }
    const float top = top_of(w, odd);
    const int e = grow<Fmt>(top, lo > 0, a.c.v_scale + block, again);
    const float to_units = power2(-e);
    if (again != 1.f) {
      // the earlier tokens' groups in the new units (of a group with new tokens: below)
#pragma unroll 1
      for (int g = sub; (g + 1) * kGroup <= lo; g += TPW) {
        u32x4* const c = reinterpret_cast<u32x4*>(codes + (g * D + ch) * kGroup);
        if (TPW * (g / TPW + 1) * kGroup > lo) continue;   // (its step is below)
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          u32x4 o = c[m];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const f32x2 f = decode_half<Fmt, false>(o[q]), h = decode_half<Fmt, true>(o[q]);
            o[q] = encode2<Fmt>(f[0] * again, f[1] * again) | encode2<Fmt>(h[0] * again, h[1] * again) << 16;
          }
          c[m] = o;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int g = sub + TPW * i;
      if (TPW * i * kGroup < hi && TPW * (i + 1) * kGroup > lo) {
        u32x4 c0, c1;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t t[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t r = w[kGroup * i + 4 * q + j];
            t[j] = odd ? code2<Fmt, true>(r, to_units) : code2<Fmt, false>(r, to_units);
          }
          // bytes of the first channel, of the second
          const uint32_t p = __builtin_amdgcn_perm(t[1], t[0], 0x05010400u), r = __builtin_amdgcn_perm(t[3], t[2], 0x05010400u);
          c0[q] = (p & 0xffffu) | r << 16;
          c1[q] = (p >> 16) | (r & 0xffff0000u);
        }
        if (TPW * i * kGroup < lo || TPW * (i + 1) * kGroup > hi) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int s0 = g * kGroup + 4 * q;     // slots s0 .. s0 + 3: the first `before` hold earlier tokens, from `end` on nothing new
            const int before = min(max(lo - s0, 0), 4), end = min(max(hi - s0, 0), 4);
            const uint32_t early = before == 4 ? ~0u : (1u << (8 * before)) - 1, upto = end == 4 ? ~0u : (1u << (8 * end)) - 1, fresh_bytes = upto & ~early;
            uint32_t o0 = old[i][0][q], o1 = old[i][1][q];
            if (again != 1.f) {
              const f32x2 f0 = decode_half<Fmt, false>(o0), h0 = decode_half<Fmt, true>(o0), f1 = decode_half<Fmt, false>(o1), h1 = decode_half<Fmt, true>(o1);
              const uint32_t n0 = encode2<Fmt>(f0[0] * again, f0[1] * again) | encode2<Fmt>(h0[0] * again, h0[1] * again) << 16;
              const uint32_t n1 = encode2<Fmt>(f1[0] * again, f1[1] * again) | encode2<Fmt>(h1[0] * again, h1[1] * again) << 16;
              o0 = (n0 & early) | (o0 & ~early);
              o1 = (n1 & early) | (o1 & ~early);
            }
            c0[q] = (c0[q] & fresh_bytes) | (o0 & ~fresh_bytes);
            c1[q] = (c1[q] & fresh_bytes) | (o1 & ~fresh_bytes);
          }
        }
        if (g < Groups) {
          u32x4* const c = reinterpret_cast<u32x4*>(codes + (g * D + ch) * kGroup);
          c[0] = c0;
          c[1] = c1;
        }
      }
    }
  }
}

template <int D, int Fmt>
void launch_append(const AppendArgs& a, dim3 grid, hipStream_t st) {
  auto kernel = a.c.page == 16 ? append_kernel<D, Fmt, 1> : a.c.page == 32 ? append_kernel<D, Fmt, 2> : a.c.page == 64 ? append_kernel<D, Fmt, 4> : append_kernel<D, Fmt, 8>;
  kernel<<<grid, dim3(256), 0, st>>>(a);
}

}  // namespace

int check_cache(const char* who, const fcp_cache* cache, bool needs_weight, CacheView* out) {
  if (!cache) return fail(FCP_ERR_INVALID_ARG, "%s: null cache", who);
  const fcp_cache& c = *cache;
  if (!c.k || !c.v || !c.k_scale || !c.v_scale || c.n_pages < 1 || c.hkv < 1)
    return fail(FCP_ERR_INVALID_ARG, "%s: the cache has a null pointer or no pages or heads", who);
  if (needs_weight && !c.weight) return fail(FCP_ERR_INVALID_ARG, "%s: the cache has no weights", who);
  if (c.head_dim != 64 && c.head_dim != 128) return fail(FCP_ERR_UNSUPPORTED, "%s: head_dim %d is not 64 or 128", who, c.head_dim);
  int log_page = 4;
  while (log_page < 7 && (1 << log_page) != c.page_tokens) ++log_page;
  if ((1 << log_page) != c.page_tokens) return fail(FCP_ERR_UNSUPPORTED, "%s: page_tokens %d is not 16, 32, 64 or 128", who, c.page_tokens);
  if (c.format != FCP_CACHE_E4M3 && c.format != FCP_CACHE_INT8) return fail(FCP_ERR_UNSUPPORTED, "%s: format %d is not known", who, c.format);
  if (c.hkv > 4096) return fail(FCP_ERR_UNSUPPORTED, "%s: %d KV heads, at most 4096", who, c.hkv);
  if ((uintptr_t)c.k % 16 || (uintptr_t)c.v % 16 || (uintptr_t)c.weight % 16 || (uintptr_t)c.k_scale % 4 || (uintptr_t)c.v_scale % 4)
    return fail(FCP_ERR_INVALID_ARG, "%s: the cache's arrays are not aligned", who);
  *out = {static_cast<uint8_t*>(c.k), static_cast<uint8_t*>(c.v), c.k_scale, c.v_scale, c.weight, c.n_pages, c.hkv, c.page_tokens, log_page};
  return FCP_OK;
}

int check_sizes(const char* who, const CacheView& c, int32_t n_seqs, int32_t max_pages, int32_t n_rows) {
  if (n_seqs < 0 || max_pages < 0 || n_rows < 0) return fail(FCP_ERR_INVALID_ARG, "%s: negative size", who);
  if (n_seqs > 1 << 20) return fail(FCP_ERR_UNSUPPORTED, "%s: more than 2^20 sequences", who);
  if ((int64_t)max_pages * c.page > 1 << 30) return fail(FCP_ERR_UNSUPPORTED, "%s: a table of more than 2^30 tokens", who);
  return FCP_OK;
}

int check_seqs(const char* who, const CacheView& c, const int32_t* cu, bool needs_cu, const int32_t* kv_len, const int32_t* pages, int32_t n_seqs, int32_t max_pages, int32_t n_rows) {
  if (int rc = check_sizes(who, c, n_seqs, max_pages, n_rows)) return rc;
  if (n_seqs > 0 && ((needs_cu && !cu) || !kv_len || (max_pages > 0 && !pages))) return fail(FCP_ERR_INVALID_ARG, "%s: null argument", who);
  return FCP_OK;
}

}  // namespace fcp

extern "C" int fcp_cache_append(const fcp_cache* cache, const void* k, int64_t k_row, const void* v, int64_t v_row, int32_t n_rows,
                                const int32_t* cu_seqlens, const int32_t* kv_len, const int32_t* pages, int32_t n_seqs, int32_t max_pages, void* stream) {
  using namespace fcp;
  clear_error();
  const char* who = "fcp_cache_append";
  AppendArgs a = {};
  if (int rc = check_cache(who, cache, false, &a.c)) return rc;
  if (int rc = check_seqs(who, a.c, cu_seqlens, true, kv_len, pages, n_seqs, max_pages, n_rows)) return rc;
  if (n_rows == 0 || n_seqs == 0 || max_pages == 0) return FCP_OK;
  if (!k || !v) return fail(FCP_ERR_INVALID_ARG, "%s: null argument", who);
  const int64_t width = (int64_t)cache->hkv * cache->head_dim;
  if (k_row < width || v_row < width || k_row % 8 || v_row % 8 || (uintptr_t)k % 16 || (uintptr_t)v % 16)
    return fail(FCP_ERR_INVALID_ARG, "%s: rows must be at least hkv * head_dim elements apart, a multiple of 8, and 16-byte aligned", who);
  a.s = {cu_seqlens, kv_len, pages, n_seqs, max_pages, n_rows};
  a.x[0] = static_cast<const __bf16*>(k);
  a.x[1] = static_cast<const __bf16*>(v);
  a.row[0] = k_row;
  a.row[1] = v_row;
  a.units = (n_rows >> a.c.log_page) + 2 * n_seqs;
  if (!fits_axis(a.units, 256)) return fail(FCP_ERR_UNSUPPORTED, "%s: rows that may lie in 2^24 pages or more", who);
  hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)a.units, (unsigned)((2 * a.c.hkv + 3) / 4));
  const bool e4m3 = cache->format == FCP_CACHE_E4M3;
  (cache->head_dim == 128 ? (e4m3 ? launch_append<128, kE4m3> : launch_append<128, kInt8>) : (e4m3 ? launch_append<64, kE4m3> : launch_append<64, kInt8>))(a, grid, st);
  FCP_HIP_CHECK(hipGetLastError());
  return FCP_OK;
}
