// fcp_cache_append: new key and value rows quantised into a paged 8-bit cache, and the checks that all calls of the cache share.
//
// A unit is one page that gets new tokens, for one KV head, keys or values: a wave works it alone, since all of the page's codes share one
// scale 2^e, e the least exponent that holds the largest magnitude.  Reads 2 bytes and writes 1 per element: the memory bounds long prompts, the chain
// table -> page -> scale -> codes single tokens.
// A lane owns two neighbouring channels.  Key rows are written as they come; for the values a lane collects a group of 16 tokens, which in the
// cache's order is 16 bytes for each of its channels, so the transposition costs nothing.
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
__device__ inline int seq_of_unit(const SeqView& s, int log_page, int u) {
  int lo = 0, n = s.n_seqs;                        // the sequence is in lo .. lo + n - 1
  while (n > 1) {
    const int step = (n + 63) / 64, at = lo + (int)(threadIdx.x & 63) * step;
    const bool below = at < lo + n && first_unit(s, log_page, at) <= u;
    const int k = __popcll(__ballot(below)) - 1;   // (true for a run of lanes from the first on; lane 0's always is)
    const int next = lo + max(k, 0) * step;
    n = min(step, lo + n - next);
    lo = next;
  }
  return lo;
}

template <int D, int Fmt>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
  constexpr int LPR = D / 2, TPW = 64 / LPR;       // lanes of a row; rows (keys), groups (values) a wave works at a time
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int job = blockIdx.y * 4 + wave;           // (KV head, keys or values)
  if (job >= 2 * a.c.hkv) return;
  const int head = job >> 1, P = a.c.page, u = blockIdx.x;
  const bool value = job & 1;
  const int seq = seq_of_unit(a.s, a.c.log_page, u);
  const SeqSizes z = seq_sizes(a.s, seq, P);
  // tokens len - n .. len - 1; those before the first slot (a caller's error) are not written
  const int64_t first = (int64_t)z.len - z.n;
  if (z.n == 0 || z.len == 0) return;
  const int32_t place = (int32_t)((first > 0 ? first : 0) >> a.c.log_page) + (int32_t)(u - first_unit(a.s, a.c.log_page, seq));
  const int64_t t0 = (int64_t)place << a.c.log_page;
  if (t0 >= z.len) return;
  const int32_t page = page_at(a.s, a.c, seq, place);
  if (page < 0) return;
  const int lo = (int)max(first - t0, (int64_t)0), hi = (int)min((int64_t)P, z.len - t0);
  const int sub = lane / LPR, ch = 2 * (lane % LPR);
  // row of slot j: row0 + (t0 + j - first)
  const __bf16* const x = a.x[value] + ((int64_t)z.row0 + t0 - first) * a.row[value] + head * D + ch;
  const int64_t block = block_of(a.c, page, head);
  uint8_t* const codes = (value ? a.c.v : a.c.k) + block * P * D;
  float* const scale = (value ? a.c.v_scale : a.c.k_scale) + block;

  // largest finite magnitude: bf16 magnitudes are ordered as integers
  uint32_t top = 0;
#pragma unroll 8
  for (int j = lo + sub; j < hi; j += TPW) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(x + j * a.row[value]);
    const uint32_t p = w & 0x7fffu, q = (w >> 16) & 0x7fffu;
    top = max(top, max(p < 0x7f80u ? p : 0u, q < 0x7f80u ? q : 0u));
  }
  int e = exponent_for<Fmt>(wave_maxf(__uint_as_float(top << 16)));
  float again = 1.f;                               // units of the earlier tokens' codes, in new units
  if (lo > 0) {
    const int before = exponent_of(*scale);
    e = max(e, before);
    again = power2(before - e);
  }
  const float to_units = power2(-e);
  if (lane == 0) *scale = power2(e);

  if (!value) {
    if (again != 1.f)
      for (int j = sub; j < lo; j += TPW) {
        uint16_t* const c = reinterpret_cast<uint16_t*>(codes + j * D + ch);
        const f32x2 f = decode2<Fmt>(*c);
        *c = (uint16_t)encode2<Fmt>(f[0] * again, f[1] * again);
      }
#pragma unroll 8
    for (int j = lo + sub; j < hi; j += TPW) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(x + j * a.row[0]);
      *reinterpret_cast<uint16_t*>(codes + j * D + ch) = (uint16_t)encode2<Fmt>(__uint_as_float(w << 16) * to_units, __uint_as_float(w & 0xffff0000u) * to_units);
    }
    if (a.c.weight)
      for (int j = lo + lane; j < hi; j += 64) a.c.weight[block * P + j] = 0.f;
  } else {
    for (int g = sub; g * kGroup < hi; g += TPW) {
      const int j0 = g * kGroup;
      if (j0 + kGroup <= lo && again == 1.f) continue;
      u32x4* const c = reinterpret_cast<u32x4*>(codes + (g * D + ch) * kGroup);     // the two channels' 16 bytes lie next to each other
      u32x4 w0 = {0, 0, 0, 0}, w1 = {0, 0, 0, 0};
      if (j0 < lo || j0 + kGroup > hi) { w0 = c[0]; w1 = c[1]; }                    // codes that stay
#pragma unroll
      for (int j = 0; j < kGroup; ++j) {
        const int slot = j0 + j, word = j / 4, shift = 8 * (j % 4);
        uint32_t two = ((w0[word] >> shift) & 0xffu) | (((w1[word] >> shift) & 0xffu) << 8);
        if (slot < lo) {
          if (again != 1.f) {
            const f32x2 f = decode2<Fmt>(two);
            two = encode2<Fmt>(f[0] * again, f[1] * again);
          }
        } else if (slot < hi) {
          const uint32_t r = *reinterpret_cast<const uint32_t*>(x + slot * a.row[1]);
          two = encode2<Fmt>(__uint_as_float(r << 16) * to_units, __uint_as_float(r & 0xffff0000u) * to_units);
        }
        w0[word] = (w0[word] & ~(0xffu << shift)) | ((two & 0xffu) << shift);
        w1[word] = (w1[word] & ~(0xffu << shift)) | ((two >> 8) << shift);
      }
      c[0] = w0;
      c[1] = w1;
    }
  }
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

int check_seqs(const char* who, const int32_t* cu, bool needs_cu, const int32_t* kv_len, const int32_t* pages, int32_t n_seqs, int32_t max_pages, int32_t n_rows) {
  if (n_seqs < 0 || max_pages < 0 || n_rows < 0) return fail(FCP_ERR_INVALID_ARG, "%s: negative size", who);
  if (n_seqs > 0 && ((needs_cu && !cu) || !kv_len || (max_pages > 0 && !pages))) return fail(FCP_ERR_INVALID_ARG, "%s: null argument", who);
  if (n_seqs > 1 << 20) return fail(FCP_ERR_UNSUPPORTED, "%s: more than 2^20 sequences", who);
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
  if (int rc = check_seqs(who, cu_seqlens, true, kv_len, pages, n_seqs, max_pages, n_rows)) return rc;
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
  hipStream_t st = static_cast<hipStream_t>(stream);
  const dim3 grid((unsigned)a.units, (unsigned)((2 * a.c.hkv + 3) / 4));
  const bool e4m3 = cache->format == FCP_CACHE_E4M3;
  auto kernel = cache->head_dim == 128 ? (e4m3 ? append_kernel<128, kE4m3> : append_kernel<128, kInt8>) : (e4m3 ? append_kernel<64, kE4m3> : append_kernel<64, kInt8>);
  kernel<<<grid, dim3(256), 0, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  return FCP_OK;
}
