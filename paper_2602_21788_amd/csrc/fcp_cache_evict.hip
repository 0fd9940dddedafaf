// fcp_cache_evict: the cached tokens with the greatest attention weight kept, per KV head, and moved to new pages.
//
// Two launches.  The first finds, for a (sequence, KV head), the k-th greatest weight among the tokens that are neither among the first nor the most recent, by
// counting 8 bits of an ordered integer at a time, and lists the kept tokens in order.  The second moves them: a wave per (new page, KV head, keys or
// values) gathers the page's tokens from wherever they lie, finds the page's scale and writes the codes in its units.
#include "fcp_cache.h"

namespace fcp {
namespace {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;

struct EvictArgs {
  CacheView c;
  SeqView s;                           // (no rows)
  const int32_t* new_pages;
  int32_t max_new, budget, first, recent;
  int32_t* kept;
  int32_t* new_len;
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
// weight of token t (0 where its page is missing)
__device__ inline uint32_t order_at(const EvictArgs& a, int seq, int head, int t) {
  const int32_t p = page_at(a.s, a.c, seq, t >> a.c.log_page);
  return p < 0 ? order_of(0.f) : order_of(a.c.weight[block_of(a.c, p, head) * a.c.page + (t & (a.c.page - 1))]);
}

__global__ __launch_bounds__(kSelectThreads) void select_kernel(EvictArgs a) {
  __shared__ int32_t bins[256];
  __shared__ int32_t waves[2][kSelectWaves];
  __shared__ uint32_t s_prefix;
  __shared__ int32_t s_want;
  const int seq = blockIdx.x / a.c.hkv, head = blockIdx.x % a.c.hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = cached(a, seq), n_new = min(n, a.budget);
  int32_t* const kept = a.kept + ((int64_t)seq * a.c.hkv + head) * a.budget;
  if (head == 0 && tid == 0) a.new_len[seq] = n_new;
  for (int i = n_new + tid; i < a.budget; i += kSelectThreads) kept[i] = -1;
  if (n <= a.budget) {
    for (int i = tid; i < n; i += kSelectThreads) kept[i] = i;
    return;
  }
  // tokens lo .. hi - 1 compete for `want` places
  const int lo = a.first, hi = n - a.recent;
  int32_t want = a.budget - a.first - a.recent;
  uint32_t prefix = 0;                             // upper bits of the last kept weight
  for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
    if (tid < 256) bins[tid] = 0;
    __syncthreads();
    for (int t = lo + tid; t < hi; t += kSelectThreads) {
      const uint32_t u = order_at(a, seq, head, t);
      if (shift == 24 || (u >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&bins[(u >> shift) & 255], 1);
    }
    __syncthreads();
    // the bin that holds the want-th greatest: wave 0, four bins a lane, from the greatest down
    if (wave == 0) {
      int32_t mine[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) sum += mine[i] = bins[255 - 4 * lane - i];
      int32_t upto = wave_prefix_sum(sum), above = upto - sum;
      if (above < want && want <= upto) {
        int i = 0;
        while (above + mine[i] < want) above += mine[i++];
        s_prefix = prefix | (uint32_t)(255 - 4 * lane - i) << shift;
        s_want = want - above;
      }
    }
    __syncthreads();
    prefix = s_prefix;
    want = s_want;
  }
  // kept: the protected, those above the border, and the first `want` at it.  A wave lists a run of tokens; how many the runs before it keep comes from a count first
  const bool none = a.budget == a.first + a.recent;
  const int run = ((n + kSelectWaves - 1) / kSelectWaves + 63) & ~63, t0 = min(wave * run, n), t1 = min(t0 + run, n);
  int32_t above = 0, equal = 0;
  for (int t = t0 + lane; t < t1; t += 64) {
    const bool safe = t < lo || t >= hi;
    const uint32_t u = safe || none ? 0 : order_at(a, seq, head, t);
    above += safe || (!none && u > prefix);
    equal += !safe && !none && u == prefix;
  }
  above = __builtin_amdgcn_readlane(wave_prefix_sum(above), 63);
  equal = __builtin_amdgcn_readlane(wave_prefix_sum(equal), 63);
  if (lane == 0) { waves[0][wave] = above; waves[1][wave] = equal; }
  __syncthreads();
  int32_t place = 0, equals = 0;                   // listed and equal ones before the run
  for (int w = 0; w < wave; ++w) {
    place += waves[0][w] + min(waves[1][w], max(want - equals, 0));
    equals += waves[1][w];
  }
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int t = t0 + lane; t - lane < t1; t += 64) {
    const bool in = t < t1, safe = in && (t < lo || t >= hi);
    const uint32_t u = !in || safe || none ? 0 : order_at(a, seq, head, t);
    const bool eq = in && !safe && !none && u == prefix;
    const uint64_t eqs = __ballot(eq);
    const bool keep = safe || (in && !none && u > prefix) || (eq && equals + __popcll(eqs & below) < want);
    const uint64_t keeps = __ballot(keep);
    if (keep) kept[place + __popcll(keeps & below)] = t;
    place += __popcll(keeps);
    equals += __popcll(eqs);
  }
}

template <int D, int Fmt>
__global__ __launch_bounds__(256) void move_kernel(EvictArgs a) {
  constexpr int LPR = D / 2, TPW = 64 / LPR;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int job = blockIdx.y * 4 + wave;
  if (job >= 2 * a.c.hkv) return;
  const int head = job >> 1, P = a.c.page, seq = blockIdx.x / a.max_new, place = blockIdx.x % a.max_new;
  const bool value = job & 1;
  const int n_new = min(cached(a, seq), a.budget), count = min(P, n_new - place * P);
  if (count <= 0) return;
  const int32_t page = a.new_pages[(int64_t)seq * a.max_new + place];
  if ((uint32_t)page >= (uint32_t)a.c.n_pages) return;
  const int32_t* const kept = a.kept + ((int64_t)seq * a.c.hkv + head) * a.budget + place * P;
  const int sub = lane / LPR, ch = 2 * (lane % LPR);
  const uint8_t* const from = value ? a.c.v : a.c.k;
  const float* const scales = value ? a.c.v_scale : a.c.k_scale;
  // the lane's two channels of the token in slot j, as they stand (0 past the last and where a page is missing)
  auto fetch = [&](int j) -> f32x2 {
    if (j >= count) return f32x2{0.f, 0.f};
    const int t = kept[j];
    const int32_t p = page_at(a.s, a.c, seq, t >> a.c.log_page);
    if (p < 0) return f32x2{0.f, 0.f};
    const int64_t block = block_of(a.c, p, head);
    const int slot = t & (P - 1);
    const float s = scales[block];
    uint32_t two;
    if (!value) {
      two = *reinterpret_cast<const uint16_t*>(from + (block * P + slot) * D + ch);
    } else {
      const uint8_t* b = from + (block * P + (slot & ~(kGroup - 1))) * D + ch * kGroup + (slot & (kGroup - 1));
      two = b[0] | (uint32_t)b[kGroup] << 8;
    }
    const f32x2 f = decode2<Fmt>(two);
    return f32x2{f[0] * s, f[1] * s};
  };
  float top = 0.f;
#pragma unroll 4
  for (int j = sub; j < count; j += TPW) {
    const f32x2 f = fetch(j);
    const float x = fabsf(f[0]), y = fabsf(f[1]);
    top = fmaxf(top, fmaxf(x < INFINITY ? x : 0.f, y < INFINITY ? y : 0.f));
  }
  const int e = exponent_for<Fmt>(wave_maxf(top));
  const float to_units = power2(-e);
  const int64_t block = block_of(a.c, page, head);
  if (lane == 0) (value ? a.c.v_scale : a.c.k_scale)[block] = power2(e);
  uint8_t* const codes = (value ? a.c.v : a.c.k) + block * P * D;
  if (!value) {
#pragma unroll 4
    for (int j = sub; j < P; j += TPW) {
      const f32x2 f = fetch(j);
      *reinterpret_cast<uint16_t*>(codes + j * D + ch) = (uint16_t)encode2<Fmt>(f[0] * to_units, f[1] * to_units);
    }
    for (int j = lane; j < P; j += 64) {
      float w = 0.f;
      if (j < count) {
        const int t = kept[j];
        const int32_t p = page_at(a.s, a.c, seq, t >> a.c.log_page);
        if (p >= 0) w = a.c.weight[block_of(a.c, p, head) * P + (t & (P - 1))];
      }
      a.c.weight[block * P + j] = w;
    }
  } else {
    for (int g = sub; g * kGroup < P; g += TPW) {
      u32x4 w0 = {0, 0, 0, 0}, w1 = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < kGroup; ++j) {
        const f32x2 f = fetch(g * kGroup + j);
        const uint32_t two = encode2<Fmt>(f[0] * to_units, f[1] * to_units);
        w0[j / 4] |= (two & 0xffu) << (8 * (j % 4));
        w1[j / 4] |= (two >> 8) << (8 * (j % 4));
      }
      u32x4* const c = reinterpret_cast<u32x4*>(codes + (g * D + ch) * kGroup);
      c[0] = w0;
      c[1] = w1;
    }
  }
}

}  // namespace

size_t evict_scratch_bytes(const CacheView&, int32_t, int32_t) { return 256; }

}  // namespace fcp

extern "C" int fcp_cache_evict(const fcp_cache* cache, const int32_t* pages, const int32_t* kv_len, int32_t n_seqs, int32_t max_pages,
                               const int32_t* new_pages, int32_t max_new_pages, int32_t budget, int32_t n_first, int32_t n_recent, int32_t* kept,
                               int32_t* new_len, void* scratch, size_t scratch_bytes, void* stream) {
  using namespace fcp;
  clear_error();
  const char* who = "fcp_cache_evict";
  EvictArgs a = {};
  if (int rc = check_cache(who, cache, true, &a.c)) return rc;
  if (int rc = check_seqs(who, nullptr, false, kv_len, pages, n_seqs, max_pages, 0)) return rc;
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
  const size_t need = evict_scratch_bytes(a.c, n_seqs, max_pages);
  if (scratch_bytes < need) return fail(FCP_ERR_CAPACITY, "%s: scratch has %zu bytes, %zu are needed", who, scratch_bytes, need);
  const int64_t use = (most + a.c.page - 1) / a.c.page;      // (further entries of new_pages are not used)
  if ((int64_t)n_seqs * a.c.hkv > INT32_MAX || (int64_t)n_seqs * max_new_pages > INT32_MAX)
    return fail(FCP_ERR_UNSUPPORTED, "%s: more than 2^31 - 1 pages or heads of all sequences", who);
  a.s = {nullptr, kv_len, pages, n_seqs, max_pages, 0};
  a.new_pages = new_pages;
  a.max_new = max_new_pages;
  a.budget = budget;
  a.first = n_first;
  a.recent = n_recent;
  a.kept = kept;
  a.new_len = new_len;
  hipStream_t st = static_cast<hipStream_t>(stream);
  select_kernel<<<dim3((unsigned)(n_seqs * a.c.hkv)), dim3(kSelectThreads), 0, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  if (use == 0) return FCP_OK;
  const dim3 grid((unsigned)(n_seqs * max_new_pages), (unsigned)((2 * a.c.hkv + 3) / 4));
  const bool e4m3 = cache->format == FCP_CACHE_E4M3;
  auto kernel = cache->head_dim == 128 ? (e4m3 ? move_kernel<128, kE4m3> : move_kernel<128, kInt8>) : (e4m3 ? move_kernel<64, kE4m3> : move_kernel<64, kInt8>);
  kernel<<<grid, dim3(256), 0, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  return FCP_OK;
}
