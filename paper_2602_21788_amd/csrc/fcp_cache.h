// What the kernels of the paged 8-bit cache share: the cache as kernels take it, its codes, and the places of pages and rows.
#pragma once
#include "fcp_device.h"

namespace fcp {

constexpr int kGroup = 16;             // tokens of a value group, and the least page
constexpr int kLeastExponent = -110;   // of a scale: 2^110 times a value that needs less is still finite
constexpr int kE4m3 = FCP_CACHE_E4M3, kInt8 = FCP_CACHE_INT8;

typedef float f32x2 __attribute__((ext_vector_type(2)));

// fcp_cache with its sizes as the kernels use them.
struct CacheView {
  uint8_t* k;
  uint8_t* v;
  float* k_scale;
  float* v_scale;
  float* weight;
  int32_t n_pages, hkv, page, log_page;
};

// Sequences of a call: rows of cu_seqlens, cached tokens, page table.
struct SeqView {
  const int32_t* cu;
  const int32_t* kv_len;
  const int32_t* pages;
  int32_t n_seqs, max_pages, n_rows;
};

// First row, rows and cached tokens of a sequence, whatever the tables hold: rows inside 0 .. n_rows, tokens inside the table.
struct SeqSizes { int32_t row0, n, len; };
__device__ inline SeqSizes seq_sizes(const SeqView& s, int seq, int page) {
  const int32_t a = min(max(s.cu[seq], 0), s.n_rows), b = min(max(s.cu[seq + 1], a), s.n_rows);
  const int64_t room = (int64_t)s.max_pages * page;
  const int32_t len = max(s.kv_len[seq], 0);
  return {a, b - a, len < room ? len : (int32_t)room};
}
// The page at `place` in the sequence's table, -1 if there is none.
__device__ inline int32_t page_at(const SeqView& s, const CacheView& c, int seq, int32_t place) {
  if (place < 0 || place >= s.max_pages) return -1;
  const int32_t p = s.pages[(int64_t)seq * s.max_pages + place];
  return (uint32_t)p < (uint32_t)c.n_pages ? p : -1;
}
// (page, KV head) as one number: scales, weights and codes lie in this order
__device__ inline int64_t block_of(const CacheView& c, int32_t page, int head) { return (int64_t)page * c.hkv + head; }

// ---- codes --------------------------------------------------------------------------------------
template <int Fmt> __device__ constexpr float most() { return Fmt == kE4m3 ? 448.f : 127.f; }

// The least e with amax 2^more <= most 2^e: 448 = 0.875 * 2^9, 127 = (127 / 128) 2^7.  amax: finite, >= 0.
template <int Fmt>
__device__ inline int exponent_for(float amax, int more = 0) {
  if (!(amax > 0.f)) return kLeastExponent;
  const float m = __builtin_amdgcn_frexp_mantf(amax);
  const int x = __builtin_amdgcn_frexp_expf(amax);
  const int e = Fmt == kE4m3 ? x - 9 + (m > 0.875f) : x - 7 + (m > 127.f / 128.f);
  return max(e + more, kLeastExponent);
}
// 2^e for -126 <= e <= 127, 0 below
__device__ inline float power2(int e) { return e < -126 ? 0.f : __int_as_float((e + 127) << 23); }
// exponent of a scale that is a power of two
__device__ inline int exponent_of(float scale) { return ((__float_as_int(scale) >> 23) & 255) - 127; }

// Two values, already in units of their scale, as two codes in the low 16 bits.
template <int Fmt>
__device__ inline uint32_t encode2(float a, float b) {
  if constexpr (Fmt == kE4m3) {
    a = __builtin_isnan(a) ? a : fminf(fmaxf(a, -448.f), 448.f);
    b = __builtin_isnan(b) ? b : fminf(fmaxf(b, -448.f), 448.f);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu;
  } else {
    const int i = __builtin_isnan(a) ? 0 : (int)rintf(fminf(fmaxf(a, -127.f), 127.f));
    const int j = __builtin_isnan(b) ? 0 : (int)rintf(fminf(fmaxf(b, -127.f), 127.f));
    return (uint32_t)(i & 0xff) | ((uint32_t)(j & 0xff) << 8);
  }
}
// The two codes in the low 16 bits as floats.
template <int Fmt>
__device__ inline f32x2 decode2(uint32_t u) {
  if constexpr (Fmt == kE4m3) return __builtin_amdgcn_cvt_pk_f32_fp8(u, false);
  else return f32x2{(float)(int8_t)u, (float)(int8_t)(u >> 8)};
}
// The two codes in the lower or upper half of a word as floats; two values, within the format, as codes in that half.
template <int Fmt, bool Upper>
__device__ inline f32x2 decode_half(uint32_t u) {
  if constexpr (Fmt == kE4m3) return __builtin_amdgcn_cvt_pk_f32_fp8(u, Upper);
  else return f32x2{(float)(int8_t)(u >> (Upper ? 16 : 0)), (float)(int8_t)(u >> (Upper ? 24 : 8))};
}
template <int Fmt, bool Upper>
__device__ inline uint32_t encode_half(float a, float b, uint32_t word) {
  if constexpr (Fmt == kE4m3) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)word, Upper);
  } else {
    const uint32_t two = ((uint32_t)(int)rintf(a) & 0xffu) | ((uint32_t)(int)rintf(b) & 0xffu) << 8;
    return Upper ? (word & 0xffffu) | two << 16 : (word & 0xffff0000u) | two;
  }
}
// Eight codes in two words as bf16: both formats' values are exact there (4 and 7 significant bits).
template <int Fmt>
__device__ inline bf16x8 decode8(uint32_t lo, uint32_t hi) {
  if constexpr (Fmt == kE4m3) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  } else {
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[i] = (__bf16)(float)(int8_t)(lo >> (8 * i));
      r[4 + i] = (__bf16)(float)(int8_t)(hi >> (8 * i));
    }
    return r;
  }
}

// One wave-wide LDS-direct load: the 16 bytes at every lane's own address land at LDS offset `lds` (the same for the wave) + 16 lane.  In assembly for the reasons given at
// lds_fill_b128: the caller waits with s_waitcnt vmcnt before the wave reads them.
__device__ inline void lds_load_b128(const void* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(from) : "memory");
}

__device__ inline float wave_maxf(float x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}

// ---- host ---------------------------------------------------------------------------------------
// Checks what every call of the cache checks, and fills the view.  needs_weight: the call reads or writes weights.  Sizes apart: those who only ask for scratch have no tables yet.
int check_cache(const char* who, const fcp_cache* cache, bool needs_weight, CacheView* out);
int check_sizes(const char* who, const CacheView& c, int32_t n_seqs, int32_t max_pages, int32_t n_rows);
int check_seqs(const char* who, const CacheView& c, const int32_t* cu, bool needs_cu, const int32_t* kv_len, const int32_t* pages, int32_t n_seqs, int32_t max_pages, int32_t n_rows);

}  // namespace fcp
