// Rotary positions: rows of queries, keys or their gradients turned by the angles of their positions (fcp_rotary), and the host's frequencies.
//
// A pair (a, b) of channels with frequency f at position p becomes (a cos t - b sin t, a sin t + b cos t), t = 2 pi frac(p f).  Every element is read
// and written once and takes part in two products, so the memory bounds it.  The angle is the same for all heads of a row: a block takes a few rows
// of one tensor, forms their cosines and sines once in LDS, and its threads then work 16 bytes at a time, head after head.
// p f is formed in 64 bits and reduced to a fraction of a turn there: at p = 10^6 a product in 32 bits is off by 0.06 of a radian.  The fraction, at
// most half a turn, has 24 good bits as a float (angle off by 2e-7).
#include <math.h>

#include "fcp_device.h"

namespace fcp {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotLds = 1024;         // cosines and sines a block holds: rows * rot_dim / 2
constexpr int kRotItem = 16;          // head_dim and rot_dim are multiples of it where 16 bytes move at a time

struct RotaryArgs {
  fcp_rotary_part part[FCP_ROTARY_MAX_PARTS];
  int32_t first[FCP_ROTARY_MAX_PARTS + 1];      // first block of each part
  int32_t n_parts, head_dim, rot, rows, heads;  // rows and heads of a block
  const double* turns;
  float magnitude, sign;
};

template <class T> __device__ inline float load1(const T* p);
template <> __device__ inline float load1(const float* p) { return *p; }
template <> __device__ inline float load1(const __bf16* p) { return (float)*p; }

// W neighbouring channels: 16 bytes of what is read
template <int W> struct Channels { float f[W]; };
__device__ inline Channels<4> load16(const float* p) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p);
  return {{a[0], a[1], a[2], a[3]}};
}
__device__ inline Channels<8> load16(const __bf16* p) {
  const bf16x8 a = *reinterpret_cast<const bf16x8*>(p);
  Channels<8> r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.f[i] = (float)a[i];
  return r;
}
template <int W>
__device__ inline void store(float* p, const Channels<W>& x) {
#pragma unroll
  for (int i = 0; i < W; i += 4) *reinterpret_cast<f32x4*>(p + i) = f32x4{x.f[i], x.f[i + 1], x.f[i + 2], x.f[i + 3]};
}
__device__ inline void store(__bf16* p, const Channels<4>& x) { *reinterpret_cast<bf16x4*>(p) = bf16x4{(__bf16)x.f[0], (__bf16)x.f[1], (__bf16)x.f[2], (__bf16)x.f[3]}; }
__device__ inline void store(__bf16* p, const Channels<8>& x) {
  bf16x8 a;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = (__bf16)x.f[i];
  *reinterpret_cast<bf16x8*>(p) = a;
}

// Division by a number that stays: by 2^32 / d rounded up, at most one too large.  (There are two for each item of 16 bytes, and the
// compiler's division of integers is some twenty instructions.)
struct Divisor {
  uint32_t d, m;
  __device__ explicit Divisor(int by) : d(by), m(by == 1 ? 0u : 0xffffffffu / (uint32_t)by + 1) {}
  __device__ int operator()(int x, int& rest) const {
    int q = d == 1 ? x : (int)__umulhi((uint32_t)x, m);
    rest = x - q * (int)d;
    if (rest < 0) { --q; rest += (int)d; }
    return q;
  }
};

template <class X, class Y, bool Half, bool Wide>
__device__ void turn_rows(const RotaryArgs& a, const fcp_rotary_part& p, int row0, int rows, int head0, int heads, const float2* cs) {
  const int half = a.rot / 2;
  const X* const x0 = static_cast<const X*>(p.x) + (int64_t)row0 * p.x_row + (int64_t)head0 * p.x_head;
  Y* const y0 = static_cast<Y*>(p.y) + (int64_t)row0 * p.y_row + (int64_t)head0 * p.y_head;
  if constexpr (Wide) {
    // An item is 16 bytes of what is read, or, where a pair's channels lie apart, twice 16 bytes: neighbouring lanes read and write neighbouring bytes.  Items that turn and items that
    // are copied load and store alike, and at the same place in the program: a wave often has both.
    constexpr int W = 16 / sizeof(X), kItem = Half ? 2 * W : W;
    const int turning = a.rot / kItem, per_head = a.head_dim / kItem, n = rows * heads * per_head;
    const Divisor by_head(per_head), by_row(heads);
    for (int it = threadIdx.x; it < n; it += kRotThreads) {
      int i, h;
      const int r = by_row(by_head(it, i), h);
      const bool turns = i < turning;
      const int ca = Half && turns ? W * i : kItem * i, cb = Half && turns ? half + W * i : kItem * i + W;
      const X* x = x0 + r * p.x_row + h * p.x_head;
      Y* y = y0 + r * p.y_row + h * p.y_head;
      Channels<W> u = load16(x + ca), v = u;
      if (Half) v = load16(x + cb);
      if (turns) {
        const float2* t = cs + r * half + (Half ? W : W / 2) * i;
#pragma unroll
        for (int j = 0; j < (Half ? W : W / 2); ++j) {
          float &xa = Half ? u.f[j] : u.f[2 * j], &xb = Half ? v.f[j] : u.f[2 * j + 1];
          const float2 c = t[j];
          const float ya = xa * c.x - xb * c.y, yb = xa * c.y + xb * c.x;
          xa = ya;
          xb = yb;
        }
      }
      store(y + ca, u);
      if (Half) store(y + cb, v);
    }
  } else {                                         // items of one pair, or of one channel that does not turn
    const int per_head = half + a.head_dim - a.rot, n = rows * heads * per_head;
    const Divisor by_head(per_head), by_row(heads);
    for (int it = threadIdx.x; it < n; it += kRotThreads) {
      int i, h;
      const int r = by_row(by_head(it, i), h);
      const X* x = x0 + r * p.x_row + h * p.x_head;
      Y* y = y0 + r * p.y_row + h * p.y_head;
      if (i >= half) {
        y[half + i] = (Y)load1(x + half + i);
      } else {
        const int ca = Half ? i : 2 * i, cb = Half ? half + i : 2 * i + 1;
        const float xa = load1(x + ca), xb = load1(x + cb);
        const float2 c = cs[r * half + i];
        y[ca] = (Y)(xa * c.x - xb * c.y);
        y[cb] = (Y)(xa * c.y + xb * c.x);
      }
    }
  }
}

template <bool Half, bool Wide>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a) {
  __shared__ float2 cs[kRotLds];
  int at = 0;
#pragma unroll
  for (int i = 1; i < FCP_ROTARY_MAX_PARTS; ++i) at += i < a.n_parts && (int)blockIdx.x >= a.first[i];
  const fcp_rotary_part& p = a.part[at];
  const int b = blockIdx.x - a.first[at], per_row = (p.heads + a.heads - 1) / a.heads;
  const int row0 = b / per_row * a.rows, head0 = b % per_row * a.heads;
  const int rows = min(a.rows, p.rows - row0), heads = min(a.heads, p.heads - head0), half = a.rot / 2;
  for (int i = threadIdx.x; i < rows * half; i += kRotThreads) {
    const double t = (double)p.pos[row0 + i / half] * a.turns[i % half];
    float s, c;
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    cs[i] = make_float2(c * a.magnitude, s * a.magnitude * a.sign);
  }
  __syncthreads();
  if (p.x_type == FCP_BF16 && p.y_type == FCP_BF16) turn_rows<__bf16, __bf16, Half, Wide>(a, p, row0, rows, head0, heads, cs);
  else if (p.x_type == FCP_F32 && p.y_type == FCP_BF16) turn_rows<float, __bf16, Half, Wide>(a, p, row0, rows, head0, heads, cs);
  else if (p.x_type == FCP_F32) turn_rows<float, float, Half, Wide>(a, p, row0, rows, head0, heads, cs);
  else turn_rows<__bf16, float, Half, Wide>(a, p, row0, rows, head0, heads, cs);
}

bool multiple16(const void* p, int64_t row, int64_t head, int type) {
  const int n = type == FCP_BF16 ? 8 : 4;
  return (uintptr_t)p % 16 == 0 && row % n == 0 && head % n == 0;
}

}  // namespace
}  // namespace fcp

extern "C" int fcp_rotary_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double original_len, double low,
                                      double high, double* turns, float* magnitude) {
  using fcp::fail;
  fcp::clear_error();
  const char* who = "fcp_rotary_frequencies";
  if (!turns || rot_dim < 2 || rot_dim % 2 || !(base > 0) || !isfinite(base))
    return fail(FCP_ERR_INVALID_ARG, "%s: turns, an even rot_dim of at least 2 and a base above 0 are required", who);
  if (scaling < FCP_ROTARY_PLAIN || scaling > FCP_ROTARY_PARTS) return fail(FCP_ERR_UNSUPPORTED, "%s: scaling %d is not known", who, scaling);
  if (scaling != FCP_ROTARY_PLAIN && !(factor >= 1 && isfinite(factor))) return fail(FCP_ERR_INVALID_ARG, "%s: factor must be at least 1", who);
  if (scaling == FCP_ROTARY_BASE && rot_dim == 2) return fail(FCP_ERR_INVALID_ARG, "%s: a scaled base needs rot_dim of at least 4", who);
  if (scaling == FCP_ROTARY_PARTS && !(original_len > 0 && isfinite(original_len) && low >= 0 && high > low && isfinite(high)))
    return fail(FCP_ERR_INVALID_ARG, "%s: original_len above 0 and 0 <= low < high are required", who);
  const double pi = 3.14159265358979323846;
  if (scaling == FCP_ROTARY_BASE) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
  for (int32_t i = 0; i < rot_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / rot_dim) / (2 * pi);
    if (scaling == FCP_ROTARY_LINEAR) f /= factor;
    if (scaling == FCP_ROTARY_PARTS) {
      const double kept = fmin(1, fmax(0, (original_len * f - low) / (high - low)));
      f = kept * f + (1 - kept) * f / factor;
    }
    turns[i] = f;
  }
  if (magnitude) *magnitude = scaling == FCP_ROTARY_PARTS && factor > 1 ? (float)(0.1 * log(factor) + 1) : 1.f;
  return FCP_OK;
}

extern "C" int fcp_rotary(const fcp_rotary_part* parts, int32_t n_parts, const double* turns, int32_t head_dim, int32_t rot_dim, int32_t layout,
                          float magnitude, int32_t backward, void* stream) {
  using namespace fcp;
  clear_error();
  const char* who = "fcp_rotary";
  if (n_parts < 0 || (n_parts > 0 && !parts) || !turns) return fail(FCP_ERR_INVALID_ARG, "%s: null argument or negative n_parts", who);
  if (n_parts > FCP_ROTARY_MAX_PARTS) return fail(FCP_ERR_UNSUPPORTED, "%s: %d parts, at most %d", who, n_parts, FCP_ROTARY_MAX_PARTS);
  if (head_dim < 2 || head_dim > 1024) return fail(FCP_ERR_UNSUPPORTED, "%s: head_dim %d is not between 2 and 1024", who, head_dim);
  if (rot_dim < 2 || rot_dim > head_dim || rot_dim % 2) return fail(FCP_ERR_INVALID_ARG, "%s: rot_dim %d is not even and between 2 and head_dim", who, rot_dim);
  if (layout != FCP_ROTARY_HALF && layout != FCP_ROTARY_PAIRS) return fail(FCP_ERR_INVALID_ARG, "%s: layout %d is not known", who, layout);
  if (!(magnitude > 0) || !isfinite(magnitude) || (backward != 0 && backward != 1))
    return fail(FCP_ERR_INVALID_ARG, "%s: magnitude must be above 0 and backward 0 or 1", who);
  RotaryArgs a = {};
  bool wide = head_dim % kRotItem == 0 && rot_dim % kRotItem == 0;
  int64_t head_rows = 0, row_bytes = 1;
  for (int32_t i = 0; i < n_parts; ++i) {
    const fcp_rotary_part& p = parts[i];
    if (p.rows < 0 || p.heads < 0) return fail(FCP_ERR_INVALID_ARG, "%s: parts[%d] has negative sizes", who, i);
    if (p.rows == 0 || p.heads == 0) continue;
    if (!p.x || !p.y || !p.pos) return fail(FCP_ERR_INVALID_ARG, "%s: parts[%d] has a null pointer", who, i);
    if ((p.x_type != FCP_BF16 && p.x_type != FCP_F32) || (p.y_type != FCP_BF16 && p.y_type != FCP_F32))
      return fail(FCP_ERR_UNSUPPORTED, "%s: parts[%d] has a type that is not known", who, i);
    if (p.x_row < 0 || p.x_head < 0 || p.y_row < 0 || p.y_head < 0) return fail(FCP_ERR_INVALID_ARG, "%s: parts[%d] has a negative stride", who, i);
    if ((p.rows > 1 && p.y_row < head_dim) || (p.heads > 1 && p.y_head < head_dim))
      return fail(FCP_ERR_INVALID_ARG, "%s: rows or heads of parts[%d].y overlap", who, i);
    if (p.x == p.y && (p.x_type != p.y_type || p.x_row != p.y_row || p.x_head != p.y_head))
      return fail(FCP_ERR_INVALID_ARG, "%s: parts[%d] in place needs the same type and strides", who, i);
    if ((uintptr_t)p.x % (p.x_type == FCP_BF16 ? 2 : 4) || (uintptr_t)p.y % (p.y_type == FCP_BF16 ? 2 : 4))
      return fail(FCP_ERR_INVALID_ARG, "%s: parts[%d] is not aligned to its type", who, i);
    wide = wide && multiple16(p.x, p.x_row, p.x_head, p.x_type) && multiple16(p.y, p.y_row, p.y_head, p.y_type);
    head_rows += (int64_t)p.rows * p.heads;
    const int64_t bytes = (int64_t)p.heads * head_dim * ((p.x_type == FCP_BF16 ? 2 : 4) + (p.y_type == FCP_BF16 ? 2 : 4));
    if (bytes > row_bytes) row_bytes = bytes;
    a.part[a.n_parts++] = p;
  }
  if (a.n_parts == 0) return FCP_OK;
  // Rows of a block: as many as leave a thread one cosine to form (more than 512 pairs in a row: one row), but no more than 64 KB of traffic, or a launch ends with a few blocks that the
  // others wait for (9363 rows of 40 and 8 heads, half of 128 channels turn, fp32 to bf16: 2 rows 67.8 us, 4 rows 73.2; 32768 rows of 32 and 8 heads, bf16: 2 rows 125.2, 4 rows 120.4).
  // Heads: all of them, except where that makes fewer blocks than two per CU; then a block has few enough that every thread has about one item.
  a.head_dim = head_dim;
  a.rot = rot_dim;
  const int64_t fit = 65536 / row_bytes;
  a.rows = rot_dim / 2 >= kRotThreads ? 1 : kRotThreads / (rot_dim / 2);
  if (a.rows > fit) a.rows = fit < 1 ? 1 : (int32_t)fit;
  const int per_head = wide ? head_dim / kRotItem : head_dim - rot_dim / 2;
  if (head_rows * per_head < (int64_t)512 * kRotThreads) {
    a.rows = 1;
    a.heads = kRotThreads / per_head < 1 ? 1 : kRotThreads / per_head;
  } else {
    a.heads = 4096;                                  // (rows * heads * items stay below 2^31)
  }
  int64_t blocks = 0;
  for (int32_t i = 0; i < a.n_parts; ++i) {
    a.first[i] = (int32_t)blocks;
    const fcp_rotary_part& p = a.part[i];
    blocks += ((int64_t)p.rows + a.rows - 1) / a.rows * (a.heads >= p.heads ? 1 : ((int64_t)p.heads + a.heads - 1) / a.heads);
    if (!fits_axis(blocks, kRotThreads)) return fail(FCP_ERR_UNSUPPORTED, "%s: 2^24 blocks of rows or more", who);
  }
  a.first[a.n_parts] = (int32_t)blocks;
  a.turns = turns;
  a.magnitude = magnitude;
  a.sign = backward ? -1.f : 1.f;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool half = layout == FCP_ROTARY_HALF;
  auto kernel = half ? (wide ? rotary_kernel<true, true> : rotary_kernel<true, false>) : (wide ? rotary_kernel<false, true> : rotary_kernel<false, false>);
  kernel<<<dim3((unsigned)blocks), dim3(kRotThreads), 0, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  return FCP_OK;
}
