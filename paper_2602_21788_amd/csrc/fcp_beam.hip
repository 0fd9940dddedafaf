// fcp_beam_select: the best continuations of every prompt, over its beams and the vocabulary.
//
// The score of token t behind beam b is score_b + x_bt - ln sum_u exp x_bu.  The order of a beam's tokens is that of its logits, so a beam offers its `keep` greatest logits, and the
// logarithm is needed only to put beams beside each other.  Sums and scores are held in 64 bits, and the logarithm is off by 1e-10 at most: by 5.4e-11 from the terms of a chunk's sum (NearSum), and where
// a row has several by 4.3e-11 from bringing their sums together (Exp).  Candidates of different beams that lie nearer than 2e-10 may come in either order.
//
// First launch: a block takes a chunk of a row, up to 32 neighbouring logits a thread (8 where there are few rows), which stay in registers for three looks:
//   * the greatest of every four threads, 64 in all (of each of the 256 threads, if more than 32 are kept); the keep-th greatest of those, T, found bit by bit: at least `keep` logits of the chunk are T
//     or more, and as a rule few others;
//   * the sum of exp(x - greatest);
//   * logits beyond T, and those equal to it in T's threads and earlier ones, go to a list in LDS, which is put in order by counting how many are beyond each.  Where there are more than the list has
//     places, T becomes the keep-th greatest logit itself.
// Second launch: a block for each prompt joins the sums and finds the best candidates of all lists the same way, all lists' best first.
//
// 64 prompts of 8 beams, 131072 bf16 logits each, 16 kept: 48.5 us (43 and 7.7 under a profiler; a copy's rate would read the logits in 27); vector instructions bound the first, loads and barriers that
// wait for each other the second, and all of small calls: one prompt of 4 beams over 32000 tokens 11.8 us (6 to 7, and 6.2).
#include <float.h>

#include "fcp_device.h"

namespace fcp {
namespace {

constexpr int kThreads = 256, kGroups = 64;   // groups of neighbouring threads whose greatest element stands for them: a lane each
constexpr int kPerGroup = kThreads / kGroups;

struct BeamArgs {
  const void* logits;
  int64_t row;
  int32_t rows, beams, vocab, chunks, length, each, keep, end_token;         // length: logits of a chunk (of a row's last one a few less); each: of a thread
  const float* score;
  const uint8_t* done;
  int32_t* parent;
  int32_t* token;
  float* new_score;
  uint8_t* new_done;
  uint64_t* lists;                     // [rows][chunks][keep]: ordered logit, then ~token; 0: none
  double* sums;                        // [rows][chunks]: sum of exp(x - reference), reference; a sum of 0: no logits
};

// Integers that order floats: greater value, greater integer (never 0).  No NaN, no -0.
__device__ inline uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float value_of(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order); }
__device__ inline uint64_t order_of(double x) {
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
  return u >> 63 ? ~u : u | (uint64_t)1 << 63;
}
__device__ inline double score_of(uint64_t order) { return __longlong_as_double((long long)(order >> 63 ? order & ~((uint64_t)1 << 63) : ~order)); }

// A constant in scalar registers: an instruction of the vector unit takes one, and the compiler would rather move it to vector registers every time.
__device__ inline double scalar(double x) { asm volatile("" : "+s"(x)); return x; }

// exp(d), d <= 0, in 64 bits: 2^n times a polynomial in f, n + f = d log2(e), |f| <= 1/2.  The coefficients are a least-squares fit on Chebyshev nodes with weights 2^-f; the relative error is at most
// 4.3e-11.  What is below -700, and NaN, counts as -700.
struct Exp {
  double log2e = scalar(1.4426950408889634074);
  double c[8] = {scalar(0x1.ffffffffac502p-1), scalar(0x1.62e42ff12cfc5p-1), scalar(0x1.ebfbe0a416e10p-3), scalar(0x1.c6b08a80840e9p-5), scalar(0x1.3b29dcb134a69p-7),
                 scalar(0x1.5d8a9fcfc7546p-10), scalar(0x1.4469d4b220e3bp-13), 0x1.fde1039ee67bfp-17};
  __device__ double operator()(double d) const {
    const double t = fmax(d, -700.0) * log2e, shifted = t + 6755399441055744.0;      // 1.5 * 2^52: a sum's low bits are the rounded number
    const double f = t - (shifted - 6755399441055744.0);
    double p = c[7];
#pragma unroll
    for (int i = 6; i >= 0; --i) p = __builtin_fma(p, f, c[i]);
    u32x2 u = __builtin_bit_cast(u32x2, p);
    u[1] += __builtin_bit_cast(u32x2, shifted)[0] << 20;   // (n, added to the exponent, in the upper word)
    return __builtin_bit_cast(double, u);
  }
};

// Sums of exp(x), |greatest x| <= 1024: exp(x) = 2^n 2^(k / 1024) e^r, n + k / 1024 + r / ln 2 = x log2(e), |r| <= ln 2 / 2048 and a little.  2^(k / 1024) comes from a table in LDS, in 64 bits; r and
// e^r - 1 = r + r^2 / 2 + .. take 32, which is enough because they are small: r twice and e^r - 1 once are off by half a step of 2^-35, 1.46e-11, and r^3 / 6 is at most 1e-11, so a term is off by
// 5.4e-11 of itself at most, and that is how far the logarithm of a chunk's sum may be off.  Vector instructions bound the launch, and one in 64 bits takes as long as two: 512 rows of 131072 bf16 logits take 43.9 us
// so, 49.5 with a parabola in 64 bits behind a table of 512, 52.6 with the polynomial of Exp; without any sum 30, the memory's 27 of them.  What lies more than 700 below the greatest, and NaN, counts as 700 below.
constexpr int kPowers = 1024;
// The upper words of the powers lack k << 10: an element's integer part, n and k, is added whole.
__device__ inline void fill_powers(double* powers) {
  static_assert(kPowers == 4 * kThreads, "four a thread");
  const double x = (double)threadIdx.x * (0.69314718055994530942 / kPowers);         // below 0.174: what is left out of the series is below 7e-15
  double p = 1.0 / 362880;
  const double c[9] = {1, 1, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040, 1.0 / 40320};
#pragma unroll
  for (int i = 8; i >= 0; --i) p = __builtin_fma(p, x, c[i]);
  const double quarter[4] = {1, 1.18920711500272106672, 1.41421356237309504880, 1.68179283050742908606};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = threadIdx.x + i * kThreads;
    u32x2 u = __builtin_bit_cast(u32x2, p * quarter[i]);
    u[1] -= k << 10;
    powers[k] = __builtin_bit_cast(double, u);
  }
}
struct NearSum {
  static constexpr float kShift = 12582912.f, kScale = 1477.3197f;       // 1.5 * 2^23: a sum's low bits are the rounded number; 1024 log2(e)
  const double* powers;
  float base, shift, lowest;                               // base: 1024 n of the greatest
  double sum = 0, rest = 0;
  __device__ NearSum(const double* powers, float top)
      : powers(powers), base(__int_as_float(__float_as_int(__builtin_fmaf(top, kScale, kShift)) & ~(kPowers - 1)) - kShift), shift(kShift - base), lowest(top - 700.f) {}
  __device__ void add(float x) {
    x = __builtin_amdgcn_fmed3f(x, lowest, FLT_MAX);       // (one instruction; the greater of two would be quieted first; of NaN and two others it is the lesser)
    const float shifted = __builtin_fmaf(x, kScale, shift), n = shifted - shift;
    const float r = __builtin_fmaf(n, 0x1.05c61p-39f, __builtin_fmaf(n, -0x1.62e43p-11f, x)), p = __builtin_fmaf(0.5f * r, r, r);       // ln 2 / 1024 in two parts
    const uint32_t i = __float_as_uint(shifted);           // (the shift's own bits lie above those that are used)
    u32x2 u = __builtin_bit_cast(u32x2, *reinterpret_cast<const double*>(reinterpret_cast<const char*>(powers) + (i << 3 & 8 * (kPowers - 1))));
    u[1] += i << 10;                                       // (to the exponent, in the upper word)
    const double power = __builtin_bit_cast(double, u);
    sum += power;
    rest = __builtin_fma(power, (double)p, rest);
  }
  // times exp(reference): the sum of exp(x)
  __device__ double all() const { return sum + rest; }
  __device__ double reference() const { return (double)base * (0.69314718055994530942 / kPowers); }
};

__device__ inline double sum_of_wave(double x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// E elements from `from` on, of which the first `each` are the thread's and those at 0 .. there - 1 the chunk's; the others count as -inf.  The row has those at 0 .. row_end - 1.  meanwhile: what else there is to do before they arrive.
template <class T, int E, class Meanwhile>
__device__ inline void load_row(const T* from, int there, int row_end, int each, float (&v)[E], Meanwhile meanwhile) {
  if (there >= each && row_end >= E) {
    constexpr int W = 16 / sizeof(T);
    struct __attribute__((packed, aligned(sizeof(T)))) Words { uint32_t w[4]; };     // (rows may begin at any element)
    Words r[E / W];
#pragma unroll
    for (int i = 0; i < E / W; ++i) r[i] = *reinterpret_cast<const Words*>(from + W * i);
    meanwhile();
#pragma unroll
    for (int i = 0; i < E / W; ++i) {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        if constexpr (sizeof(T) == 2) v[W * i + j] = __uint_as_float(j % 2 ? r[i].w[j / 2] & 0xffff0000u : r[i].w[j / 2] << 16);
        else v[W * i + j] = __uint_as_float(r[i].w[j]);
      }
    }
    if (each < E) {
#pragma unroll
      for (int i = 1; i < E; ++i) v[i] = i < each ? v[i] : -INFINITY;
    }
  } else {
    meanwhile();
#pragma unroll
    for (int i = 0; i < E; ++i) {                          // (those behind the row's last logit ask for that one: a load under a condition is waited for before the next is asked for)
      const float x = (float)from[min(i, row_end - 1)];
      v[i] = i < min(there, each) ? x : -INFINITY;
    }
  }
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = __builtin_canonicalizef(v[i]);      // (no signalling NaN: each fmaxf would see to that anew)
}

__device__ inline float wave_top(float x) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}

// The rank-th greatest (from 1) of the numbers that a wave holds, bit for bit from the top; reach(x): how many are x or more.  The bits below the lowest one to be looked at are ones where the sign's,
// the highest, is not set, else zeros: such are the orders of bf16 numbers.
template <class Reach>
__device__ inline uint32_t greatest(Reach reach, int rank, int lowest_bit) {
  uint32_t found = 0;
  for (int b = 31; b >= lowest_bit; --b) {
    const uint32_t next = found | 1u << b;
    if (reach(next) >= rank) found = next;
  }
  return found >> 31 ? found : found | ((1u << lowest_bit) - 1);
}

// The best `keep` of n elements that differ from each other, in order: best[0 .. min(n, keep) - 1].  Ranks by counting, Threads elements at a time, the best so far among them, several threads an element where
// there are few; at(i): element i.  room: Threads elements in LDS.  Every thread calls, best and room are free before, best is complete after.
template <int Threads, bool Several, class K, class Greater, class At>
__device__ inline void best_of(K* best, K* room, int n, int keep, Greater greater, At at) {
  int kept = 0;
  for (int from = 0; from < n;) {
    const int more = min(n - from, Threads - kept), all = kept + more, i = threadIdx.x;
    if (i < all) room[i] = i < kept ? best[i] : at(from + i - kept);
    __syncthreads();
    const int log_each = Several ? min(31 - __builtin_clz(Threads / all), 4) : 0, each = 1 << log_each, mine = i >> log_each;
    int above = 0;
    if (mine < all) {
      const K x = room[mine];
#pragma unroll 4
      for (int j = i & (each - 1); j < all; j += each) above += greater(room[j], x);
    }
    for (int d = 1; d < each; d *= 2) above += __shfl_xor(above, d);
    if (mine < all && above < keep && !(i & (each - 1))) best[above] = room[mine];
    __syncthreads();
    kept = min(all, keep);
    from += more;
  }
}

constexpr int kListed = 512;           // places of the list: counting takes about as long for so many as looking for the least logit that is offered

// Where more logits may be among the best than the list has places - a mask leaves few groups something, or logits are equal: the keep-th greatest logit, bit by bit, over all that the block holds; then
// exactly those beyond it, and of those equal to it the first.  How many are in the list.  reach: zeros.  (The logits are read again: kept in registers until here they
// cost all blocks, 512 rows of 131072 logits 48.5 us instead of 44.5.)
template <class T, int E>
__device__ inline int list_best(const T* from, int there, int row_end, int each, int keep, uint16_t* list, int32_t* reach, int32_t* sums_before, int32_t& listed) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t order[E], least = 0;
  float v[E];
  load_row<T, E>(from, there, row_end, each, v, [] {});
#pragma unroll
  for (int i = 0; i < E; ++i) order[i] = v[i] > -INFINITY ? order_of(fminf(v[i], FLT_MAX) + 0.f) : 0;
  for (int b = 31; b >= 0; --b) {
    const uint32_t next = least | 1u << b;
    int n = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) n += (int)__popcll(__ballot(order[i] >= next));
    if (lane == 0) atomicAdd(reach + b, n);
    __syncthreads();
    const int all = reach[b];
    if (all >= keep) least = next;
    if (all == keep) break;
  }
  int beyond = 0, equal = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    beyond += (int)__popcll(__ballot(order[i] > least));
    equal += order[i] == least && least > 0;
  }
  const int upto = wave_prefix_sum(equal);
  if (threadIdx.x == 0) listed = 0;
  __syncthreads();
  if (lane == 63) sums_before[wave] = upto;
  if (lane == 0) atomicAdd(&listed, beyond);
  __syncthreads();
  int rank = upto - equal + listed;                        // of the thread's first that is equal, behind those beyond
  int all = listed;
  for (int w = 0; w < kThreads / 64; ++w) {
    rank += w < wave ? sums_before[w] : 0;
    all += sums_before[w];
  }
  __syncthreads();
  if (threadIdx.x == 0) listed = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const uint16_t place = (uint16_t)(threadIdx.x * each + i);
    if (order[i] > least) list[atomicAdd(&listed, 1)] = place;
    else if (order[i] == least && least > 0 && rank < keep) list[rank++] = place;
  }
  __syncthreads();
  return min(all, keep);
}

template <class T, int E>
__global__ __launch_bounds__(kThreads, 7) void beam_rows_kernel(BeamArgs a) {
  __shared__ uint64_t room[kThreads], best[FCP_BEAM_MAX_KEEP];
  constexpr int kStaged = 8;           // threads of a wave whose logits are looked at together
  __shared__ __align__(16) float tops[kThreads];
  __shared__ __align__(16) float staged[kThreads / 64][kStaged * E];
  __shared__ int32_t staged_by[kThreads / 64][kStaged];
  __shared__ double sums[kThreads / 64], powers[kPowers];
  __shared__ int32_t listed;
  __shared__ uint16_t list[kListed];   // places in the chunk
  __shared__ int32_t reach[32], sums_before[kThreads / 64];
  // (The blocks of a die are every eighth: a row begins with its own number's chunk, so that chunks that a mask leaves more than others do not meet
  // in one die.  512 rows of 131072 with a mask that leaves tokens 4000 to 5500: 79 us, 230 else.)
  const int row = blockIdx.x / a.chunks, chunk = (blockIdx.x + row) % a.chunks, unit = row * a.chunks + chunk, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float score = a.score[row];
  if (!(score > -INFINITY) || (a.done && a.done[row])) return;           // offers nothing, or one candidate whatever its logits
  const int chunk0 = chunk * a.length, first = (int)threadIdx.x * a.each, there = min(a.length, a.vocab - chunk0) - first;
  float v[E];
  const T* const x = static_cast<const T*>(a.logits) + (int64_t)row * a.row + chunk0 + first;
  load_row<T, E>(x, there, a.vocab - chunk0 - first, a.each, v, [&] { fill_powers(powers); });
  float top = -INFINITY;
#pragma unroll
  for (int i = 0; i < E; ++i) top = fmaxf(top, v[i]);      // (NaN is passed over)
  const float own_top = fminf(top, FLT_MAX);
  tops[threadIdx.x] = top;
  if (threadIdx.x == 0) listed = 0;
  if (threadIdx.x < 32) reach[threadIdx.x] = 0;
  __syncthreads();
  const f32x4 four = *reinterpret_cast<const f32x4*>(tops + kPerGroup * lane);
  const float unbounded = fmaxf(fmaxf(four[0], four[1]), fmaxf(four[2], four[3])), mine = fminf(unbounded, FLT_MAX) + 0.f;         // (-0 as 0)
  const bool infinite = __ballot(unbounded == INFINITY);
  if (infinite) {                                          // rare
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = v[i] == INFINITY ? FLT_MAX : v[i];
  }
  // the keep-th greatest of the groups, or of the threads, of equal ones the lowest first, and its last thread
  const int lowest_bit = sizeof(T) == 2 && !infinite ? 16 : 0;
  uint32_t least;
  int at;
  // (of threads costs more, and leaves fewer to be counted: 96 rows of 32000, 64 kept, 49 us with groups, 22 so; with up to 32 kept about as many are left)
  if (a.keep <= kGroups / 2) {
    const uint32_t order = order_of(mine);
    least = greatest([&](uint32_t x) { return (int)__popcll(__ballot(order >= x)); }, a.keep, lowest_bit);
    uint64_t equal = __ballot(order == least);
    for (int k = a.keep - (int)__popcll(__ballot(order > least)); k > 1; --k) equal &= equal - 1;
    at = kPerGroup * __builtin_ctzll(equal) + kPerGroup - 1;
  } else {
    uint32_t order[kPerGroup];
#pragma unroll
    for (int i = 0; i < kPerGroup; ++i) order[i] = order_of(fminf(four[i], FLT_MAX) + 0.f);
    auto reach = [&](uint32_t x) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < kPerGroup; ++i) n += (int)__popcll(__ballot(order[i] >= x));
      return n;
    };
    least = greatest(reach, a.keep, lowest_bit);
    int equal = 0, need = a.keep;                          // of the lane; of all lanes
#pragma unroll
    for (int i = 0; i < kPerGroup; ++i) {
      equal += order[i] == least;
      need -= (int)__popcll(__ballot(order[i] > least));
    }
    const int upto = wave_prefix_sum(equal);
    const int found = __builtin_ctzll(__ballot(upto >= need));           // the lane that has the last one
    int last = 0, k = need - (upto - equal);
#pragma unroll
    for (int i = kPerGroup - 1; i >= 0; --i) last = order[i] == least && equal-- == k ? i : last;
    at = kPerGroup * found + __builtin_amdgcn_readlane(last, found);
  }
  const float border = value_of(least), most = wave_top(mine);
  double sum = 0, reference = 0;
  if (most > -INFINITY) {
    if (fabsf(most) <= 1024.f) {
      NearSum near(powers, most);
#pragma unroll
      for (int i = 0; i < E; ++i) near.add(v[i]);
      sum = near.all();
      reference = near.reference();
    } else {
      const Exp e;
#pragma unroll
      for (int i = 0; i < E; ++i) sum += e((double)v[i] - most);
      reference = most;
    }
    // Few threads have something for the list: the wave looks at all logits of eight of them at once.
    for (uint64_t who = __ballot(own_top >= border); who;) {
      const int place = (int)__popcll(who & (((uint64_t)1 << lane) - 1)), n = min((int)__popcll(who), kStaged);
      if ((who >> lane & 1) && place < kStaged) {
#pragma unroll
        for (int i = 0; i < E; i += 4) *reinterpret_cast<f32x4*>(&staged[wave][place * E + i]) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
        staged_by[wave][place] = threadIdx.x;
      }
      wave_exchange();
      for (int j = lane; j < n * E; j += 64) {
        const float x = staged[wave][j] + 0.f;
        const int by = staged_by[wave][j / E];
        // (the border itself counts in its own group and earlier ones)
        if ((x > border || (x == border && by <= at)) && x > -INFINITY) {
          const int k = atomicAdd(&listed, 1);
          if (k < kListed) list[k] = (uint16_t)(by * a.each + j % E);
        }
      }
      wave_exchange();
      for (int i = 0; i < n; ++i) who &= who - 1;
    }
  }
  sum = sum_of_wave(sum);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  int n = listed;
  if (__builtin_expect(n > kListed, false)) n = list_best<T, E>(x, there, a.vocab - chunk0 - first, a.each, a.keep, list, reach, sums_before, listed);
  // (the logits themselves are read again: with them the list would take four times the LDS, and fewer blocks would run at once)
  const T* const x0 = static_cast<const T*>(a.logits) + (int64_t)row * a.row + chunk0;
  best_of<kThreads, false>(best, room, n, a.keep, [](uint64_t x, uint64_t y) { return x > y; },
                    [&](int i) { return (uint64_t)order_of(fminf((float)x0[list[i]], FLT_MAX) + 0.f) << 32 | (uint32_t)~(chunk0 + list[i]); });
  if ((int)threadIdx.x < a.keep) a.lists[(int64_t)unit * a.keep + threadIdx.x] = (int)threadIdx.x < n ? best[threadIdx.x] : 0;
  if (threadIdx.x == 0) {
    a.sums[2 * (int64_t)unit] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    a.sums[2 * (int64_t)unit + 1] = reference;
  }
}

// A candidate: its score's order, then the beam and the token, both so that lower is greater.
struct Candidate { uint64_t score, place; };
__device__ inline bool greater(const Candidate& x, const Candidate& y) { return x.score > y.score || (x.score == y.score && x.place > y.place); }

constexpr int kJoinThreads = 1024, kJoined = 2;            // candidates that a thread holds

__global__ __launch_bounds__(kJoinThreads) void beam_join_kernel(BeamArgs a) {
  __shared__ Candidate found[FCP_BEAM_MAX_KEEP + kJoinThreads * kJoined], room[kJoinThreads];     // the best so far, then those that may replace them
  __shared__ double lse[FCP_BEAM_MAX_BEAMS];
  __shared__ uint32_t groups[kGroups];
  __shared__ Candidate best[FCP_BEAM_MAX_KEEP];
  __shared__ int32_t listed;
  const int row0 = blockIdx.x * a.beams, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lists = a.beams * a.chunks, all = lists * a.keep;            // (below 2^30: 2^24 chunks in all)
  // What a thread holds of the lists, asked for before the sums are joined: a logit of a beam, or its score where it is done.  All lists' best come first, then all lists' second best, and so on: what
  // follows a round is less than what was in it.
  uint64_t key[kJoined];
  int beam[kJoined];
  bool over[kJoined];
  auto ask = [&](int q0) {
#pragma unroll
    for (int i = 0; i < kJoined; ++i) {
      const uint32_t q = q0 + i * kJoinThreads + (int)threadIdx.x, rank = q < all ? q / (uint32_t)lists : 0, l = q < all ? q - rank * lists : 0, b = l / (uint32_t)a.chunks;
      const float score = a.score[row0 + b];
      const bool done = a.done && a.done[row0 + b];
      const bool offers = q < all && score > -INFINITY;
      const uint64_t k = a.lists[((int64_t)row0 * a.chunks + l) * a.keep + rank];
      beam[i] = b;
      over[i] = done;
      key[i] = !offers ? 0 : !done ? k : rank == 0 && l == b * a.chunks ? (uint64_t)(uint32_t)~a.end_token | (uint64_t)1 << 32 : 0;
    }
  };
  ask(0);
  // as many lanes join the sums of a beam as it has chunks, 64 at most
  const int log_lanes = a.chunks > 1 ? min(32 - __builtin_clz(a.chunks - 1), 6) : 0, lanes = 1 << log_lanes;
  for (int b = threadIdx.x >> log_lanes; b < a.beams; b += kJoinThreads >> log_lanes) {
    const float score = a.score[row0 + b];
    if (!(score > -INFINITY) || (a.done && a.done[row0 + b])) continue;
    const double* const sums = a.sums + 2 * (int64_t)(row0 + b) * a.chunks;
    const int first = threadIdx.x & (lanes - 1);
    double most = -INFINITY, sum = 0;
    for (int c = first; c < a.chunks; c += lanes)
      if (sums[2 * c] > 0) most = fmax(most, sums[2 * c + 1]);
    for (int d = 1; d < lanes; d *= 2) most = fmax(most, __shfl_xor(most, d));
    const Exp e;
    for (int c = first; c < a.chunks; c += lanes)
      if (sums[2 * c] > 0) sum += sums[2 * c] * e(sums[2 * c + 1] - most);
    for (int d = 1; d < lanes; d *= 2) sum += __shfl_xor(sum, d);
    if (first == 0) lse[b] = most + log(sum);
  }
  if (threadIdx.x < kGroups) groups[threadIdx.x] = 0;
  if (threadIdx.x == 0) listed = 0;
  __syncthreads();
  const Candidate none = {0, 0};
  int kept = 0;
  for (int q0 = 0; q0 < all; q0 += kJoinThreads * kJoined) {
    Candidate c[kJoined];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kJoined; ++i) {
      const double score = a.score[row0 + beam[i]];
      const double s = over[i] ? score : score + ((double)value_of((uint32_t)(key[i] >> 32)) - lse[beam[i]]);
      c[i] = key[i] ? Candidate{order_of(s), (uint64_t)(uint32_t)~beam[i] << 32 | (uint32_t)key[i]} : none;
      top = max(top, (uint32_t)(c[i].score >> 32));
    }
    if (q0 + kJoinThreads * kJoined < all) ask(q0 + kJoinThreads * kJoined);
    // The border, by the upper words of the scores' orders (20 bits of a mantissa): whatever reaches it may be among the best.  Groups are made so that a list's
    // elements, `lists` threads apart, lie in different ones, as far as that goes.
    atomicMax(groups + (lane + 5 * wave & kGroups - 1), top);
    __syncthreads();
    const uint32_t of_group = groups[lane];
    const uint32_t border = max(max(greatest([&](uint32_t x) { return (int)__popcll(__ballot(of_group >= x)); }, a.keep, 0), 1u), kept == a.keep ? (uint32_t)(best[kept - 1].score >> 32) : 0u);
#pragma unroll
    for (int i = 0; i < kJoined; ++i)
      if (__ballot((uint32_t)(c[i].score >> 32) >= border))
        if ((uint32_t)(c[i].score >> 32) >= border) found[kept + atomicAdd(&listed, 1)] = c[i];
    __syncthreads();
    const int n = kept + listed;
    if (n == kept && lists <= kJoinThreads * kJoined) break;             // (nor does anything follow)
    best_of<kJoinThreads, true>(best, room, n, a.keep, [](const Candidate& x, const Candidate& y) { return greater(x, y); }, [&](int i) { return found[i]; });
    kept = min(n, a.keep);
    if ((int)threadIdx.x < kept) found[threadIdx.x] = best[threadIdx.x];
    if (threadIdx.x < kGroups) groups[threadIdx.x] = 0;
    if (threadIdx.x == 0) listed = 0;
    __syncthreads();
  }
  if ((int)threadIdx.x < a.keep) {
    const bool there = (int)threadIdx.x < kept;
    const Candidate k = there ? best[threadIdx.x] : none;
    const int64_t at = (int64_t)blockIdx.x * a.keep + threadIdx.x;
    const int beam = (int)~(uint32_t)(k.place >> 32), token = (int)~(uint32_t)k.place;
    a.parent[at] = there ? row0 + beam : -1;
    a.token[at] = there ? token : -1;
    a.new_score[at] = there ? (float)score_of(k.score) : -INFINITY;
    if (a.new_done) a.new_done[at] = there && ((a.done && a.done[row0 + beam]) || (token >= 0 && token == a.end_token));
  }
}

// How a call is divided: chunks of up to 8192 logits where a row has more than 2048 and they make three blocks for two CUs, else of up to 2048; all chunks of a row are alike, so that every one has
// something for nearly all of its threads (1024 rows of 256000, 32 kept: 916 us where the last chunk had a quarter of the others').  2048 / 8192, bf16 but for the
// second: 4 rows of 32000 10.8 / 12.4 us, 8 prompts of 5 over 50001 fp32 13.8 / 14.2, 8 of 8 over 32000 13.9 / 14.1, 12 13.9 / 13.7, 16 17.6 / 15.1, 64 34.5 / 24.1; 4096 rows
// of 2000 25.6 / 34.7, of 5000 48.8 / 36.4.
struct BeamPlan { int32_t room, chunks, length, each; int64_t blocks; };        // room: logits that a thread has registers for
BeamPlan plan_beam(int64_t rows, int32_t vocab) {
  auto chunks = [&](int64_t each) { return (vocab + kThreads * each - 1) / (kThreads * each); };
  BeamPlan p;
  p.room = chunks(8) > 1 && rows * chunks(32) >= 384 ? 32 : 8;
  p.chunks = (int32_t)chunks(p.room);
  p.length = (int32_t)((vocab + (int64_t)p.chunks - 1) / p.chunks);
  p.each = (p.length + kThreads - 1) / kThreads;
  p.blocks = rows * p.chunks;
  return p;
}
size_t beam_bytes(const BeamPlan& p, int32_t keep) { return pad_to((size_t)p.blocks * keep * 8, 256) + pad_to((size_t)p.blocks * 16, 256); }

int check_beam(const char* who, int32_t n_prompts, int32_t beams, int32_t vocab, int32_t keep) {
  if (n_prompts < 0 || beams < 1 || vocab < 1 || keep < 1) return fail(FCP_ERR_INVALID_ARG, "%s: n_prompts must not be negative, beams, vocab and keep at least 1", who);
  if (beams > FCP_BEAM_MAX_BEAMS || keep > FCP_BEAM_MAX_KEEP)
    return fail(FCP_ERR_UNSUPPORTED, "%s: %d beams, %d kept; at most %d and %d", who, beams, keep, FCP_BEAM_MAX_BEAMS, FCP_BEAM_MAX_KEEP);
  if (vocab > 1 << 30) return fail(FCP_ERR_UNSUPPORTED, "%s: a vocabulary of more than 2^30", who);
  if ((int64_t)n_prompts * beams > INT32_MAX || !fits_axis((int64_t)n_prompts * beams * (((int64_t)vocab + 8191) / 8192), kThreads))
    return fail(FCP_ERR_UNSUPPORTED, "%s: 2^24 chunks of 8192 logits or more", who);
  return FCP_OK;
}

template <class T, int E>
int launch_rows(const BeamArgs& a, const BeamPlan& p, hipStream_t st) {
  beam_rows_kernel<T, E><<<dim3((unsigned)p.blocks), dim3(kThreads), 0, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  return FCP_OK;
}

}  // namespace
}  // namespace fcp

extern "C" size_t fcp_beam_scratch_bytes(int32_t n_prompts, int32_t beams, int32_t vocab, int32_t keep) {
  using namespace fcp;
  clear_error();
  if (check_beam("fcp_beam_scratch_bytes", n_prompts, beams, vocab, keep)) return 0;
  const size_t n = beam_bytes(plan_beam((int64_t)n_prompts * beams, vocab), keep);
  return n ? n : 256;
}

extern "C" int fcp_beam_select(const void* logits, int32_t type, int64_t logits_row, int32_t n_prompts, int32_t beams, int32_t vocab, const float* score,
                               const uint8_t* done, int32_t end_token, int32_t keep, int32_t* parent, int32_t* token, float* new_score,
                               uint8_t* new_done, void* scratch, size_t scratch_bytes, void* stream) {
  using namespace fcp;
  clear_error();
  const char* who = "fcp_beam_select";
  if (int rc = check_beam(who, n_prompts, beams, vocab, keep)) return rc;
  if (type != FCP_BF16 && type != FCP_F32) return fail(FCP_ERR_UNSUPPORTED, "%s: type %d is not known", who, type);
  if (end_token < -1 || end_token >= vocab) return fail(FCP_ERR_INVALID_ARG, "%s: end_token %d is neither -1 nor a token", who, end_token);
  if (n_prompts == 0) return FCP_OK;
  if (!logits || !score || !parent || !token || !new_score) return fail(FCP_ERR_INVALID_ARG, "%s: null argument", who);
  if (logits_row < vocab) return fail(FCP_ERR_INVALID_ARG, "%s: rows of logits overlap", who);
  if ((uintptr_t)logits % (type == FCP_BF16 ? 2 : 4) || (uintptr_t)score % 4 || (uintptr_t)parent % 4 || (uintptr_t)token % 4 || (uintptr_t)new_score % 4)
    return fail(FCP_ERR_INVALID_ARG, "%s: an argument is not aligned to its type", who);
  if (!scratch || (uintptr_t)scratch % 256) return fail(FCP_ERR_INVALID_ARG, "%s: scratch must be 256-byte aligned", who);
  const BeamPlan p = plan_beam((int64_t)n_prompts * beams, vocab);
  const size_t need = beam_bytes(p, keep);
  if (scratch_bytes < need) return fail(FCP_ERR_CAPACITY, "%s: scratch has %zu bytes, %zu are needed", who, scratch_bytes, need);
  const int64_t rows = (int64_t)n_prompts * beams, kept = (int64_t)n_prompts * keep, element = type == FCP_BF16 ? 2 : 4;
  if (int rc = check_apart(who, {{parent, 4 * kept}, {token, 4 * kept}, {new_score, 4 * kept}, {new_done, kept}, {scratch, (int64_t)need}},
                           {{logits, vocab * element, rows, rows > 1 ? logits_row * element : 0}, {score, 4 * rows}, {done, rows}}))
    return rc;
  BeamArgs a = {logits, logits_row, n_prompts * beams, beams, vocab, p.chunks, p.length, p.each, keep, end_token, score, done, parent, token, new_score, new_done};
  char* const at = static_cast<char*>(scratch);
  a.lists = reinterpret_cast<uint64_t*>(at);
  a.sums = reinterpret_cast<double*>(at + pad_to((size_t)p.blocks * keep * 8, 256));
  hipStream_t st = static_cast<hipStream_t>(stream);
  const bool bf16 = type == FCP_BF16;
  if (int rc = p.room == 32 ? (bf16 ? launch_rows<__bf16, 32>(a, p, st) : launch_rows<float, 32>(a, p, st))
                            : (bf16 ? launch_rows<__bf16, 8>(a, p, st) : launch_rows<float, 8>(a, p, st)))
    return rc;
  beam_join_kernel<<<dim3((unsigned)n_prompts), dim3(kJoinThreads), 0, st>>>(a);
  FCP_HIP_CHECK(hipGetLastError());
  return FCP_OK;
}
